// Attention of new tokens over a paged cache, on the 16-bit matrix cores.
//
// Rows.  The query rows of one kv head (new tokens x the group's q heads, token by token) are stacked, so that all of them share
// the keys that are read for them; a row's last visible key follows from its token.  As in the forward step, S^T = K Q^T puts a
// query row into one lane (softmax statistics in the lane, one exchange with the lane 32 places away) and the probabilities into
// the operand layout of O^T += V^T P^T.
//
// Two kernels.  few: up to 32 rows a kv head (decoding; a few drafted tokens).  Bound by HBM: 2 e head_dim bytes a key.  Every wave has
// keys and buffers of its own and waits for nobody; while one of its K and V tiles is used the other is on its way.
// many: 256 rows, eight waves of 32, on K/V tiles of 64 keys staged four deep for all of them, as in the forward step.  Bound by
// the matrix cores and what feeds them.
//
// Division of the work.  Lengths are in device memory, so the launch is made for what they may be at most and every wave works
// out the division from what they are: units (sequence, kv head, row tile) are cut into spans of keys, equal ones, so that
// all spans together are about as many as the chip takes at a time, however unequal the lengths.  A unit of several spans is
// added up by the last of them to arrive (split_exchange.h), in order.
//
// Pages.  The span's part of the page table lies in LDS (`win`), checked once: a number outside the cache becomes page 0,
// and rows that would see its keys are NaN at the end.  A lane finds the address of the piece that it stages from there.
#include <hip/hip_runtime.h>

#include <cmath>

#include "device_utils.h"
#include "loong_internal.h"
#include "split_exchange.h"

namespace loong {
namespace {

constexpr float kRescaleSlack = 8.f;   // the running maximum may lag the true one by 2^8
constexpr int kWin = 2048;             // page numbers in LDS
constexpr int kFewRows = 32, kManyRows = 256;
constexpr int kFewWaves = 4, kManyWaves = 8;

typedef __attribute__((address_space(3))) void lds_void_t;

struct PagedParams {
  const uint16_t *q, *k, *v;
  const int32_t *seq_start, *kv_len, *table;
  float *out, *lse;
  uint16_t* o;
  int64_t qs[2], os[2], cs[3], ts;
  int32_t n_seqs, n_tokens, max_new, hq, hkv, G;
  int32_t n_pages, max_pages, page_size;
  int32_t cap;          // keys that a row of the page table has pages for
  uint32_t page_mul;    // key / page_size = mulhi(2 key, page_mul) >> page_shift
  int32_t page_shift;
  float c;              // softmax_scale * log2(e)
  int32_t causal;
  int32_t spans;        // so many spans are aimed at
  int32_t least;        // keys of a span at the least
  uint32_t* counters;
  float* parts;
  int32_t slot_floats;
};

// ---- which span of which unit a workgroup works on ---------------------------------------------------------------
struct Span {
  int b, hk, tile;
  int start, n, rows;      // first row of the sequence's tokens; its new tokens; its query rows of a kv head
  int kv;                  // its keys, also those it has no pages for
  int keys;                // keys per span
  int part;                // number of this span among the unit's
  int slot;                // number of the unit's first span among those of all divided units
};

__device__ __forceinline__ int64_t wave_sum(int64_t x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m, 64);
  return x;
}
__device__ __forceinline__ int wave_scan(int x, int lane) {   // inclusive
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int y = __shfl_up(x, m, 64);
    x += lane >= m ? y : 0;
  }
  return x;
}

struct Seq { int start, n, rows, kv, paged; };   // paged: keys that it has pages for
__device__ __forceinline__ Seq sequence(const PagedParams& p, int b) {
  Seq s;
  s.start = min(max(p.seq_start[b], 0), p.n_tokens);
  s.n = min(max(p.seq_start[b + 1], s.start), p.n_tokens) - s.start;
  s.rows = min(s.n, p.max_new) * p.G;
  s.kv = max(p.kv_len[b], 0);
  s.paged = min(s.kv, p.cap);
  return s;
}

// Every wave for itself: lane l looks at sequences l, l + 64, ...
template <int ROWS>
__device__ __forceinline__ bool find_span(const PagedParams& p, uint32_t block, bool by_xcd, Span& out) {
  const int lane = threadIdx.x & 63;
  auto tiles_of = [](const Seq& s) { return (s.rows + ROWS - 1) / ROWS; };
  Seq mine{};
  if (lane < p.n_seqs) mine = sequence(p, lane);
  auto seq_at = [&](int base) {
    if (base == 0) return mine;
    Seq s{};
    if (base + lane < p.n_seqs) s = sequence(p, base + lane);
    return s;
  };
  int64_t load = 0;   // keys that are read, a tile's once
  for (int base = 0; base < p.n_seqs; base += 64) {
    const Seq s = seq_at(base);
    load += (int64_t)tiles_of(s) * s.paged;
  }
  load = wave_sum(load) * p.hkv;
  const int64_t even = ((load + p.spans - 1) / p.spans + 63) / 64 * 64;
  const int keys = (int)(even < p.least ? p.least : even > 0x7fffffc0 ? 0x7fffffc0 : even);
  auto parts_of = [&](const Seq& s) { return s.paged <= keys ? 1 : (int)(((int64_t)s.paged + keys - 1) / keys); };
  int64_t all = 0;
  for (int base = 0; base < p.n_seqs; base += 64) {
    const Seq s = seq_at(base);
    all += (int64_t)tiles_of(s) * parts_of(s);
  }
  all = wave_sum(all) * p.hkv;
  if (all > gridDim.x) return false;   // (more than there can be: seq_start decreases somewhere)
  // neighbours share an XCD and its L2 where they read the same keys
  int64_t item = block;
  if (by_xcd) {
    const int64_t per = (all + 7) / 8, idx = block >> 3;
    if (idx >= per) return false;
    item = (block & 7) * per + idx;
  }
  if (item >= all) return false;
  int64_t before = 0;
  int slot = 0;
  for (int base = 0; base < p.n_seqs; base += 64) {
    const Seq s = seq_at(base);
    const int parts = parts_of(s), n = tiles_of(s) * parts * p.hkv;
    const int upto = wave_scan(n, lane), slots = wave_scan(parts > 1 ? n : 0, lane);
    const uint64_t past = __builtin_amdgcn_ballot_w64(before + upto > item);
    if (past) {
      const int l = __builtin_ctzll(past);
      const int at = (int)(item - before) - (__shfl(upto, l, 64) - __shfl(n, l, 64));
      out.b = base + l;
      out.start = __builtin_amdgcn_readfirstlane(__shfl(s.start, l, 64));
      out.n = __builtin_amdgcn_readfirstlane(__shfl(s.n, l, 64));
      out.rows = __builtin_amdgcn_readfirstlane(__shfl(s.rows, l, 64));
      out.kv = __builtin_amdgcn_readfirstlane(__shfl(s.kv, l, 64));
      const int np = __builtin_amdgcn_readfirstlane(__shfl(parts, l, 64)), nt = (out.rows + ROWS - 1) / ROWS;
      const int at_s = __builtin_amdgcn_readfirstlane(at);
      out.keys = keys;
      out.hk = at_s / (np * nt);
      const int rest = at_s - out.hk * np * nt;
      out.part = rest / nt;
      out.tile = nt - 1 - (rest - out.part * nt);      // (the tiles that see most first)
      out.slot = slot + __builtin_amdgcn_readfirstlane(__shfl(slots, l, 64) - __shfl(parts > 1 ? n : 0, l, 64)) + (out.hk * nt + out.tile) * np;
      return true;
    }
    before += __shfl(upto, 63, 64);
    slot += __shfl(slots, 63, 64);
  }
  return false;
}

// first key that row `row` of a span's sequence does not see
__device__ __forceinline__ int limit_of(const PagedParams& p, const Span& s, int row) {
  if (!p.causal) return s.kv;
  const int64_t last = (int64_t)s.kv - s.n + row / p.G + 1;
  return last < 0 ? 0 : (int)last;
}

// Waits that the compiler moves no memory access across: without a barrier nothing else orders a tile's reads against its loads.
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N >= 0 && N < 64, "vmcnt has six bits");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// ---- pages -----------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t page_of(const PagedParams& p, uint32_t key) { return __umulhi(2 * key, p.page_mul) >> p.page_shift; }
// keys whose pages are in LDS at a time
__device__ __forceinline__ int64_t window_keys(const PagedParams& p) { return (int64_t)(kWin - 2) * p.page_size / 64 * 64; }
// The workgroup's waves: pages of keys [k0, k1).  Barriers are the caller's.
__device__ __forceinline__ void fill_window(const PagedParams& p, int b, int k0, int k1, int32_t* win, int* first_bad) {
  const int p0 = (int)page_of(p, k0), n = (int)page_of(p, k1 - 1) - p0 + 1;
  for (int e = threadIdx.x; e < n; e += blockDim.x) {
    const int idx = p0 + e;
    const int page = idx < p.max_pages ? p.table[b * p.ts + idx] : -1;
    const bool ok = (uint32_t)page < (uint32_t)p.n_pages;
    win[e] = ok ? page : 0;
    if (!ok) atomicMin(first_bad, (int)min((int64_t)idx * p.page_size, (int64_t)0x7fffffff));
  }
}

// ---- masked tiles whose values are not all finite ---------------------------------------------------------------
// 0 x infinity is no zero: in tiles of which some row does not see all keys, values that are not finite are taken out of the
// product (and noticed in `odd`), and when all keys are done the rows that do see them get the infinity or NaN added.
template <class E>
__device__ __forceinline__ uint32_t finite_part(uint32_t x, uint32_t& odd) {
  // an exponent of all ones carries into the halves' sign bits
  const uint32_t m = ((x & 0x7fff7fffu) + (E::code == LOONG_FP16 ? 0x04000400u : 0x00800080u)) & 0x80008000u;
  odd |= m;
  return x & ~((m << 1) - (m >> 15));
}
template <class E>
__device__ __forceinline__ bf16x8_t finite_part(bf16x8_t f, uint32_t& odd) {
  const uint4 w = __builtin_bit_cast(uint4, f);
  return as_bf16x8(make_uint4(finite_part<E>(w.x, odd), finite_part<E>(w.y, odd), finite_part<E>(w.z, odd), finite_part<E>(w.w, odd)));
}

// ---- one tile of BNS keys for a wave's 32 rows ------------------------------------------------------------------
template <int D>
struct RowState {
  float m, l;               // maximum (log2 units), this half's sum
  floatx16_t o[D / 32];     // O^T
  __device__ __forceinline__ void clear() {
    m = -INFINITY; l = 0.f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[db][v] = 0.f;
  }
};

// LDS read offsets of a lane inside a tile (laid out as in the forward step)
template <int D>
struct TileReads {
  static constexpr int ROWB = D * 2, CH = D / 8, RP = 256 / ROWB;
  uint32_t k[D / 16], v[D / 32];
  __device__ __forceinline__ TileReads(int lane) {
    const int l32 = lane & 31, hh = lane >> 5;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) k[ks] = l32 * ROWB + ((2 * ks + hh) ^ ((l32 / RP) & (CH - 1))) * 16;
    const int i16 = lane & 15, r = i16 >> 2, qd = i16 & 3, strip = (lane >> 4) & 1;
    const int sw = ((r / RP) & (4 / RP - 1)) * 4;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) v[db] = (4 * hh + r) * ROWB + ((db * 4 + strip * 2 + (qd >> 1)) ^ sw) * 16 + (qd & 1) * 8;
  }
};

// S^T = K Q^T of NJB x 32 keys; operands requested PF products ahead
template <class E, int D, int NJB, int PF>
__device__ __forceinline__ void scores(const unsigned char* Kt, const TileReads<D>& rd, const bf16x8_t (&qf)[D / 16], floatx16_t (&s)[NJB]) {
  constexpr int NIT = D / 16 * NJB, ROWB = D * 2;
  auto k_frag = [&](int it) { return as_bf16x8(*reinterpret_cast<const uint4*>(Kt + (it % NJB) * 32 * ROWB + rd.k[it / NJB])); };
  bf16x8_t ring[PF + 1];
  static_for<0, PF>([&](auto i) { ring[i.value] = k_frag(i.value); });
  floatx16_t zero;
#pragma unroll
  for (int v = 0; v < 16; ++v) zero[v] = 0.f;
  static_for<0, NIT>([&](auto i) {
    constexpr int it = i.value;
    if constexpr (it + PF < NIT) ring[(it + PF) % (PF + 1)] = k_frag(it + PF);
    __builtin_amdgcn_sched_barrier(0);
    s[it % NJB] = E::mfma(ring[it % (PF + 1)], qf[it / NJB], it < NJB ? zero : s[it % NJB]);
  });
}

// online softmax with a lagging maximum; P^T as operand fragments
template <class E, int D, int NJB>
__device__ __forceinline__ void softmax(const floatx16_t (&s)[NJB], float c, RowState<D>& st, uint4 (&pk)[NJB][2]) {
  float mx = s[0][0];
#pragma unroll
  for (int jb = 0; jb < NJB; ++jb)
#pragma unroll
    for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[jb][v]);
  mx = max_with_other_half(mx);
  const float m_cand = mx * c;
  if (__builtin_amdgcn_ballot_w64(m_cand > st.m + kRescaleSlack) != 0) {
    const float m_new = fmaxf(st.m, m_cand);
    const float alpha = m_new == -INFINITY ? 1.f : fast_exp2(st.m - m_new);
    st.l *= alpha;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) st.o[db][v] *= alpha;
    st.m = m_new;
  }
  const float m_use = st.m == -INFINITY ? 0.f : st.m;
#pragma unroll
  for (int jb = 0; jb < NJB; ++jb) {
    float e[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      e[v] = fast_exp2(fmaf(s[jb][v], c, -m_use));
      st.l += e[v];   // (P is rounded to the storage type for its product only)
    }
#pragma unroll
    for (int sl = 0; sl < 2; ++sl)
      pk[jb][sl] = make_uint4(E::pack2(e[8 * sl + 0], e[8 * sl + 1]), E::pack2(e[8 * sl + 2], e[8 * sl + 3]),
                              E::pack2(e[8 * sl + 4], e[8 * sl + 5]), E::pack2(e[8 * sl + 6], e[8 * sl + 7]));
  }
}

// O^T += V^T P^T.  `masked`: some row does not see some key of the tile
template <class E, int D, int NJB>
__device__ __forceinline__ void values(const unsigned char* Vt, const TileReads<D>& rd, const uint4 (&pk)[NJB][2], RowState<D>& st, bool masked,
                                       uint32_t& odd) {
  constexpr int ROWB = D * 2;
  auto product = [&](auto part_of) {
#pragma unroll
    for (int jb = 0; jb < NJB; ++jb)
#pragma unroll
      for (int sl = 0; sl < 2; ++sl)
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
          const unsigned char* vp = Vt + (jb * 32 + sl * 16) * ROWB + rd.v[db];
          st.o[db] = E::mfma(part_of(read_tr_pair(vp, vp + 8 * ROWB)), as_bf16x8(pk[jb][sl]), st.o[db]);
        }
  };
  if (masked) product([&](bf16x8_t f) { return finite_part<E>(f, odd); });
  else product([](bf16x8_t f) { return f; });
}

// What the lane's row gets from values of keys [from, to) that are not finite and were left out.
template <class E, int D>
__device__ __forceinline__ void add_odd_values(const PagedParams& p, const Span& s, int from, int to, int hh, RowState<D>& st) {
  for (int key = from; key < to; ++key) {
    const int idx = (int)page_of(p, key), page = p.table[s.b * p.ts + idx];   // (below cap, so the table has it)
    if ((uint32_t)page >= (uint32_t)p.n_pages) continue;
    const uint16_t* row = p.v + page * p.cs[0] + s.hk * p.cs[1] + (key - idx * p.page_size) * p.cs[2] + 4 * hh;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      const uint2 w = *reinterpret_cast<const uint2*>(row + i * 8);
      auto add = [&](int e, float x) { st.o[i / 4][4 * (i % 4) + e] += x - x == 0.f ? 0.f : x; };
      add(0, E::lo(w.x)); add(1, E::hi(w.x)); add(2, E::lo(w.y)); add(3, E::hi(w.y));
    }
  }
}

template <int NJB>
__device__ __forceinline__ void mask_scores(floatx16_t (&s)[NJB], int j0, int limit, int hh) {
#pragma unroll
  for (int jb = 0; jb < NJB; ++jb)
#pragma unroll
    for (int v = 0; v < 16; ++v) s[jb][v] = j0 + jb * 32 + acc_row(v, hh) < limit ? s[jb][v] : -INFINITY;
}

// ---- results ---------------------------------------------------------------------------------------------------
// A sum of nothing gives the neutral element; NaN stays NaN.
__device__ __forceinline__ float inverse_of(float l) { return l == 0.f ? 0.f : 1.f / l; }
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -INFINITY : (m + fast_log2(l)) * kLn2; }

template <class E>
__device__ __forceinline__ void store_out(const PagedParams& p, int token, int head, int col, float4 x) {
  const int64_t at = token * p.os[0] + head * p.os[1] + col;
  if (p.out) *reinterpret_cast<float4*>(p.out + at) = x;
  if (p.o) *reinterpret_cast<uint2*>(p.o + at) = make_uint2(E::pack2(x.x, x.y), E::pack2(x.z, x.w));
}

// (m, l) of a part, 8 bytes with device scope
__device__ __forceinline__ void store_ml(__amdgpu_buffer_rsrc_t buf, uint32_t off, float m, float l) {
  const uintx2_t w = {__float_as_uint(m), __float_as_uint(l)};
  __builtin_amdgcn_raw_buffer_store_b64(w, buf, off, 0, kDeviceScope);
}
__device__ __forceinline__ float2 load_ml(__amdgpu_buffer_rsrc_t buf, uint32_t off) {
  const uintx2_t w = __builtin_bit_cast(uintx2_t, __builtin_amdgcn_raw_buffer_load_b64(buf, off, 0, kDeviceScope));
  return make_float2(__uint_as_float(w[0]), __uint_as_float(w[1]));
}

// Running combination of partial results of a row: (m, l, x) += (m2, l2, y), x not normalised.
struct Joined {
  float m, l;
  floatx4_t x;
  __device__ __forceinline__ void add(float m2, float l2, floatx4_t y) {
    const float top = fmaxf(m, m2), ref = top == -INFINITY ? 0.f : top;
    const float a = fast_exp2(m - ref), b = fast_exp2(m2 - ref);
    l = l * a + l2 * b;
    x = x * a + y * b;
    m = top;
  }
};

// ================================================================================================================
// few rows: a workgroup of four waves, each with keys and LDS of its own; two workgroups a unit
// ================================================================================================================
template <int D>
struct FewCfg {
  static constexpr int BNS = 4096 / D;            // keys per tile: 8 KB
  static constexpr int NJB = BNS / 32, ROWB = D * 2, CH = D / 8, RP = 256 / ROWB, RPI = 1024 / ROWB, LI = 8;
  static constexpr int TILE_B = 8192, WAVE_B = 2 * TILE_B;
  static constexpr int COLS = D / 4;              // float4 columns of a row
};

template <class E, int D>
__global__ __launch_bounds__(kFewWaves * 64, 2) void paged_few_kernel(const PagedParams p) {
  using C = FewCfg<D>;
  constexpr int NT = kFewWaves * 64, NDB = D / 32, NJB = C::NJB, BNS = C::BNS;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kFewWaves * C::WAVE_B];
  __shared__ int32_t win[kWin];
  __shared__ float2 ml[kFewWaves][64];
  __shared__ int first_bad, odd_from, role;

  Span sp;
  if (!find_span<kFewRows>(p, blockIdx.x, false, sp)) return;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = min(l32, sp.rows - 1);
  const int head = sp.hk * p.G + row % p.G, token = sp.start + row / p.G;
  const int limit = limit_of(p, sp, row);
  const int seen = min(limit_of(p, sp, sp.rows - 1), p.cap), seen_by_all = limit_of(p, sp, 0);
  const int parts = seen <= sp.keys ? 1 : (int)(((int64_t)seen + sp.keys - 1) / sp.keys);
  if (sp.part >= parts) return;
  const int k0 = (int)min((int64_t)sp.part * sp.keys, (int64_t)seen), k1 = (int)min((int64_t)k0 + sp.keys, (int64_t)seen);

  bf16x8_t qf[D / 16];
  {
    const uint16_t* qrow = p.q + token * p.qs[0] + head * p.qs[1];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(qrow + ks * 16 + hh * 8));
  }
  if (tid == 0) { first_bad = p.cap; odd_from = 0x7fffffff; }

  const TileReads<D> rd(lane);
  unsigned char* const Kt = smem + wave * C::WAVE_B;
  const unsigned char* const Vt = Kt + C::TILE_B;
  const uint32_t k_lds = (uint32_t)(uintptr_t)(lds_void_t*)smem + wave * C::WAVE_B, v_lds = k_lds + C::TILE_B;
  const unsigned char* const kbase = reinterpret_cast<const unsigned char*>(p.k + sp.hk * p.cs[1]);
  const unsigned char* const vbase = reinterpret_cast<const unsigned char*>(p.v + sp.hk * p.cs[1]);
  const int ld_row = lane / C::CH, ld_pos = lane % C::CH;
  const int64_t page_b = p.cs[0] * 2, slot_b = p.cs[2] * 2;

  RowState<D> st;
  st.clear();
  const int64_t wkeys = window_keys(p);
  for (int64_t w0 = k0; w0 < k1; w0 += wkeys) {
    const int w1 = (int)min(w0 + wkeys, (int64_t)k1);
    __syncthreads();   // the last window's page numbers have been read (first time: first_bad is set)
    fill_window(p, sp.b, (int)w0, w1, win, &first_bad);
    __syncthreads();
    const int page0 = (int)page_of(p, (uint32_t)w0);
    const int tiles = (w1 - (int)w0 + BNS - 1) / BNS;
    int64_t off[C::LI];   // this lane's rows of a tile, bytes from the head's first
    auto place = [&](int t) {
#pragma unroll
      for (int i = 0; i < C::LI; ++i) {
        const int key = min((int)w0 + t * BNS + i * C::RPI + ld_row, w1 - 1);
        const int pg = (int)page_of(p, key);
        off[i] = win[pg - page0] * page_b + (key - pg * p.page_size) * slot_b;
      }
    };
    auto issue_k = [&] {
#pragma unroll
      for (int i = 0; i < C::LI; ++i) {
        const int r = i * C::RPI + ld_row;
        load_to_lds_16(kbase + off[i] + (ld_pos ^ ((r / C::RP) & (C::CH - 1))) * 16, k_lds + i * 1024);
      }
    };
    auto issue_v = [&] {
#pragma unroll
      for (int i = 0; i < C::LI; ++i) {
        const int r = i * C::RPI + ld_row;
        load_to_lds_16(vbase + off[i] + (ld_pos ^ (((r / C::RP) & (4 / C::RP - 1)) * 4)) * 16, v_lds + i * 1024);
      }
    };
    int t = wave;
    wait_loads<0>();   // (whatever the compiler has in flight)
    if (t < tiles) { place(t); issue_k(); issue_v(); }
    for (; t < tiles; t += kFewWaves) {
      const int j0 = (int)w0 + t * BNS;
      const bool more = t + kFewWaves < tiles, masked = j0 + BNS > min(seen_by_all, w1);
      wait_loads<C::LI>();   // K has landed when only V's loads are outstanding
      floatx16_t s[NJB];
      scores<E, D, NJB, 4>(Kt, rd, qf, s);
      if (more) {
        place(t + kFewWaves);
        wait_reads();   // (of K)
        issue_k();
      }
      if (masked) mask_scores<NJB>(s, j0, min(limit, w1), hh);
      uint4 pk[NJB][2];
      uint32_t odd = 0;
      softmax<E, D, NJB>(s, p.c, st, pk);
      if (more) wait_loads<C::LI>();
      else wait_loads<0>();
      values<E, D, NJB>(Vt, rd, pk, st, masked, odd);
      if (odd != 0) atomicMin(&odd_from, j0);
      if (more) {
        wait_reads();   // (of V)
        issue_v();
      }
    }
  }

  // ---- the waves' results, in wave order: wave w adds up columns 32 w .. + 31
  __syncthreads();   // (also: first_bad and odd_from are final)
  if (limit > first_bad) st.l = NAN;
  if (wave == 0) add_odd_values<E, D>(p, sp, odd_from, min(limit, k1), hh, st);   // (behind a masked tile all are)
  float4* const slots = reinterpret_cast<float4*>(smem);
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int vq = 0; vq < 4; ++vq)
      slots[((wave * NDB + db) * 4 + vq) * 64 + lane] = make_float4(st.o[db][4 * vq], st.o[db][4 * vq + 1], st.o[db][4 * vq + 2], st.o[db][4 * vq + 3]);
  ml[wave][lane] = make_float2(st.m, st.l);
  __syncthreads();
  float m_all = -INFINITY, l_all = 0.f, w[kFewWaves];
#pragma unroll
  for (int k = 0; k < kFewWaves; ++k) m_all = fmaxf(m_all, ml[k][lane].x);
  const float m_ref = m_all == -INFINITY ? 0.f : m_all;
#pragma unroll
  for (int k = 0; k < kFewWaves; ++k) {
    w[k] = fast_exp2(ml[k][lane].x - m_ref);
    l_all += ml[k][lane].y * w[k];
  }
  const float l_tot = sum_with_other_half(l_all);
  const bool ok = l32 < sp.rows;
  float4 acc[4];
  if (wave < NDB) {
#pragma unroll
    for (int vq = 0; vq < 4; ++vq) {
      acc[vq] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kFewWaves; ++k) {
        const float4 x = slots[((k * NDB + wave) * 4 + vq) * 64 + lane];
        acc[vq].x += x.x * w[k]; acc[vq].y += x.y * w[k]; acc[vq].z += x.z * w[k]; acc[vq].w += x.w * w[k];
      }
    }
  }
  if (parts == 1) {
    const float inv = inverse_of(l_tot);
    if (wave < NDB && ok) {
#pragma unroll
      for (int vq = 0; vq < 4; ++vq)
        store_out<E>(p, token, head, wave * 32 + 8 * vq + 4 * hh, make_float4(acc[vq].x * inv, acc[vq].y * inv, acc[vq].z * inv, acc[vq].w * inv));
      if (wave == 0 && hh == 0) p.lse[(int64_t)token * p.hq + head] = lse_of(m_all, l_tot);
    }
    return;
  }

  // ---- one of several spans: park [row][D], then (m, l) of the rows; the last to arrive adds all of them up
  constexpr uint32_t ML_AT = kFewRows * D * 4;
  {
    const __amdgpu_buffer_rsrc_t mine = part_buffer(p.parts + (int64_t)(sp.slot + sp.part) * p.slot_floats);
    if (wave < NDB && ok) {
#pragma unroll
      for (int vq = 0; vq < 4; ++vq) {
        const floatx4_t x = {acc[vq].x, acc[vq].y, acc[vq].z, acc[vq].w};
        store_part(mine, (uint32_t)(l32 * D + wave * 32 + 8 * vq + 4 * hh) * 4, x);
      }
      if (wave == 0 && hh == 0) store_ml(mine, ML_AT + l32 * 8, m_all, l_tot);
    }
  }
  wait_vmcnt<0>();
  __syncthreads();   // every wave's part is in memory, and the slots in LDS have been read
  if (tid == 0) role = arrive(p.counters + sp.slot, parts);
  __syncthreads();
  if (role == kLeaves) return;

  // threads: COLS float4 columns x rows (a power of two), and what is left of the workgroup shares the parts
  int rows2 = 1;
  while (rows2 < sp.rows) rows2 <<= 1;
  const int items = min(rows2 * C::COLS, NT), groups = NT / items, grp = tid / items;
  const __amdgpu_buffer_rsrc_t all = part_buffer(p.parts + (int64_t)sp.slot * p.slot_floats);
  Joined* const red = reinterpret_cast<Joined*>(smem);
  for (int base = 0; base < rows2 * C::COLS; base += items) {
    const int idx = base + tid % items, r = idx / C::COLS, col = idx % C::COLS;
    const int rr = min(r, sp.rows - 1);
    Joined j{-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
    constexpr int AHEAD = 8;
    for (int k = grp; k < parts; k += groups * AHEAD) {
      floatx4_t x[AHEAD];
      float2 s[AHEAD];
#pragma unroll
      for (int a = 0; a < AHEAD; ++a) {
        const uint32_t from = (uint32_t)min(k + a * groups, parts - 1) * (uint32_t)p.slot_floats * 4;   // (below 2^25)
        x[a] = load_part(all, from + (rr * D + col * 4) * 4);
        s[a] = load_ml(all, from + ML_AT + rr * 8);
      }
#pragma unroll
      for (int a = 0; a < AHEAD; ++a)
        if (k + a * groups < parts) j.add(s[a].x, s[a].y, x[a]);
    }
    if (groups > 1) {
      __syncthreads();
      red[tid] = j;
      __syncthreads();
      for (int g = 1; g < groups && grp == 0; ++g) j.add(red[tid + g * items].m, red[tid + g * items].l, red[tid + g * items].x);
    }
    if (grp == 0 && r < sp.rows) {
      if (role == kCountsWrong) j.l = NAN;
      const float inv = inverse_of(j.l);
      const int tk = sp.start + r / p.G, hd = sp.hk * p.G + r % p.G;
      store_out<E>(p, tk, hd, col * 4, make_float4(j.x[0] * inv, j.x[1] * inv, j.x[2] * inv, j.x[3] * inv));
      if (col == 0) p.lse[(int64_t)tk * p.hq + hd] = lse_of(j.m, j.l);
    }
  }
}

// ================================================================================================================
// many rows: eight waves of 32 rows on shared tiles of 64 keys
// ================================================================================================================
template <int D>
struct ManyCfg {
  static constexpr int BNS = 64, NJB = 2, ROWB = D * 2, CH = D / 8, RP = 256 / ROWB, RPI = 1024 / ROWB;
  static constexpr int TILE_B = BNS * ROWB, BUF_B = 2 * TILE_B, NBUF = 4, PD = NBUF - 1;
  static constexpr int KI = TILE_B / 1024 / kManyWaves;   // loads per wave and tile
};

template <class E, int D>
__global__ __launch_bounds__(kManyWaves * 64, 2) void paged_many_kernel(const PagedParams p) {
  using C = ManyCfg<D>;
  constexpr int NDB = D / 32, NJB = C::NJB, BNS = C::BNS, KI = C::KI, PD = C::PD, NBUF = C::NBUF;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[NBUF * C::BUF_B];
  __shared__ int32_t win[kWin];
  __shared__ int first_bad, role;

  Span sp;
  if (!find_span<kManyRows>(p, blockIdx.x, true, sp)) return;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row0 = sp.tile * kManyRows + wave * 32, tile_last = min((sp.tile + 1) * kManyRows, sp.rows) - 1;
  const bool wave_live = row0 < sp.rows, ok = row0 + l32 < sp.rows;
  const int row = min(row0 + l32, sp.rows - 1);
  const int head = sp.hk * p.G + row % p.G, token = sp.start + row / p.G;
  const int limit = limit_of(p, sp, row);
  const int seen = min(limit_of(p, sp, tile_last), p.cap);
  const int wave_all = limit_of(p, sp, min(row0, sp.rows - 1)), wave_any = limit_of(p, sp, min(row0 + 31, sp.rows - 1));
  const int parts = seen <= sp.keys ? 1 : (int)(((int64_t)seen + sp.keys - 1) / sp.keys);
  if (sp.part >= parts) return;
  const int k0 = (int)min((int64_t)sp.part * sp.keys, (int64_t)seen), k1 = (int)min((int64_t)k0 + sp.keys, (int64_t)seen);

  bf16x8_t qf[D / 16];
  {
    const uint16_t* qrow = p.q + token * p.qs[0] + head * p.qs[1];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(qrow + ks * 16 + hh * 8));
  }
  if (tid == 0) first_bad = p.cap;

  const TileReads<D> rd(lane);
  const uint32_t lds = (uint32_t)(uintptr_t)(lds_void_t*)smem;
  const unsigned char* const kbase = reinterpret_cast<const unsigned char*>(p.k + sp.hk * p.cs[1]);
  const unsigned char* const vbase = reinterpret_cast<const unsigned char*>(p.v + sp.hk * p.cs[1]);
  const int ld_row = wave * C::RPI + lane / C::CH, ld_pos = lane % C::CH;   // of load 0; later loads add 8 RPI rows
  const int64_t page_b = p.cs[0] * 2, slot_b = p.cs[2] * 2;

  RowState<D> st;
  st.clear();
  int odd_from = 0x7fffffff;
  const int64_t wkeys = window_keys(p);
  for (int64_t w0 = k0; w0 < k1; w0 += wkeys) {
    const int w1 = (int)min(w0 + wkeys, (int64_t)k1);
    __syncthreads();
    fill_window(p, sp.b, (int)w0, w1, win, &first_bad);
    __syncthreads();
    const int page0 = (int)page_of(p, (uint32_t)w0);
    const int tiles = (w1 - (int)w0 + BNS - 1) / BNS;
    auto issue = [&](int t) {
      const uint32_t kl = lds + (t % NBUF) * C::BUF_B + wave * 1024, vl = kl + C::TILE_B;
#pragma unroll
      for (int i = 0; i < KI; ++i) {
        const int r = ld_row + i * 8 * C::RPI;
        const int key = min((int)w0 + t * BNS + r, w1 - 1);
        const int pg = (int)page_of(p, key);
        const int64_t off = win[pg - page0] * page_b + (key - pg * p.page_size) * slot_b;
        load_to_lds_16(kbase + off + (ld_pos ^ ((r / C::RP) & (C::CH - 1))) * 16, kl + i * 8192);
        load_to_lds_16(vbase + off + (ld_pos ^ (((r / C::RP) & (4 / C::RP - 1)) * 4)) * 16, vl + i * 8192);
      }
    };
    wait_vmcnt<0>();   // (whatever the compiler has in flight)
#pragma unroll
    for (int t = 0; t < PD; ++t)
      if (t < tiles) issue(t);
    for (int t = 0; t < tiles; ++t) {
      const int later = min(PD - 1, tiles - 1 - t);
      if (later >= 2) wait_vmcnt<2 * 2 * KI>();
      else if (later == 1) wait_vmcnt<2 * KI>();
      else wait_vmcnt<0>();
      __syncthreads();   // every wave's part of the tile is in LDS; everyone has finished the one before
      if (t + PD < tiles) issue(t + PD);
      const int j0 = (int)w0 + t * BNS;
      if (!wave_live || j0 >= wave_any) continue;
      const unsigned char* const Kt = smem + (t % NBUF) * C::BUF_B;
      const bool masked = j0 + BNS > min(wave_all, w1);
      floatx16_t s[NJB];
      scores<E, D, NJB, D == 128 ? 6 : 4>(Kt, rd, qf, s);
      if (masked) mask_scores<NJB>(s, j0, min(limit, w1), hh);
      uint4 pk[NJB][2];
      softmax<E, D, NJB>(s, p.c, st, pk);
      uint32_t odd = 0;
      values<E, D, NJB>(Kt + C::TILE_B, rd, pk, st, masked, odd);
      if (__builtin_amdgcn_ballot_w64(odd != 0) != 0) odd_from = min(odd_from, j0);
    }
  }
  __syncthreads();   // first_bad is final
  if (limit > first_bad) st.l = NAN;
  add_odd_values<E, D>(p, sp, odd_from, min(limit, k1), hh, st);   // (behind a masked tile all are)

  float l_tot = sum_with_other_half(st.l);
  if (parts > 1) {
    // park in accumulator layout: [wave][16-byte piece][lane], then (m, l) by [wave][lane]; the last to arrive adds them up in order
    constexpr int PIECES = NDB * 4;
    constexpr uint32_t ML_AT = kManyRows * D * 4;
    float* const first = p.parts + (int64_t)sp.slot * p.slot_floats;
    const uint32_t at = (uint32_t)(wave * PIECES * 64 + lane) * 16, ml_at = ML_AT + (uint32_t)(wave * 64 + lane) * 8;
    if (wave_live) {
      const __amdgpu_buffer_rsrc_t mine = part_buffer(first + (int64_t)sp.part * p.slot_floats);
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const floatx4_t x = {st.o[i / 4][4 * (i % 4)], st.o[i / 4][4 * (i % 4) + 1], st.o[i / 4][4 * (i % 4) + 2], st.o[i / 4][4 * (i % 4) + 3]};
        store_part(mine, at + i * 1024, x);
      }
      store_ml(mine, ml_at, st.m, l_tot);
    }
    wait_vmcnt<0>();
    __syncthreads();
    if (tid == 0) role = arrive(p.counters + sp.slot, parts);
    __syncthreads();
    if (role == kLeaves || !wave_live) return;
    float m_all = -INFINITY;
    for (int k = 0; k < parts; ++k) m_all = fmaxf(m_all, load_ml(part_buffer(first + (int64_t)k * p.slot_floats), ml_at).x);
    const float m_ref = m_all == -INFINITY ? 0.f : m_all;
    st.clear();
    l_tot = 0.f;
    for (int k = 0; k < parts; ++k) {
      const __amdgpu_buffer_rsrc_t buf = part_buffer(first + (int64_t)k * p.slot_floats);
      const float2 s = load_ml(buf, ml_at);
      const float w = fast_exp2(s.x - m_ref);
      l_tot += s.y * w;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const floatx4_t x = load_part(buf, at + i * 1024);
#pragma unroll
        for (int e = 0; e < 4; ++e) st.o[i / 4][4 * (i % 4) + e] += x[e] * w;
      }
    }
    st.m = m_all;
    if (role == kCountsWrong) l_tot = NAN;
  }
  if (!ok) return;
  const float inv = inverse_of(l_tot);
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int vq = 0; vq < 4; ++vq)
      store_out<E>(p, token, head, db * 32 + 8 * vq + 4 * hh,
                   make_float4(st.o[db][4 * vq] * inv, st.o[db][4 * vq + 1] * inv, st.o[db][4 * vq + 2] * inv, st.o[db][4 * vq + 3] * inv));
  if (hh == 0) p.lse[(int64_t)token * p.hq + head] = lse_of(st.m, l_tot);
}

// ---- host ------------------------------------------------------------------------------------------------------
struct PagedPlan {
  bool few;
  int spans, least;
  int64_t workgroups;      // units that there may be, and the spans that divided ones have more
  int64_t slots;           // spans of divided units at the most
  int slot_floats;
};

// Keys that a sequence has pages for (kv_len is an int32).
int64_t cached_keys(const loong_paged_desc& d) {
  const int64_t n = (int64_t)d.max_pages * d.page_size;
  return n < 0x7fffffff ? n : 0x7fffffff;
}

// Every divided unit has more keys than a span, and spans are as long as makes `spans` of them cover all keys: there are at most
// `spans` of them and a remainder a unit, and at most as many units are divided.
PagedPlan plan_paged(const loong_paged_desc& d, int cus) {
  PagedPlan pl{};
  const int64_t g = d.n_q_heads / d.n_kv_heads, new_most = d.max_new < d.n_tokens ? d.max_new : d.n_tokens;
  pl.few = new_most * g <= kFewRows;
  const int rows = pl.few ? kFewRows : kManyRows;
  const int64_t seqs = d.n_seqs < d.n_tokens ? d.n_seqs : d.n_tokens;
  int64_t units = seqs;
  if (!pl.few) units += d.n_tokens * g / rows;
  units *= d.n_kv_heads;
  pl.spans = (pl.few ? 4 : 2) * cus;
  pl.least = pl.few ? 256 : 512;
  const int64_t most_keys = cached_keys(d);
  const int64_t per_unit = most_keys <= pl.least ? 1 : (most_keys + pl.least - 1) / pl.least;
  pl.workgroups = units + pl.spans;
  if (units * per_unit < pl.workgroups) pl.workgroups = units * per_unit;
  pl.workgroups = (pl.workgroups + 7) / 8 * 8;
  pl.slots = per_unit == 1 ? 0 : 2 * (int64_t)pl.spans < pl.workgroups ? 2 * (int64_t)pl.spans : pl.workgroups;
  pl.slot_floats = rows * (d.head_dim + (pl.few ? 2 : 4));
  return pl;
}
int64_t workspace_of(const PagedPlan& pl) { return pl.slots ? kWsHeadBytes + pl.slots * pl.slot_floats * 4 : 0; }

int check_attn(const loong_paged_desc* d) {
  if (int rc = check_paged(d, LOONG_WORKSPACE_CLEAN)) return rc;
  if (!std::isfinite(d->softmax_scale) || d->softmax_scale <= 0.f) return fail(LOONG_E_SHAPE, "softmax_scale must be finite and positive");
  return LOONG_OK;
}

template <class E, int D>
void launch_paged(const PagedParams& p, bool few, unsigned grid, hipStream_t st) {
  if (few) paged_few_kernel<E, D><<<dim3(grid), dim3(kFewWaves * 64), 0, st>>>(p);
  else paged_many_kernel<E, D><<<dim3(grid), dim3(kManyWaves * 64), 0, st>>>(p);
}

}  // namespace
}  // namespace loong

using namespace loong;

extern "C" {

int loong_paged_workspace_bytes(const loong_paged_desc* desc, int64_t* bytes) {
  clear_error();
  if (!bytes) return fail(LOONG_E_NULL, "loong_paged_workspace_bytes: NULL result");
  if (int rc = check_attn(desc)) return rc;
  *bytes = workspace_of(plan_paged(*desc, planning_cus()));
  return LOONG_OK;
}

int loong_paged_attn(const loong_paged_desc* desc, const void* q, const void* k_cache, const void* v_cache, const int32_t* seq_start,
                     const int32_t* kv_len, const int32_t* page_table, float* out, void* o, float* lse, void* workspace,
                     int64_t workspace_bytes, void* stream) {
  clear_error();
  if (int rc = check_attn(desc)) return rc;
  const loong_paged_desc& d = *desc;
  if (!q || !k_cache || !v_cache || !seq_start || !kv_len || !page_table || !lse || (!out && !o)) return fail(LOONG_E_NULL, "loong_paged_attn: NULL argument");
  for (const void* x : {q, k_cache, v_cache, (const void*)out, (const void*)o, (const void*)workspace})
    if (!aligned16(x)) return fail(LOONG_E_ALIGN, "loong_paged_attn: tensor not 16-byte aligned");
  for (const void* x : {(const void*)seq_start, (const void*)kv_len, (const void*)page_table, (const void*)lse})
    if (reinterpret_cast<uintptr_t>(x) & 3) return fail(LOONG_E_ALIGN, "loong_paged_attn: table or lse not 4-byte aligned");
  if (d.n_tokens == 0 || d.n_seqs == 0 || d.max_new == 0) return LOONG_OK;
  if (d.n_pages == 0) return fail(LOONG_E_SHAPE, "loong_paged_attn: a cache without pages");
  DeviceFacts dev;
  if (int rc = device_facts(&dev)) return rc;
  const PagedPlan pl = plan_paged(d, dev.cus);
  const int64_t need = workspace_of(pl);
  if (need > 0) {
    if (!workspace) return fail(LOONG_E_NULL, "loong_paged_attn: NULL workspace");
    if (workspace_bytes < need)
      return fail(LOONG_E_SHAPE, "loong_paged_attn: workspace of %lld bytes, %lld are needed", (long long)workspace_bytes, (long long)need);
  }
  if (!launch_fits(pl.workgroups, kManyWaves * 64)) return fail(LOONG_E_UNSUPPORTED, "loong_paged_attn: grid too large");
  PagedParams p{};
  p.q = (const uint16_t*)q; p.k = (const uint16_t*)k_cache; p.v = (const uint16_t*)v_cache;
  p.seq_start = seq_start; p.kv_len = kv_len; p.table = page_table;
  p.out = out; p.lse = lse; p.o = (uint16_t*)o;
  for (int i = 0; i < 2; ++i) { p.qs[i] = d.q_stride[i]; p.os[i] = d.o_stride[i]; }
  for (int i = 0; i < 3; ++i) p.cs[i] = d.cache_stride[i];
  p.ts = d.table_stride;
  p.n_seqs = d.n_seqs; p.n_tokens = d.n_tokens; p.max_new = d.max_new; p.hq = d.n_q_heads; p.hkv = d.n_kv_heads; p.G = d.n_q_heads / d.n_kv_heads;
  p.n_pages = d.n_pages; p.max_pages = d.max_pages; p.page_size = d.page_size;
  p.cap = (int32_t)cached_keys(d);
  // 2^(31 + s) / page_size rounded up, s = ceil(log2 page_size): exact for keys below 2^31
  int s = 0;
  while ((1 << s) < d.page_size) ++s;
  p.page_shift = s;
  p.page_mul = (uint32_t)((((uint64_t)1 << (31 + s)) + d.page_size - 1) / d.page_size);
  p.c = d.softmax_scale * kLog2e; p.causal = d.causal != 0;
  p.spans = pl.spans; p.least = pl.least;
  p.counters = static_cast<uint32_t*>(workspace);
  p.parts = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + kWsHeadBytes);
  p.slot_floats = pl.slot_floats;
  if (need > 0 && !(d.flags & LOONG_WORKSPACE_CLEAN))
    if (int rc = launch_clear_head(workspace, stream)) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const unsigned grid = (unsigned)pl.workgroups;
  if (d.dtype == LOONG_BF16) {
    if (d.head_dim == 128) launch_paged<Bf16, 128>(p, pl.few, grid, st);
    else launch_paged<Bf16, 64>(p, pl.few, grid, st);
  } else {
    if (d.head_dim == 128) launch_paged<Fp16, 128>(p, pl.few, grid, st);
    else launch_paged<Fp16, 64>(p, pl.few, grid, st);
  }
  return check_launch("loong_paged_attn");
}

}  // extern "C"
