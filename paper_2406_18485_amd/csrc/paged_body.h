// What the two kernels of paged attention share: the arguments, sums over a wave, page addresses, one tile's products and softmax,
// and how results are stored.
#pragma once
#include <hip/hip_runtime.h>

#include "device_utils.h"
#include "loong_internal.h"
#include "paged_params.h"
#include "split_exchange.h"

namespace loong {

constexpr float kRescaleSlack = 8.f;   // the running maximum may lag the true one by 2^8
// What is kept is the maximum less so much (log2): the largest probability is then 2^kRaise to 2^(kRaise + kRescaleSlack).  In half, whose
// steps end at 2^-24, 2^7: 10^5 keys of 2^-25 of the largest one's probability would else be lost from the product together, and not from the sum.
template <class E>
constexpr float kRaise = E::code == LOONG_FP16 ? 7.f : 0.f;

typedef __attribute__((address_space(3))) void lds_void_t;

// ---- sums over a wave, on the vector ALU (an exchange through LDS costs some 60 clocks a step) -----------------------
template <int CTRL, int ROWS>
__device__ __forceinline__ int from_lane(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false); }
// f over what lies before and at every lane; x of lanes that are not there counts as zero
template <class F>
__device__ __forceinline__ int wave_scan(int x, F f) {
  x = f(x, from_lane<0x111, 0xf>(x));   // one, two, four, eight lanes down inside a row of 16
  x = f(x, from_lane<0x112, 0xf>(x));
  x = f(x, from_lane<0x114, 0xf>(x));
  x = f(x, from_lane<0x118, 0xf>(x));
  x = f(x, from_lane<0x142, 0xa>(x));   // the last lane of a row to the next one
  return f(x, from_lane<0x143, 0xc>(x));
}
__device__ __forceinline__ int wave_prefix(int x) { return wave_scan(x, [](int a, int b) { return a + b; }); }
__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, 63); }
__device__ __forceinline__ int wave_total(int x) { return last_lane(wave_prefix(x)); }
__device__ __forceinline__ int wave_most(int x) { return last_lane(wave_scan(x, [](int a, int b) { return max(a, b); })); }   // (x >= 0)
__device__ __forceinline__ float wave_total(float x) {
  return __int_as_float(last_lane(wave_scan(__float_as_int(x), [](int a, int b) { return __float_as_int(__int_as_float(a) + __int_as_float(b)); })));
}

struct Seq { int start, n, rows, kv, paged; };   // first row; new tokens; query rows of a kv head; keys; those it has pages for
__device__ __forceinline__ Seq sequence(const PagedParams& p, int b) {
  Seq s;
  s.start = min(max(p.seq_start[b], 0), p.n_tokens);
  s.n = min(max(p.seq_start[b + 1], s.start), p.n_tokens) - s.start;
  s.rows = min(s.n, p.max_new) * p.G;
  s.kv = max(p.kv_len[b], 0);
  s.paged = min(s.kv, p.cap);
  return s;
}

// what a workgroup works on: a tile of a sequence's rows of one kv head
struct Unit { int b, hk, tile, start, n, rows, kv; };

// first key that row `row` of the unit's sequence does not see
__device__ __forceinline__ int limit_of(const PagedParams& p, const Unit& s, int row) {
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
// Before a loop over tiles: everything, also by the compiler's count, which else waits inside the loop for what it loaded before,
// and with that for tiles in flight.
__device__ __forceinline__ void wait_all_loads() {
  wait_vmcnt<0>();
  wait_loads<0>();
}
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// ---- pages -----------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t page_of(const PagedParams& p, uint32_t key) { return __umulhi(2 * key, p.page_mul) >> p.page_shift; }
// Where a key's row begins, in bytes from its head's first; page0: the first page in `win`.  (A slot's stride is below 2^32 bytes.)
__device__ __forceinline__ int64_t row_at(const PagedParams& p, const int64_t* win, int page0, int key) {
  const uint32_t page = page_of(p, key), slot = key - page * p.page_size;
  return win[(int)page - page0] + (int64_t)((uint64_t)slot * (uint32_t)(p.cs[2] * 2));
}
// keys whose pages are in LDS at a time
__device__ __forceinline__ int64_t window_keys(const PagedParams& p) { return (int64_t)(kWin - 2) * p.page_size / 128 * 128; }
// The workgroup's waves: where the pages of keys [k0, k1) begin, in bytes.  Barriers are the caller's.
__device__ __forceinline__ void fill_window(const PagedParams& p, int b, int k0, int k1, int64_t* win, int* first_bad) {
  const int p0 = (int)page_of(p, k0), n = (int)page_of(p, k1 - 1) - p0 + 1;
  for (int e = threadIdx.x; e < n; e += blockDim.x) {
    const int idx = p0 + e;
    const int page = idx < p.max_pages ? p.table[b * p.ts + idx] : -1;
    const bool ok = (uint32_t)page < (uint32_t)p.n_pages;
    win[e] = ok ? page * p.cs[0] * 2 : 0;
    if (!ok) atomicMin(first_bad, (int)min((int64_t)idx * p.page_size, (int64_t)0x7fffffff));
  }
}

// ---- masked tiles whose values are not all finite ---------------------------------------------------------------
// 0 x infinity is no zero: in tiles of which some row does not see all keys, values that are not finite are replaced by zeros
// (and noted in `odd_from`, the first key of the first such tile), and when all keys are done the rows that do see them get the
// infinity or NaN added.
template <class E>
__device__ __forceinline__ uint32_t finite_part(uint32_t x, uint32_t& odd) {
  // an exponent of all ones carries into the halves' sign bits
  const uint32_t m = ((x & 0x7fff7fffu) + (E::code == LOONG_FP16 ? 0x04000400u : 0x00800080u)) & 0x80008000u;
  odd |= m;
  return x & ~((m << 1) - (m >> 15));
}
// 16 bytes of a V tile whose first key is j0, in LDS, by the wave that loaded them
template <class E>
__device__ __forceinline__ void make_finite(unsigned char* piece, int j0, int* odd_from) {
  uint4 w = *reinterpret_cast<const uint4*>(piece);
  uint32_t odd = 0;
  w = make_uint4(finite_part<E>(w.x, odd), finite_part<E>(w.y, odd), finite_part<E>(w.z, odd), finite_part<E>(w.w, odd));
  if (odd) {
    *reinterpret_cast<uint4*>(piece) = w;
    atomicMin(odd_from, j0);
  }
}

// ---- one tile of BNS keys for a wave's 32 rows ------------------------------------------------------------------
template <int D>
struct RowState {
  float m, l;               // maximum less kRaise (log2 units), this half's sum
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

// The same in two registers, an instruction more a read, for tiles laid out by tile_swizzle (see device_utils.h).
template <int D>
struct PackedReads {
  uint32_t k_base, v_base;
  __device__ __forceinline__ PackedReads(int lane) : k_base(row_read_base<D>(lane)), v_base(tr_read_base<D>(lane)) {}
};
template <int D>
__device__ __forceinline__ const unsigned char* k_at(const unsigned char* Kt, const TileReads<D>& rd, int jb, int ks) { return Kt + jb * 64 * D + rd.k[ks]; }
template <int D>
__device__ __forceinline__ const unsigned char* k_at(const unsigned char* Kt, const PackedReads<D>& rd, int jb, int ks) {
  return Kt + jb * 64 * D + (rd.k_base ^ row_read_xor(ks));
}
template <int D>
__device__ __forceinline__ bf16x8_t v_frag(const unsigned char* Vt, const TileReads<D>& rd, int jb, int sl, int db) {
  const unsigned char* vp = Vt + (jb * 32 + sl * 16) * 2 * D + rd.v[db];
  return read_tr_pair(vp, vp + 16 * D);
}
template <int D>
__device__ __forceinline__ bf16x8_t v_frag(const unsigned char* Vt, const PackedReads<D>& rd, int jb, int sl, int db) {
  const unsigned char* vp = Vt + (jb * 32 + sl * 16) * 2 * D;
  return read_tr_pair(vp + (rd.v_base ^ tr_read_xor(db, 0)), vp + 16 * D + (rd.v_base ^ tr_read_xor(db, 1)));
}

// S^T = K Q^T of NJB x 32 keys; operands requested PF products ahead
template <class E, int D, int NJB, int PF, class Reads>
__device__ __forceinline__ void scores(const unsigned char* Kt, const Reads& rd, const bf16x8_t (&qf)[D / 16], floatx16_t (&s)[NJB]) {
  constexpr int NIT = D / 16 * NJB;
  auto k_frag = [&](int it) { return as_bf16x8(*reinterpret_cast<const uint4*>(k_at<D>(Kt, rd, it % NJB, it / NJB))); };
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

// online softmax with a lagging maximum; P^T as operand fragments, in one piece or in two: what the storage type holds of a probability,
// and what it holds of the rest.  Two leave o no further from 64 bits than its own rounding is (one: 1.35 times as far).  Few rows, whose
// matrix cores are idle for most of the time, have two: one sequence of 1000 keys 12.2 -> 12.7 us, 48 of up to 8192 137.5 -> 138.9.  Many
// rows have one, as the forward step: 2048 tokens over 32768 keys would be 1026 -> 1411 us.
template <class E, int D, int NJB, int PIECES>
__device__ __forceinline__ void softmax(const floatx16_t (&s)[NJB], float c, RowState<D>& st, uint4 (&pk)[PIECES][NJB][2]) {
  float mx = s[0][0];
#pragma unroll
  for (int jb = 0; jb < NJB; ++jb)
#pragma unroll
    for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[jb][v]);
  mx = max_with_other_half(mx);
  const float m_cand = fmaf(mx, c, -kRaise<E>);
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
      st.l += e[v];   // (the sum is of P before it is rounded)
    }
#pragma unroll
    for (int piece = 0; piece < PIECES; ++piece)
#pragma unroll
      for (int sl = 0; sl < 2; ++sl) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float &x = e[8 * sl + 2 * i], &y = e[8 * sl + 2 * i + 1];
          w[i] = E::pack2(x, y);
          if (piece + 1 < PIECES) { x -= E::lo(w[i]); y -= E::hi(w[i]); }
        }
        pk[piece][jb][sl] = make_uint4(w[0], w[1], w[2], w[3]);
      }
  }
}

// O^T += V^T P^T
template <class E, int D, int NJB, int PIECES, class Reads>
__device__ __forceinline__ void values(const unsigned char* Vt, const Reads& rd, const uint4 (&pk)[PIECES][NJB][2], RowState<D>& st) {
#pragma unroll
  for (int jb = 0; jb < NJB; ++jb)
#pragma unroll
    for (int sl = 0; sl < 2; ++sl) {
      if constexpr (PIECES == 1) {
#pragma unroll
        for (int db = 0; db < D / 32; ++db) st.o[db] = E::mfma(v_frag<D>(Vt, rd, jb, sl, db), as_bf16x8(pk[0][jb][sl]), st.o[db]);
      } else {   // (a product does not wait for the one before it)
        bf16x8_t v[D / 32];
#pragma unroll
        for (int db = 0; db < D / 32; ++db) v[db] = v_frag<D>(Vt, rd, jb, sl, db);
#pragma unroll
        for (int piece = 0; piece < PIECES; ++piece)
#pragma unroll
          for (int db = 0; db < D / 32; ++db) st.o[db] = E::mfma(v[db], as_bf16x8(pk[piece][jb][sl]), st.o[db]);
      }
    }
}

// Four of a key's values, those of a lane's half: f(element, value)
template <class E, class F>
__device__ __forceinline__ void four_values(const uint16_t* at, F f) {
  const uint2 w = *reinterpret_cast<const uint2*>(at);
  f(0, E::lo(w.x)); f(1, E::hi(w.x)); f(2, E::lo(w.y)); f(3, E::hi(w.y));
}
// A key's values of this half (the keys are below cap, so the table has their pages); NULL: a page outside the cache
__device__ __forceinline__ const uint16_t* values_of(const PagedParams& p, const Unit& s, int key, int hh) {
  const int idx = (int)page_of(p, key), page = p.table[s.b * p.ts + idx];
  if ((uint32_t)page >= (uint32_t)p.n_pages) return nullptr;
  return p.v + page * p.cs[0] + s.hk * p.cs[1] + (key - idx * p.page_size) * p.cs[2] + 4 * hh;
}
__device__ __forceinline__ float odd_part(float x) { return x - x == 0.f ? 0.f : x; }

// What the lane's row gets from values of keys [from, to) that are not finite and were left out.
template <class E, int D>
__device__ __forceinline__ void add_odd_values(const PagedParams& p, const Unit& s, int from, int to, int hh, RowState<D>& st) {
  for (int key = from; key < to; ++key) {
    const uint16_t* row = values_of(p, s, key, hh);
    if (!row) continue;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) four_values<E>(row + i * 8, [&](int e, float x) { st.o[i / 4][4 * (i % 4) + e] += odd_part(x); });
  }
}
// Infinite values are multiplied like others where every row sees them.  A probability that is zero in the storage type, or a second piece
// that is zero or negative, makes a NaN of them: rows that have one, and got no other from their scores, look for such values among their
// keys [from, to), and a column that has any is their sum.  By whole waves: lanes look at 64 keys at a time for those that have any.
// (Meanwhile the results are in `mem`, 128 D bytes of the wave's own LDS, where loops can index them: unrolled over registers, this made the
// code so long that calls which never come here took 0.5 to 1.3 us more.  A NaN that all see: 2048 tokens over 32768 keys 1.1 -> 2.8 ms.)
template <class E, int D>
__device__ __forceinline__ void settle_odd_values(const PagedParams& p, const Unit& s, int from, int to, int hh, RowState<D>& st, floatx4_t* mem) {
  float any[8] = {};   // (sums: NaN also where infinities of both signs meet; the search does no harm)
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) any[v % 8] += st.o[db][v];
  const float all = ((any[0] + any[1]) + (any[2] + any[3])) + ((any[4] + any[5]) + (any[6] + any[7]));
  bool looks = all != all && st.l == st.l;
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(looks) == 0, 1)) return;
  const int lane = lane_again(), end = wave_most(looks ? max(to, 0) : 0);
  floatx4_t* const mine = mem + lane;   // of 4 columns each, 64 apart
#pragma unroll
  for (int i = 0; i < D / 8; ++i) mine[i * 64] = floatx4_t{st.o[i / 4][4 * (i % 4)], st.o[i / 4][4 * (i % 4) + 1], st.o[i / 4][4 * (i % 4) + 2], st.o[i / 4][4 * (i % 4) + 3]};
  uint64_t met = 0, nan = 0;   // this lane's columns that have had one; those that are NaN by that, whatever comes
  for (int base = from; base < end && __builtin_amdgcn_ballot_w64(looks) != 0; base += 64) {
    uint32_t odd = 0;
    const uint16_t* row = base + lane < end ? values_of(p, s, base + lane, 0) : nullptr;
#pragma unroll 1
    for (int i = 0; i < (row ? D : 0); i += 32) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint4 w = *reinterpret_cast<const uint4*>(row + i + 8 * k);
        finite_part<E>(w.x, odd); finite_part<E>(w.y, odd); finite_part<E>(w.z, odd); finite_part<E>(w.w, odd);
      }
    }
    for (uint64_t keys = __builtin_amdgcn_ballot_w64(odd != 0); keys != 0; keys &= keys - 1) {
      const int key = base + __builtin_ctzll(keys);
      if (!looks || key >= to) continue;
      const uint16_t* at = values_of(p, s, key, hh);
#pragma unroll 1
      for (int i = 0; i < D / 8; ++i) {
        floatx4_t o = mine[i * 64];
        four_values<E>(at + i * 8, [&](int e, float x) {
          if (x - x == 0.f) return;
          const uint64_t bit = (uint64_t)1 << (4 * i + e);
          o[e] = met & bit ? o[e] + x : x;
          met |= bit;
          nan |= o[e] != o[e] ? bit : 0;
        });
        mine[i * 64] = o;
      }
      looks = ~nan << (64 - D / 2) != 0;
    }
  }
#pragma unroll
  for (int i = 0; i < D / 8; ++i) {
    const floatx4_t o = mine[i * 64];
#pragma unroll
    for (int e = 0; e < 4; ++e) st.o[i / 4][4 * (i % 4) + e] = o[e];
  }
}

template <int NJB>
__device__ __forceinline__ void mask_scores(floatx16_t (&s)[NJB], int j0, int limit, int hh) {
  const int left = limit - j0 - 4 * hh;   // keys of the tile that the row sees, from this half's first
#pragma unroll
  for (int jb = 0; jb < NJB; ++jb)
#pragma unroll
    for (int v = 0; v < 16; ++v) s[jb][v] = jb * 32 + acc_row(v, 0) < left ? s[jb][v] : -INFINITY;
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

}  // namespace loong
