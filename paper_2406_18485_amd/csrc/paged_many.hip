// Paged attention of many rows (a chunk of a prompt, alone or beside decoding sequences).
//
// Bound by the matrix cores and what feeds them, like the forward step (attn_fwd.hip), whose loop this is: eight waves = 8 / KS blocks
// of 32 rows x KS key splits; a tile of K and V is staged for all of them, several tiles deep.  The query rows of a kv head (token by
// token, the group's q heads of each) are cut into tiles of 256 / KS.
//
// Division.  A unit (sequence, kv head, row tile) may be cut into spans of keys, which are added up by the last of them to arrive
// (split_exchange.h), kManyFan at a time.  Tiles of 256 rows use the matrix cores best (KS = 1: 1030 to 1090 TFLOP/s over long contexts,
// KS = 2 840, KS = 4 640 to 710), but where there are fewer of them than units of the chip either they are cut, which costs an exchange of
// 128 KB a span, or the tiles are made smaller.  Which is faster goes by the lengths, which are in device memory: every wave works out,
// for the three tiles and for a few lengths of a span, how many spans there would be and about how long they would take, and all take
// the best.  (1000 tokens, 8 heads on 2, KS = 1 / 2 / 4 in us: over 1000 keys 27 / 22 / 22, 6000 53 / 55 / 54, 16000 90 / 100 / 110, 64000
// 271 / 312 / 365; with the choice 20, 49, 93, 272.  Beside eight decoding sequences, 6000 keys: 59 / 52 / 64, with it 52.5.)
//
// 2048 tokens over 32768 keys, 32 heads on 8: 995 to 1050 us by the box's clock (1020 to 1080 TFLOP/s, the matrix cores busy for 51 % of
// their cycles); what keeps them waiting is the vector work of the softmax, as in the forward step.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "paged_body.h"
#include "paged_division.h"

namespace loong {
namespace {

constexpr int kManyWaves = 8;
constexpr int kManyLevels = 6;         // 4^6 parts are more than a unit has

struct ManySpan {
  Unit u;
  int part;
  int slot;                // number of the unit's first span among those of all cut units
};

// The sequences, 64 at a time: a lane looks at base + lane.
struct Lanes {
  Seq mine;
  __device__ __forceinline__ Lanes(const PagedParams& p) : mine{} {
    const int lane = threadIdx.x & 63;
    if (lane < p.n_seqs) mine = sequence(p, lane);
  }
  __device__ __forceinline__ Seq at(const PagedParams& p, int base) const {
    Seq s = mine;
    if (base > 0) {
      const int b = base + (threadIdx.x & 63);
      s = Seq{};
      if (b < p.n_seqs) s = sequence(p, b);
    }
    return s;
  }
};
__device__ __forceinline__ int tiles_of(const Seq& s, int rows) { return row_tiles(s.rows, rows); }
__device__ __forceinline__ int parts_of(const Seq& s, int keys) { return key_parts(s.paged, keys); }

// What the division asks of all sequences, by a wave.
struct WaveSums {
  const PagedParams& p;
  const Lanes& lanes;
  static __device__ __forceinline__ float rcp(float x) { return __builtin_amdgcn_rcpf(x); }
  __device__ __forceinline__ int longest() const {
    int most = 0;
    for (int base = 0; base < p.n_seqs; base += 64) {
      const Seq s = lanes.at(p, base);
      most = max(most, s.rows ? s.paged : 0);
    }
    return wave_most(most);
  }
  __device__ __forceinline__ void tiles(int rows, float& load, float& units) const {
    load = units = 0.f;
    for (int base = 0; base < p.n_seqs; base += 64) {
      const Seq s = lanes.at(p, base);
      const float t = (float)tiles_of(s, rows);
      load += t * (float)s.paged;
      units += t;
    }
    load = wave_total(load);
    units = wave_total(units);
  }
  __device__ __forceinline__ float spans(int rows, float inv) const {
    float n = 0.f;
    for (int base = 0; base < p.n_seqs; base += 64) {
      const Seq s = lanes.at(p, base);
      n += (float)tiles_of(s, rows) * fmaxf(ceilf((float)s.paged * inv - 1e-4f), 1.f);
    }
    return wave_total(n);
  }
  __device__ __forceinline__ int all(const Division& d) const {
    int n = 0;
    for (int base = 0; base < p.n_seqs && !d.none; base += 64) {
      const Seq s = lanes.at(p, base);
      n += tiles_of(s, d.rows) * parts_of(s, d.keys);
    }
    return wave_total(n) * p.hkv;
  }
};

__device__ __forceinline__ bool find_span(const PagedParams& p, const Division& d, const Lanes& lanes, int item, ManySpan& out) {
  int before = 0, slot = 0;
  for (int base = 0; base < p.n_seqs; base += 64) {
    const Seq s = lanes.at(p, base);
    const int parts = parts_of(s, d.keys), n = tiles_of(s, d.rows) * parts * p.hkv, cut = parts > 1 ? n : 0;
    const int upto = wave_prefix(n), slots = wave_prefix(cut);
    const uint64_t past = __builtin_amdgcn_ballot_w64(before + upto > item);
    if (past) {
      const int l = __builtin_ctzll(past);
      const int at = item - before - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(n, l));
      out.u.b = base + l;
      out.u.start = __builtin_amdgcn_readlane(s.start, l); out.u.n = __builtin_amdgcn_readlane(s.n, l);
      out.u.rows = __builtin_amdgcn_readlane(s.rows, l); out.u.kv = __builtin_amdgcn_readlane(s.kv, l);
      const int np = __builtin_amdgcn_readlane(parts, l), nt = tiles_of(Seq{0, 0, out.u.rows, 0, 0}, d.rows);
      out.u.hk = at / (np * nt);
      const int rest = at - out.u.hk * np * nt;
      out.part = rest / nt;
      out.u.tile = nt - 1 - (rest - out.part * nt);      // (the tiles that see most first)
      out.slot = slot + __builtin_amdgcn_readlane(slots, l) - __builtin_amdgcn_readlane(cut, l) + (out.u.hk * nt + out.u.tile) * np;
      return true;
    }
    before += last_lane(upto);
    slot += last_lane(slots);
  }
  return false;
}

template <int D, int KS>
struct ManyCfg {
  static constexpr int NRB = kManyWaves / KS, ROWS = 32 * NRB;
  static constexpr int BNS = KS == 1 ? 64 : 32, TK = KS * BNS, NJB = BNS / 32, NDB = D / 32;   // keys of a wave, of a tile
  static constexpr int ROWB = D * 2, CH = D / 8, RP = 256 / ROWB, RPI = 1024 / ROWB;
  static constexpr int TILE_B = TK * ROWB, BUF_B = 2 * TILE_B, NBUF = BUF_B * 4 <= 131072 ? 4 : 2, PD = NBUF - 1;
  static constexpr int KI = TILE_B / 1024 / kManyWaves;   // loads per wave and tile
  static constexpr int DBW = (NDB + KS - 1) / KS;         // 32-column blocks that a wave adds up
  static constexpr int SLOT_F4 = NDB * 4 + 1;
  static constexpr int COMB_B = KS > 1 ? kManyWaves * SLOT_F4 * 64 * 16 : 0;
  static constexpr int SMEM_B = NBUF * BUF_B > COMB_B ? NBUF * BUF_B : COMB_B;
  static constexpr int PART_FLOATS = ROWS * D + ROWS * 4;
};

struct ManyShared {
  int64_t win[kWin];
  int first_bad, odd_from, role;
};

// One span.  (The lane is counted anew: what derives from it would else be kept in registers from span to span.)
template <class E, int D, int KS>
__device__ __forceinline__ void many_span(const PagedParams& p, const ManySpan& sp, int keys, unsigned char* smem, ManyShared& sh) {
  using C = ManyCfg<D, KS>;
  constexpr int NDB = C::NDB, NJB = C::NJB, BNS = C::BNS, TK = C::TK, KI = C::KI, PD = C::PD, NBUF = C::NBUF, NRB = C::NRB, DBW = C::DBW;
  int64_t* const win = sh.win;
  int &first_bad = sh.first_bad, &odd_from = sh.odd_from, &role = sh.role;
  const Unit& u = sp.u;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rb = wave % NRB, ksp = wave / NRB;
  const int lane = lane_again(), l32 = lane & 31, hh = lane >> 5, tid = wave * 64 + lane;
  const int row0 = u.tile * C::ROWS + rb * 32, tile_last = min((u.tile + 1) * C::ROWS, u.rows) - 1;
  const bool wave_live = row0 < u.rows, ok = row0 + l32 < u.rows;
  const int row = min(row0 + l32, u.rows - 1);
  const int head = u.hk * p.G + row % p.G, token = u.start + row / p.G;
  const int limit = limit_of(p, u, row);
  const int seen = min(limit_of(p, u, tile_last), p.cap);
  const int tile_all = limit_of(p, u, u.tile * C::ROWS), wave_all = limit_of(p, u, min(row0, u.rows - 1)), wave_any = limit_of(p, u, min(row0 + 31, u.rows - 1));
  const int parts = seen <= keys ? 1 : (seen - 1) / keys + 1;
  if (sp.part >= parts) return;
  const int k0 = (int)min((int64_t)sp.part * keys, (int64_t)seen), k1 = (int)min((int64_t)k0 + keys, (int64_t)seen);

  bf16x8_t qf[D / 16];
  {
    const uint16_t* qrow = p.q + token * p.qs[0] + head * p.qs[1];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(qrow + ks * 16 + hh * 8));
  }
  if (tid == 0) { first_bad = p.cap; odd_from = 0x7fffffff; }

  const TileReads<D> rd(lane);
  const uint32_t lds = (uint32_t)(uintptr_t)(lds_void_t*)smem;
  const unsigned char* const kbase = reinterpret_cast<const unsigned char*>(p.k + u.hk * p.cs[1]);
  const unsigned char* const vbase = reinterpret_cast<const unsigned char*>(p.v + u.hk * p.cs[1]);
  const int ld_row = wave * C::RPI + lane / C::CH, ld_pos = lane % C::CH;   // of load 0; later loads add 8 RPI rows

  RowState<D> st;
  st.clear();
  const int64_t wkeys = window_keys(p);
  for (int64_t w0 = k0; w0 < k1; w0 += wkeys) {
    const int w1 = (int)min(w0 + wkeys, (int64_t)k1);
    __syncthreads();   // the last window's page numbers have been read (first time: first_bad is set)
    fill_window(p, u.b, (int)w0, w1, win, &first_bad);
    __syncthreads();
    const int page0 = (int)page_of(p, (uint32_t)w0);
    const int tiles = (w1 - (int)w0 + TK - 1) / TK;
    auto issue = [&](int t) {
      const uint32_t kl = lds + (t % NBUF) * C::BUF_B + wave * 1024, vl = kl + C::TILE_B;
#pragma unroll
      for (int i = 0; i < KI; ++i) {
        const int r = ld_row + i * 8 * C::RPI;
        const int key = min((int)w0 + t * TK + r, w1 - 1);
        const int64_t off = row_at(p, win, page0, key);
        load_to_lds_16(kbase + off + (ld_pos ^ ((r / C::RP) & (C::CH - 1))) * 16, kl + i * 8192);
        load_to_lds_16(vbase + off + (ld_pos ^ (((r / C::RP) & (4 / C::RP - 1)) * 4)) * 16, vl + i * 8192);
      }
    };
    wait_all_loads();
#pragma unroll
    for (int t = 0; t < PD; ++t)
      if (t < tiles) issue(t);
    for (int t = 0; t < tiles; ++t) {
      const int later = min(PD - 1, tiles - 1 - t);
      if (later >= 2) wait_loads<2 * 2 * KI>();
      else if (later == 1) wait_loads<2 * KI>();
      else wait_loads<0>();
      const int t0 = (int)w0 + t * TK;
      if (t0 + TK > min(tile_all, w1)) {
#pragma unroll
        for (int i = 0; i < KI; ++i) make_finite<E>(smem + (t % NBUF) * C::BUF_B + C::TILE_B + wave * 1024 + i * 8192 + lane * 16, t0, &odd_from);
      }
      __syncthreads();   // every wave's part of the tile is in LDS; everyone has finished the one before
      if (t + PD < tiles) issue(t + PD);
      const int j0 = t0 + ksp * BNS;
      if (!wave_live || j0 >= min(wave_any, w1)) continue;
      const unsigned char* const Kt = smem + (t % NBUF) * C::BUF_B + ksp * BNS * C::ROWB;
      const bool masked = j0 + BNS > min(wave_all, w1);
      floatx16_t s[NJB];
      scores<E, D, NJB, D / 16 * NJB >= 16 ? 6 : 4>(Kt, rd, qf, s);
      if (masked) mask_scores<NJB>(s, j0, min(limit, w1), hh);
      uint4 pk[1][NJB][2];
      softmax<E, D, NJB, 1>(s, p.c, st, pk);
      values<E, D, NJB, 1>(Kt + C::TILE_B, rd, pk, st);
    }
  }
  __syncthreads();   // first_bad and odd_from are final, and the tiles have been read
  static_assert(KS > 1 || C::SMEM_B >= kManyWaves * 128 * D, "a wave's results fit into its part of the tiles");
  // (where splits are combined, that is the place this wave puts its results in afterwards)
  settle_odd_values<E, D>(p, u, k0, min(limit, k1), hh, st, reinterpret_cast<floatx4_t*>(smem) + wave * (KS > 1 ? C::SLOT_F4 * 64 : 8 * D));
  if (limit > first_bad) st.l = NAN;
  if (ksp == 0) add_odd_values<E, D>(p, u, odd_from, min(limit, k1), hh, st);   // (behind a masked tile all are)

  // ---- the key splits' results, added up in order: split j takes DBW column blocks from j DBW on
  float m_all = st.m, l_tot;
  floatx4_t acc[DBW * 4];
  const int db0 = KS == 1 ? 0 : ksp * DBW;
  if constexpr (KS == 1) {
    l_tot = sum_with_other_half(st.l);
#pragma unroll
    for (int i = 0; i < DBW * 4; ++i) acc[i] = floatx4_t{st.o[i / 4][4 * (i % 4)], st.o[i / 4][4 * (i % 4) + 1], st.o[i / 4][4 * (i % 4) + 2], st.o[i / 4][4 * (i % 4) + 3]};
  } else {
    floatx4_t* const slots = reinterpret_cast<floatx4_t*>(smem);
    floatx4_t* const mine = slots + wave * C::SLOT_F4 * 64 + lane;
#pragma unroll
    for (int i = 0; i < NDB * 4; ++i) mine[i * 64] = floatx4_t{st.o[i / 4][4 * (i % 4)], st.o[i / 4][4 * (i % 4) + 1], st.o[i / 4][4 * (i % 4) + 2], st.o[i / 4][4 * (i % 4) + 3]};
    mine[NDB * 4 * 64] = floatx4_t{st.m, st.l, 0.f, 0.f};
    __syncthreads();
    float ms[KS], ls[KS], w[KS];
    m_all = -INFINITY;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const floatx4_t x = slots[((k * NRB + rb) * C::SLOT_F4 + NDB * 4) * 64 + lane];
      ms[k] = x[0]; ls[k] = x[1];
      m_all = fmaxf(m_all, x[0]);
    }
    const float m_ref = m_all == -INFINITY ? 0.f : m_all;
    float l_all = 0.f;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      w[k] = fast_exp2(ms[k] - m_ref);
      l_all += ls[k] * w[k];
    }
    l_tot = sum_with_other_half(l_all);
#pragma unroll
    for (int i = 0; i < DBW * 4; ++i) {
      acc[i] = floatx4_t{0.f, 0.f, 0.f, 0.f};
      if (db0 + i / 4 < NDB) {
#pragma unroll
        for (int k = 0; k < KS; ++k) acc[i] += slots[((k * NRB + rb) * C::SLOT_F4 + db0 * 4 + i) * 64 + lane] * w[k];
      }
    }
  }
  const bool has = wave_live && db0 < NDB;   // does this wave have columns of rows?

  if (parts > 1) {
    // park [row block][16-byte piece][lane], then (m, l) by [row block][lane]; of every kManyFan neighbours the last to arrive adds
    // theirs up in the place of the first, and so on with these, until one has the result
    constexpr uint32_t ML_AT = C::ROWS * D * 4, PART_B = C::PART_FLOATS * 4;
    unsigned char* const first_slot = reinterpret_cast<unsigned char*>(p.parts) + (int64_t)sp.slot * PART_B;
    const uint32_t at = (uint32_t)((rb * NDB + db0) * 4 * 64 + lane) * 16, ml_at = ML_AT + (uint32_t)(rb * 64 + lane) * 8;
    auto park = [&](int part) {
      if (!has) return;
      const __amdgpu_buffer_rsrc_t buf = part_buffer(first_slot + (int64_t)part * PART_B);
#pragma unroll
      for (int i = 0; i < DBW * 4; ++i) store_part(buf, at + i * 1024, acc[i]);
      if (ksp == 0) store_ml(buf, ml_at, m_all, l_tot);
    };
    park(sp.part);
    int n = parts, idx = sp.part, stride = 1, level = 0;
    for (;; ++level) {
      const int g = idx / kManyFan, count = min(kManyFan, n - g * kManyFan), first = g * kManyFan * stride;
      const bool last = n <= kManyFan;
      if (count > 1) {   // (a single one is as it was)
        wait_vmcnt<0>();
        __syncthreads();   // every wave's stores are in memory
        if (tid == 0) role = arrive(p.counters + (sp.slot + first) * kManyLevels + level, count);
        __syncthreads();
        if (role == kLeaves) return;
        float2 s[kManyFan];
        if (has) {
          // (a part's pieces all at once, and the next one's while they are added)
          floatx4_t x[2][DBW * 4];
          auto ask = [&](int k) {
            const __amdgpu_buffer_rsrc_t buf = part_buffer(first_slot + (int64_t)(first + min(k, count - 1) * stride) * PART_B);
#pragma unroll
            for (int i = 0; i < DBW * 4; ++i) x[k % 2][i] = load_part(buf, at + i * 1024);
          };
#pragma unroll
          for (int k = 0; k < kManyFan; ++k) s[k] = load_ml(part_buffer(first_slot + (int64_t)(first + min(k, count - 1) * stride) * PART_B), ml_at);
          ask(0);
          m_all = -INFINITY;
#pragma unroll
          for (int k = 0; k < kManyFan; ++k)
            if (k < count) m_all = fmaxf(m_all, s[k].x);
          const float m_ref = m_all == -INFINITY ? 0.f : m_all;
          l_tot = 0.f;
#pragma unroll
          for (int i = 0; i < DBW * 4; ++i) acc[i] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < kManyFan; ++k) {
            if (k + 1 < kManyFan) ask(k + 1);
            if (k >= count) continue;
            const float w = fast_exp2(s[k].x - m_ref);
            l_tot += s[k].y * w;
#pragma unroll
            for (int i = 0; i < DBW * 4; ++i) acc[i] += x[k % 2][i] * w;
          }
          if (role == kCountsWrong) l_tot = NAN;
        }
        if (!last) {
          __syncthreads();   // (the other splits of the row block have read what is overwritten)
          park(first);
        }
      }
      if (last) break;
      idx = g;
      stride *= kManyFan;
      n = (n + kManyFan - 1) / kManyFan;
    }
  }
  if (!has || !ok) return;
  const float inv = inverse_of(l_tot);
#pragma unroll
  for (int i = 0; i < DBW * 4; ++i)
    if (db0 + i / 4 < NDB) store_out<E>(p, token, head, (db0 + i / 4) * 32 + 8 * (i % 4) + 4 * hh, make_float4(acc[i][0] * inv, acc[i][1] * inv, acc[i][2] * inv, acc[i][3] * inv));
  if (ksp == 0 && hh == 0) p.lse[(int64_t)token * p.hq + head] = lse_of(m_all, l_tot);
}

// SMALLER: row tiles of 128 and 64 too; with every unit of the chip holding one workgroup, which goes on from span to span.
// Else, at head_dim 64, two workgroups a unit fit, in 128 registers and with 72 bytes of scratch memory, of which the loop over
// tiles reads one value: 8000 tokens over 30000 keys, 32 heads on 8, 2125 -> 1996 us.  (The other side: 2500 tokens' own prompt, 32 heads of own keys, 320
// tiles for 256 units, 60 -> 80 us, as the units that hold two end last; over 8000 keys, where tiles are cut, 249 -> 227.)
template <class E, int D, bool SMALLER>
__global__ __launch_bounds__(kManyWaves * 64, D == 64 && !SMALLER ? 4 : 2) void paged_many_kernel(const PagedParams p, const ManyArgs a) {
  constexpr int BYTES = SMALLER ? std::max({ManyCfg<D, 1>::SMEM_B, ManyCfg<D, 2>::SMEM_B, ManyCfg<D, 4>::SMEM_B}) : ManyCfg<D, 1>::SMEM_B;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[BYTES];
  __shared__ ManyShared sh;
  const Lanes lanes(p);
  const WaveSums sums{p, lanes};
  const Division d = choose_division<SMALLER, D>(sums, p.hkv, a);
  const int all = sums.all(d);   // spans
  // neighbours share an XCD and its L2 where they read the same keys
  const int per = (all + 7) / 8, xcd = blockIdx.x & 7;
  bool again = false;
  for (int idx = blockIdx.x >> 3; idx < per; idx += gridDim.x >> 3) {
    ManySpan sp;
    const int item = xcd * per + idx;
    if (item >= all || !find_span(p, d, lanes, item, sp)) break;
    if (again) __syncthreads();   // the span before is done with LDS
    again = true;
    if (!SMALLER || d.rows == 256) many_span<E, D, 1>(p, sp, d.keys, smem, sh);
    else if constexpr (SMALLER) {
      if (d.rows == 128) many_span<E, D, 2>(p, sp, d.keys, smem, sh);
      else many_span<E, D, 4>(p, sp, d.keys, smem, sh);
    }
  }
}

template <class E, int D>
void launch(const PagedParams& p, bool smaller, const ManyArgs& a, unsigned grid, hipStream_t st) {
  const dim3 g(grid), b(kManyWaves * 64);
  if (smaller) paged_many_kernel<E, D, true><<<g, b, 0, st>>>(p, a);
  else paged_many_kernel<E, D, false><<<g, b, 0, st>>>(p, a);
}

}  // namespace

PagedPlan plan_paged_many(const loong_paged_desc& d, int cus) { return plan_many(d, cus); }

void launch_paged_many(const PagedParams& p, const loong_paged_desc& d, int cus, unsigned grid, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool smaller = !rows_fill(d, cus);
  const ManyArgs a = many_args(d, cus);
  if (d.dtype == LOONG_BF16) {
    if (d.head_dim == 128) launch<Bf16, 128>(p, smaller, a, grid, st);
    else launch<Bf16, 64>(p, smaller, a, grid, st);
  } else {
    if (d.head_dim == 128) launch<Fp16, 128>(p, smaller, a, grid, st);
    else launch<Fp16, 64>(p, smaller, a, grid, st);
  }
}

}  // namespace loong
