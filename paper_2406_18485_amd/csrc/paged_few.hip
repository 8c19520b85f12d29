// Paged attention of few rows: up to 32 query rows of a kv head (one new token, or a few drafted ones).
//
// Bound by HBM, 2 e head_dim bytes a key: the 24 matrix instructions of 32 keys, for 32 rows however few there are, keep a SIMD for 768
// clocks, and a unit's share of the memory's rate needs 1000 for their 16 KB.  Every wave has tiles of keys and LDS of its own and waits for nobody;
// while one of its K and V tiles is used the other is on its way: 8 waves a unit keep 64 to 128 KB in flight.
//
// Division.  All keys of all units (a sequence's rows of one kv head) are put in one line and cut into equal shares, one for every
// workgroup of a launch that the chip holds at once: however unequal the lengths, all end together.  A workgroup works on
// the units of its share one after the other.  Lengths are in device memory: every wave works out the line from them (a lane a
// sequence, or a run of them).  Units of up to kShort grains are not cut: they are whole in the share that they begin in, and where there
// are workgroups enough every unit begins with a share of its own.  (48 sequences of 1000 to 8192 keys, 8 kv heads: 148.5 us with spans of
// one length that the hardware deals out, 138.8 with shares; one sequence of 4000 keys, 8 heads, shares that straddle units 16.2, apart 12.3.)
//
// A cut unit's shares are added up by the last to arrive (split_exchange.h), kFewFan at a time, so that the results of a context spread
// over the whole chip are not read by one workgroup.  (Two contexts of 262144 keys, one kv head: 127 us with 512 parts added up by
// one workgroup, 77 sixteen at a time.  A further level costs 5 us: 16000 keys of 8 heads, 62 parts, 22.5 us in two, 20.3 in one.)
//
// 48 sequences, 708 MB of keys and values: 138 us, 5.1 TB/s (64 of 4000 keys 5.6).  The shortest call, one sequence of up to 32 keys, takes 7.8 us, a launch
// alone 2.3: the rest is the chain of loads lengths -> page numbers -> keys, a microsecond each, and the sums over waves; an
// exchange adds 3.5.
#include <hip/hip_runtime.h>

#include "paged_body.h"

namespace loong {
namespace {

constexpr int kFewWaves = 4, kFewPerCu = 2;
constexpr int kPieces = 2;             // of a probability, see softmax()
constexpr int kFewFan = 64;            // parts that are added up at a time
constexpr int kFewLevels = 4;          // 64^4 parts are more than there are shares
constexpr int kGrain = 64;             // keys that are not divided
constexpr int kShort = 8;              // grains of a unit that is not divided, see above
constexpr int kLeast = 4;              // grains of a share, at the least, of units that are

// ---- the line of all units, in grains of kGrain << shift keys -------------------------------------------------------
// What a lane found out stays in LDS, where every wave writes the same and reads what it wrote.
struct LineLanes {
  int here[64], upto[64];   // grains of a lane's sequences, and of all up to them
  int start[64], n[64], rows[64], kv[64], grains[64], room[64];   // its sequence, if it has one; of a unit: its grains, and what it takes of the line
};
struct Line {
  int per;             // sequences a lane looks at
  int total, share;    // grains altogether, and of a share
  int shift;           // (0 unless a grain of 64 keys makes more than 2^29 of them)
  bool apart;          // every unit begins with a share of its own
  LineLanes& lanes;

  static __device__ __forceinline__ int grains(const Seq& s, int shift) { return s.paged <= kGrain ? 1 : ((s.paged - 1) >> shift) / kGrain + 1; }

  __device__ __forceinline__ Line(const PagedParams& p, LineLanes& l) : lanes(l) {
    const int lane = threadIdx.x & 63;
    per = (p.n_seqs + 63) / 64;
    shift = 0;
    Seq mine{};
    int here, most;
    float all;
    for (;; ++shift) {
      here = 0;
      most = 0;
      all = 0.f;
      for (int i = 0; i < per; ++i) {
        if (lane * per + i >= p.n_seqs) break;
        const Seq s = sequence(p, lane * per + i);
        if (i == 0) mine = s;
        if (s.rows == 0) continue;
        const int g = grains(s, shift);
        here += g * p.hkv;
        most = max(most, g);
        all += (float)g * (float)p.hkv;
      }
      all = wave_total(all);
      if (all < 5e8f || shift == 24) break;
    }
    int upto = wave_prefix(here);
    total = all < 2e9f ? last_lane(upto) : 0;   // (so many units have no rows: seq_start decreases somewhere)
    most = wave_most(most);
    const int even = (total + (int)gridDim.x - 1) / (int)gridDim.x, least = most <= kShort ? most : kLeast;
    share = max(max(even, least), 1);
    // where there are workgroups enough, no share has the end of one unit and the beginning of the next
    apart = true;
    int spread = 0;
    float room = 0.f;
    for (int i = 0; i < per; ++i) {
      if (lane * per + i >= p.n_seqs) break;
      const Seq s = per == 1 ? mine : sequence(p, lane * per + i);
      if (s.rows == 0) continue;
      const int n = room_of(grains(s, shift));
      spread += n * p.hkv;
      room += (float)n * (float)p.hkv;
    }
    apart = wave_total(room) <= (float)gridDim.x * (float)share;
    if (apart) {
      here = spread;
      upto = wave_prefix(here);
      total = last_lane(upto);
    }
    lanes.here[lane] = here; lanes.upto[lane] = upto;
    lanes.start[lane] = mine.start; lanes.n[lane] = mine.n; lanes.rows[lane] = mine.rows; lanes.kv[lane] = mine.kv;
    lanes.grains[lane] = grains(mine, shift); lanes.room[lane] = room_of(grains(mine, shift));
  }

  __device__ __forceinline__ int room_of(int n) const { return !apart ? n : n <= kShort ? share : (int)((uint32_t)(n + share - 1) / (uint32_t)share) * share; }

  // the unit at `pos` (below total), its first grain, its grains and what it takes of the line
  __device__ __forceinline__ Unit at(const PagedParams& p, int pos, int& start, int& n, int& room) const {
    const int lane = threadIdx.x & 63;
    const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(lanes.upto[lane] > pos));
    int before = __builtin_amdgcn_readfirstlane(lanes.upto[l] - lanes.here[l]);
    Unit u;
    if (per == 1) {
      u.b = l;
      u.start = __builtin_amdgcn_readfirstlane(lanes.start[l]); u.n = __builtin_amdgcn_readfirstlane(lanes.n[l]);
      u.rows = __builtin_amdgcn_readfirstlane(lanes.rows[l]); u.kv = __builtin_amdgcn_readfirstlane(lanes.kv[l]);
      n = __builtin_amdgcn_readfirstlane(lanes.grains[l]); room = __builtin_amdgcn_readfirstlane(lanes.room[l]);
    } else {
      for (int i = 0;; i += 64) {   // (ends: the run has the grain)
        const int b = l * per + i + lane;
        Seq s{};
        if (i + lane < per && b < p.n_seqs) s = sequence(p, b);
        const int g = s.rows ? room_of(grains(s, shift)) * p.hkv : 0, sum = wave_prefix(g);
        const uint64_t past = __builtin_amdgcn_ballot_w64(before + sum > pos);
        if (past || i + 64 >= per) {
          const int from = past ? __builtin_ctzll(past) : 63;
          before += __builtin_amdgcn_readlane(sum, from) - __builtin_amdgcn_readlane(g, from);
          u.b = __builtin_amdgcn_readlane(b, from);
          u.start = __builtin_amdgcn_readlane(s.start, from); u.n = __builtin_amdgcn_readlane(s.n, from);
          u.rows = __builtin_amdgcn_readlane(s.rows, from); u.kv = __builtin_amdgcn_readlane(s.kv, from);
          n = __builtin_amdgcn_readlane(grains(s, shift), from); room = room_of(n);
          break;
        }
        before += last_lane(sum);
      }
    }
    u.hk = (int)((uint32_t)(pos - before) / (uint32_t)room);
    u.tile = 0;
    start = before + u.hk * room;
    return u;
  }
};

// a workgroup's part of a unit: which of how many, and where they are parked
struct Part {
  int part, parts, slot0, slot1;   // slots of the first part and the second
  __device__ __forceinline__ int slot_of(int k) const { return k == 0 ? slot0 : slot1 + 2 * (k - 1); }
};

template <int D>
struct FewCfg {
  static constexpr int BNS = 4096 / D;            // keys per tile: 8 KB
  static constexpr int NJB = BNS / 32, ROWB = D * 2, CH = D / 8, RP = 256 / ROWB, RPI = 1024 / ROWB, LI = 8;
  static constexpr int TILE_B = 8192, WAVE_B = 2 * TILE_B;
  static constexpr int COLS = D / 4;              // float4 columns of a row
};

template <class E, int D>
struct FewShared {
  __attribute__((aligned(1024))) unsigned char smem[kFewWaves * FewCfg<D>::WAVE_B];
  int64_t win[kWin];
  float2 ml[kFewWaves][64];
  int first_bad, odd_from, role;
  LineLanes lanes;
};

// Keys [k0, k1) of a unit
template <class E, int D>
__device__ __forceinline__ void few_keys(const PagedParams& p, const Unit& u, int k0, int k1, FewShared<E, D>& sh, RowState<D>& st) {
  using C = FewCfg<D>;
  constexpr int NJB = C::NJB, BNS = C::BNS;
  auto& smem = sh.smem;
  auto& win = sh.win;
  int &first_bad = sh.first_bad, &odd_from = sh.odd_from;
  // (the lane is counted anew: what derives from it would else be kept in registers from unit to unit)
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_again(), l32 = lane & 31, hh = lane >> 5, tid = wave * 64 + lane;
  const int row = min(l32, u.rows - 1);
  const int limit = limit_of(p, u, row), seen_by_all = limit_of(p, u, 0);

  bf16x8_t qf[D / 16];
  {
    const uint16_t* qrow = p.q + (u.start + row / p.G) * p.qs[0] + (u.hk * p.G + row % p.G) * p.qs[1];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(qrow + ks * 16 + hh * 8));
  }
  if (tid == 0) { first_bad = p.cap; odd_from = 0x7fffffff; }

  const PackedReads<D> rd(lane);
  unsigned char* const Kt = smem + wave * C::WAVE_B;
  unsigned char* const Vt = Kt + C::TILE_B;
  const uint32_t k_lds = (uint32_t)(uintptr_t)(lds_void_t*)smem + wave * C::WAVE_B, v_lds = k_lds + C::TILE_B;
  const unsigned char* const kbase = reinterpret_cast<const unsigned char*>(p.k + u.hk * p.cs[1]);
  const unsigned char* const vbase = reinterpret_cast<const unsigned char*>(p.v + u.hk * p.cs[1]);
  const int ld_row = lane / C::CH, ld_pos = lane % C::CH;

  const int64_t wkeys = window_keys(p);
  for (int64_t w0 = k0; w0 < k1; w0 += wkeys) {
    const int w1 = (int)min(w0 + wkeys, (int64_t)k1);
    __syncthreads();   // the last window's page numbers have been read (first time: first_bad is set)
    fill_window(p, u.b, (int)w0, w1, win, &first_bad);
    __syncthreads();
    const int page0 = (int)page_of(p, (uint32_t)w0);
    const int tiles = (w1 - (int)w0 + BNS - 1) / BNS;
    int64_t off[C::LI];   // this lane's rows of a tile, bytes from the head's first
    auto place = [&](int t) {
#pragma unroll
      for (int i = 0; i < C::LI; ++i) {
        const int key = min((int)w0 + t * BNS + i * C::RPI + ld_row, w1 - 1);
        off[i] = row_at(p, win, page0, key);
      }
    };
    auto issue_k = [&] {
#pragma unroll
      for (int i = 0; i < C::LI; ++i) {
        const int r = i * C::RPI + ld_row;
        load_to_lds_16(kbase + off[i] + (ld_pos ^ tile_swizzle<D>(r)) * 16, k_lds + i * 1024);
      }
    };
    auto issue_v = [&] {
#pragma unroll
      for (int i = 0; i < C::LI; ++i) {
        const int r = i * C::RPI + ld_row;
        load_to_lds_16(vbase + off[i] + (ld_pos ^ tile_swizzle<D>(r)) * 16, v_lds + i * 1024);
      }
    };
    int t = wave;
    wait_all_loads();
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
      uint4 pk[kPieces][NJB][2];
      softmax<E, D, NJB, kPieces>(s, p.c, st, pk);
      if (more) wait_loads<C::LI>();
      else wait_loads<0>();
      if (masked) {
#pragma unroll 1
        for (int i = 0; i < C::LI; ++i) make_finite<E>(Vt + i * 1024 + lane * 16, j0, &odd_from);
      }
      values<E, D, NJB, kPieces>(Vt, rd, pk, st);
      if (more) {
        wait_reads();   // (of V)
        issue_v();
      }
    }
  }
  settle_odd_values<E, D>(p, u, k0, min(limit, k1), hh, st, reinterpret_cast<floatx4_t*>(Kt));   // (the wave's tiles are used up)
}

// The waves' results, and those of the unit's other parts.
template <class E, int D>
__device__ __forceinline__ void few_result(const PagedParams& p, const Unit& u, const Part& share, int k1, FewShared<E, D>& sh, RowState<D>& st) {
  using C = FewCfg<D>;
  constexpr int NT = kFewWaves * 64, NDB = D / 32;
  auto& smem = sh.smem;
  auto& ml = sh.ml;
  int &first_bad = sh.first_bad, &odd_from = sh.odd_from, &role = sh.role;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_again(), l32 = lane & 31, hh = lane >> 5, tid = wave * 64 + lane;
  const int row = min(l32, u.rows - 1);
  const int head = u.hk * p.G + row % p.G, token = u.start + row / p.G;
  const int limit = limit_of(p, u, row);

  // ---- the waves' results, in wave order: wave w adds up columns 32 w .. + 31
  __syncthreads();   // (also: first_bad and odd_from are final)
  if (limit > first_bad) st.l = NAN;
  if (wave == 0) add_odd_values<E, D>(p, u, odd_from, min(limit, k1), hh, st);   // (behind a masked tile all are)
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
  const bool ok = l32 < u.rows;
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
  if (share.parts == 1) {
    const float inv = inverse_of(l_tot);
    if (wave < NDB && ok) {
#pragma unroll
      for (int vq = 0; vq < 4; ++vq)
        store_out<E>(p, token, head, wave * 32 + 8 * vq + 4 * hh, make_float4(acc[vq].x * inv, acc[vq].y * inv, acc[vq].z * inv, acc[vq].w * inv));
      if (wave == 0 && hh == 0) p.lse[(int64_t)token * p.hq + head] = lse_of(m_all, l_tot);
    }
    return;
  }

  // ---- one of several spans: park [row][D], then (m, l) of the rows; of every kFewFan neighbours the last to arrive adds theirs up
  // in the place of the first, and so on with these, until one has the result
  constexpr uint32_t ML_AT = kFewRows * D * 4;
  const __amdgpu_buffer_rsrc_t all = part_buffer(p.parts);
  const uint32_t slot_b4 = (uint32_t)p.slot_floats * 4;   // (all slots together are below 2^31 bytes)
  if (wave < NDB && ok) {
    const uint32_t mine = (uint32_t)share.slot_of(share.part) * slot_b4;
#pragma unroll
    for (int vq = 0; vq < 4; ++vq) {
      const floatx4_t x = {acc[vq].x, acc[vq].y, acc[vq].z, acc[vq].w};
      store_part(all, mine + (uint32_t)(l32 * D + wave * 32 + 8 * vq + 4 * hh) * 4, x);
    }
    if (wave == 0 && hh == 0) store_ml(all, mine + ML_AT + l32 * 8, m_all, l_tot);
  }
  // threads: COLS float4 columns x rows (a power of two), and what is left of the workgroup shares the parts
  int rows2 = 1;
  while (rows2 < u.rows) rows2 <<= 1;
  const int items = min(rows2 * C::COLS, NT), groups = NT / items, grp = tid / items;
  Joined* const red = reinterpret_cast<Joined*>(smem);
  int n = share.parts, idx = share.part, stride = 1, level = 0;
  for (;; ++level) {
    const int g = idx / kFewFan, count = min(kFewFan, n - g * kFewFan), first = g * kFewFan * stride;
    const bool last = n <= kFewFan;
    if (count > 1) {   // (a single one is as it was)
      wait_vmcnt<0>();
      __syncthreads();   // every wave's stores are in memory, and LDS has been read
      if (tid == 0) role = arrive(p.counters + share.slot_of(first) * kFewLevels + level, count);
      __syncthreads();
      if (role == kLeaves) return;
      for (int base = 0; base < rows2 * C::COLS; base += items) {
        const int at = base + tid % items, r = at / C::COLS, col = at % C::COLS, rr = min(r, u.rows - 1);
        Joined j{-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
        constexpr int AHEAD = 8;
        for (int k = grp; k < count; k += groups * AHEAD) {
          floatx4_t x[AHEAD];
          float2 s[AHEAD];
#pragma unroll
          for (int a = 0; a < AHEAD; ++a) {
            const uint32_t from = (uint32_t)share.slot_of(first + min(k + a * groups, count - 1) * stride) * slot_b4;
            x[a] = load_part(all, from + (rr * D + col * 4) * 4);
            s[a] = load_ml(all, from + ML_AT + rr * 8);
          }
#pragma unroll
          for (int a = 0; a < AHEAD; ++a)
            if (k + a * groups < count) j.add(s[a].x, s[a].y, x[a]);
        }
        __syncthreads();   // (all have read what is overwritten below, and LDS)
        if (groups > 1) {
          red[tid] = j;
          __syncthreads();
          for (int h = 1; h < groups && grp == 0; ++h) j.add(red[tid + h * items].m, red[tid + h * items].l, red[tid + h * items].x);
        }
        if (grp == 0 && r < u.rows) {
          if (role == kCountsWrong) j.l = NAN;
          if (last) {
            const float inv = inverse_of(j.l);
            const int tk = u.start + r / p.G, hd = u.hk * p.G + r % p.G;
            store_out<E>(p, tk, hd, col * 4, make_float4(j.x[0] * inv, j.x[1] * inv, j.x[2] * inv, j.x[3] * inv));
            if (col == 0) p.lse[(int64_t)tk * p.hq + hd] = lse_of(j.m, j.l);
          } else {
            store_part(all, (uint32_t)share.slot_of(first) * slot_b4 + (r * D + col * 4) * 4, j.x);
            if (col == 0) store_ml(all, (uint32_t)share.slot_of(first) * slot_b4 + ML_AT + r * 8, j.m, j.l);
          }
        }
      }
    }
    if (last) return;
    idx = g;
    stride *= kFewFan;
    n = (n + kFewFan - 1) / kFewFan;
  }
}

template <class E, int D>
__global__ __launch_bounds__(kFewWaves * 64, kFewPerCu) void paged_few_kernel(const PagedParams p) {
  __shared__ FewShared<E, D> sh;
  const Line line(p, sh.lanes);
  const int s = blockIdx.x;
  int pos = __builtin_amdgcn_readfirstlane(s * line.share);   // (below 2^31: total is, and a share is at most kShort grains too long)
  const int end = min(pos + line.share, line.total);
  bool again = false;
  while (pos < end) {
    int start, n, room;
    const Unit u = line.at(p, pos, start, n, room);
    const int seen = min(limit_of(p, u, u.rows - 1), p.cap), grain = kGrain << line.shift;
    const int seen_n = max((int)(((int64_t)seen + grain - 1) / grain), 1);   // grains that any row sees
    Part part{0, 1, 0, 0};
    int to = start + room;
    if (n <= kShort) {
      if (pos > start) { pos = to; continue; }   // (the share that it begins in has it)
    } else {
      to = min(to, end);
      const int first = start / line.share, last = (start + seen_n - 1) / line.share;
      part.part = s - first;
      part.parts = last - first + 1;
      part.slot0 = 2 * first + (start != first * line.share);
      part.slot1 = 2 * first + 2;
    }
    if (part.part < part.parts) {
      const int k0 = (int)min((int64_t)(pos - start) * grain, (int64_t)seen), k1 = n <= kShort ? seen : (int)min((int64_t)(to - start) * grain, (int64_t)seen);
      if (again) __syncthreads();   // the unit before is done with LDS
      again = true;
      RowState<D> st;
      st.clear();
      few_keys<E, D>(p, u, k0, k1, sh, st);
      few_result<E, D>(p, u, part, k1, sh, st);
    }
    pos = to;
  }
}

}  // namespace

// As many workgroups as the chip holds at once, fewer where there cannot be as many parts.
PagedPlan plan_paged_few(const loong_paged_desc& d, int cus) {
  PagedPlan pl{};
  const int64_t units = (int64_t)(d.n_seqs < d.n_tokens ? d.n_seqs : d.n_tokens) * d.n_kv_heads;
  const int64_t grains = (cached_keys(d) + kGrain - 1) / kGrain, parts = grains <= kShort ? 1 : (grains + kLeast - 1) / kLeast;
  pl.workgroups = (int64_t)kFewPerCu * cus;
  if (units * parts < pl.workgroups) pl.workgroups = units * parts;
  pl.slots = parts == 1 ? 0 : 2 * pl.workgroups;
  pl.slot_floats = kFewRows * (d.head_dim + 2);
  return pl;
}

void launch_paged_few(const PagedParams& p, const loong_paged_desc& d, unsigned grid, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  const dim3 g(grid), b(kFewWaves * 64);
  if (d.dtype == LOONG_BF16) {
    if (d.head_dim == 128) paged_few_kernel<Bf16, 128><<<g, b, 0, st>>>(p);
    else paged_few_kernel<Bf16, 64><<<g, b, 0, st>>>(p);
  } else {
    if (d.head_dim == 128) paged_few_kernel<Fp16, 128><<<g, b, 0, st>>>(p);
    else paged_few_kernel<Fp16, 64><<<g, b, 0, st>>>(p);
  }
}

}  // namespace loong
