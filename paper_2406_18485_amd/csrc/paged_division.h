// How the work of paged attention over many rows is divided: sizes of row tiles and of spans of keys, from the lengths of all sequences.
//
// Every wave of a launch works this out for itself from device memory; the sums over the sequences are its part (`Sums` below), all else
// is here and runs on the host too, where it can be looked at over the whole range of lengths.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "loong_internal.h"
#include "paged_params.h"

namespace loong {

constexpr int kManyFan = 4;            // parts that are added up at a time
constexpr int kManyLeast = 256;        // keys of a span of a cut unit, at the least
constexpr int kManyMore = 2;           // spans that cutting may add, per unit of the chip
// What a span takes, in ns: per key at head_dim 128 (KS = 1, 2, 4; 0.7 of it at 64) and whatever it has; if its unit is cut, every level of
// adding parts up takes its waits, and every part that is added what one workgroup needs to read it (50 bytes a ns).
constexpr float kKeyNs[3] = {31.5f, 18.5f, 12.f}, kFixedNs = 9500.f, kCutNs = 1500.f, kLevelNs = 1500.f, kPartNs = 0.08f;

struct ManyArgs {
  int cus;
  int hold;     // workgroups that the chip holds at once: cus, or two for each
  int units;    // that there can be, at the most
};

// How all the work is divided: rows of a tile, keys of a span (at least kManyLeast).
struct Division {
  int rows, keys;
  bool none;    // there are no units, or more than there can be
};

__host__ __device__ inline int row_tiles(int rows_of_seq, int rows) { return (rows_of_seq + rows - 1) >> (rows == 64 ? 6 : rows == 128 ? 7 : 8); }
__host__ __device__ inline int key_parts(int paged, int keys) { return paged <= keys ? 1 : (int)((uint32_t)(paged - 1) / (uint32_t)keys) + 1; }
// Sums::longest(): keys of the longest sequence that has rows; tiles(rows, load, units): of one kv head, the row tiles and the keys they go
// over; spans(rows, inv): spans of 1 / inv keys, of one kv head; rcp(x): 1 / x, a step or so off.
// (Estimates in floats: an integer division is some 40 instructions, and all this is in front of the first load of a key.)
template <bool SMALLER, int D, class Sums>
__host__ __device__ inline Division choose_division(const Sums& sums, int hkv, const ManyArgs& a) {
  float best = INFINITY;
  const float hold = (float)a.hold, per_place = sums.rcp(hold), slower = hold * sums.rcp((float)a.cus);
  const int most = sums.longest();
  // (a span of the longest sequence, which cuts nothing and always fits.  In whole numbers: above 2^24 keys a float may lie below them)
  auto whole_tiles = [](int keys) { const int k = (keys + 63) / 64 * 64; return k > kManyLeast ? k : kManyLeast; };
  const int whole = whole_tiles(most);
  Division d{256, whole, false};
#pragma unroll
  for (int small = 0; small < (SMALLER ? 3 : 1); ++small) {
    const int rows = 256 >> small;
    float load, units;
    sums.tiles(rows, load, units);
    load *= hkv;
    units *= hkv;
    if (units == 0.f || units > (float)a.units) return Division{256, kManyLeast, true};   // (more than there can be: seq_start decreases somewhere)
    // not cut; cut so that there is a span of the longest for all that the chip holds; cut into equal work
    const float even = load * per_place, fit = floorf(hold * sums.rcp(units) + 1e-3f);
#pragma unroll 1
    for (int c = 0; c < 3; ++c) {
      if (c == 1 && fit < 2.f) continue;
      const float want = c == 1 ? (float)most * sums.rcp(fit) + 1.f : even;
      const int k = c == 0 ? whole : want < 2e9f ? whole_tiles((int)want) : most;
      if (c > 0 && k >= most) continue;
      // (what bounds the number of spans, and their slots: cutting adds at most kManyMore a unit of the chip)
      if (k < most && load > (float)k * (kManyMore * 0.999f) * (float)a.cus) continue;
      float n = units;
      if (k < most) n = sums.spans(rows, sums.rcp((float)k)) * hkv;
      // all alike, in rounds; unequal, in equal work and the longest at the least
      constexpr float head = D == 128 ? 1.f : 0.7f;
      float join = 0.f;
      if (k < most) {
        const float parts = ceilf((float)most * sums.rcp((float)k) - 1e-3f), second = parts > kManyFan ? ceilf(parts / kManyFan) : 0.f;
        join = kCutNs + (second > 0.f ? 2.f : 1.f) * kLevelNs + (fminf(parts, kManyFan) + second) * (rows * D * kPartNs);
      }
      const float key = kKeyNs[small] * head * slower, fixed = kFixedNs + join, span = (float)(k < most ? k : most) * key + fixed;
      const float est = 0.5f * (ceilf(n * per_place - 1e-3f) * span + fmaxf((load * key + n * fixed) * per_place, span));
      if (est < best) { best = est; d.rows = rows; d.keys = k; }
    }
  }
  return d;
}

// Are row tiles of 256 alone better?  They are where every unit of the chip has one.  At head_dim 64, where two workgroups share a unit that takes
// tiles of 256 only, they are with fewer rows too if the contexts are long, as far as the page table says: it has room for 2^18 scores
// a unit.  (32 heads on 8, 1500 tokens: over 1500 / 8000 / 30000 keys 39 / 164 / 580 us with all three tiles, 31 / 137 / 487 so; 700 tokens, over
// 1500 / 2500 / 4000 / 30000 keys 28.7 / 40.8 / 54.3 / 301 and 32.6 / 40.4 / 50.0 / 224; three prompts of 500 20.5 and 27.  A table with much more
// room than keys costs those few us; below 64 rows a unit it would cost half as much again, 400 tokens over 1500 keys 22.5 and 35.)
inline bool rows_fill(const loong_paged_desc& d, int cus) {
  const int64_t rows = (int64_t)d.n_tokens * d.n_q_heads;
  if (rows >= (int64_t)256 * cus) return true;
  return d.head_dim == 64 && rows >= (int64_t)64 * cus && cached_keys(d) >= ((int64_t)cus << 18) / rows;
}
inline int64_t most_units(const loong_paged_desc& d, int rows) {
  const int64_t group = d.n_q_heads / d.n_kv_heads;
  return ((d.n_seqs < d.n_tokens ? d.n_seqs : d.n_tokens) + d.n_tokens * group / rows) * d.n_kv_heads;
}
inline ManyArgs many_args(const loong_paged_desc& d, int cus) {
  const bool smaller = !rows_fill(d, cus);
  return ManyArgs{cus, d.head_dim == 64 && !smaller ? 2 * cus : cus, (int)most_units(d, smaller ? 64 : 256)};
}

// Where row tiles of 256 fill the chip the hardware deals the spans out, else as many workgroups as it holds take them in turn.
// Spans of cut units are longer than load / (kManyMore cus) (0.999 of it: the sum is a float), so that there are at most kManyMore cus of
// them and a remainder a unit, and at most as many units are cut.
inline PagedPlan plan_many(const loong_paged_desc& d, int cus) {
  PagedPlan pl{};
  const bool smaller = !rows_fill(d, cus);
  const int64_t units = most_units(d, smaller ? 64 : 256);
  const int64_t keys = cached_keys(d), parts = keys <= kManyLeast ? 1 : (keys + kManyLeast - 1) / kManyLeast;
  const int64_t more = (int64_t)(kManyMore * cus * 1.01) + 8;
  int64_t spans = units + more;
  if (units * parts < spans) spans = units * parts;
  pl.workgroups = smaller && spans > cus ? cus : spans;
  pl.workgroups = (pl.workgroups + 7) / 8 * 8;
  pl.slots = parts == 1 ? 0 : 2 * more < spans ? 2 * more : spans;
  pl.slot_floats = 256 * (d.head_dim + 4);
  return pl;
}

}  // namespace loong
