"""How attention of many rows divides its work, over all lengths that the interface takes, on the CPU: the kernels' own choice, with
the sums over the sequences added up in a wave's order."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

import paper_2406_18485_amd as P
from paper_2406_18485_amd import build

SOURCE = r"""
#include <cstring>
#include <vector>
#include "paged_division.h"
using namespace loong;

struct Seq { int rows, paged; };
struct HostSums {
  const std::vector<Seq>& seqs;
  int ulps;   // what a hardware reciprocal may be off
  float rcp(float x) const {
    float y = 1.f / x;
    for (int i = 0; i < (ulps < 0 ? -ulps : ulps); ++i) y = std::nextafterf(y, ulps < 0 ? 0.f : INFINITY);
    return y;
  }
  // one lane a sequence, 64 at a time; lanes in pairs inside rows of 16, then the rows in pairs
  template <class F>
  float total(F f) const {
    float x[64] = {};
    for (size_t b = 0; b < seqs.size(); ++b) x[b % 64] += f(seqs[b]);
    for (int n = 64; n > 1; n /= 2)
      for (int i = 0; i < n / 2; ++i) x[i] = x[2 * i + 1] + x[2 * i];
    return x[0];
  }
  int longest() const {
    int most = 0;
    for (auto& s : seqs) if (s.rows && s.paged > most) most = s.paged;
    return most;
  }
  void tiles(int rows, float& load, float& units) const {
    load = total([&](const Seq& s) { return (float)row_tiles(s.rows, rows) * (float)s.paged; });
    units = total([&](const Seq& s) { return (float)row_tiles(s.rows, rows); });
  }
  float spans(int rows, float inv) const {
    return total([&](const Seq& s) { return (float)row_tiles(s.rows, rows) * fmaxf(ceilf((float)s.paged * inv - 1e-4f), 1.f); });
  }
};

// out: rows, keys, none, spans, spans of cut units, most of one unit, slots, workgroups
extern "C" void divide(const loong_paged_desc* d, int cus, int ulps, const int32_t* n_new, const int32_t* kv, int64_t* out) {
  std::vector<Seq> seqs;
  const int64_t cap = cached_keys(*d);
  for (int b = 0; b < d->n_seqs; ++b)
    seqs.push_back({(n_new[b] < d->max_new ? n_new[b] : d->max_new) * (d->n_q_heads / d->n_kv_heads), (int)(kv[b] < cap ? kv[b] : cap)});
  const HostSums sums{seqs, ulps};
  const ManyArgs a = many_args(*d, cus);
  const bool smaller = !rows_fill(*d, cus);
  const Division r = d->head_dim == 128 ? (smaller ? choose_division<true, 128>(sums, d->n_kv_heads, a) : choose_division<false, 128>(sums, d->n_kv_heads, a))
                                        : (smaller ? choose_division<true, 64>(sums, d->n_kv_heads, a) : choose_division<false, 64>(sums, d->n_kv_heads, a));
  int64_t all = 0, cut = 0, most = 0;
  for (auto& s : seqs) {
    if (r.none || r.keys <= 0 || s.rows == 0) continue;
    const int64_t parts = key_parts(s.paged, r.keys), n = parts * row_tiles(s.rows, r.rows) * d->n_kv_heads;
    all += n;
    if (parts > 1) cut += n;
    if (parts > most) most = parts;
  }
  const PagedPlan pl = plan_many(*d, cus);
  const int64_t got[8] = {r.rows, r.keys, r.none, all, cut, most, pl.slots, pl.workgroups};
  memcpy(out, got, sizeof got);
}
"""


@pytest.fixture(scope="module")
def divide(tmp_path_factory):
    at = tmp_path_factory.mktemp("division")
    src, lib = str(at / "division.cpp"), str(at / "division.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run([build.hipcc(), "-x", "hip", "--offload-host-only", "-O2", "-std=c++17", "-fPIC", "-shared", "-I", build.CSRC, "-I",
                    os.path.join(build.ROOT, "include"), src, "-o", lib], check=True)
    fn = C.CDLL(lib).divide

    def call(new, kv, hq, hkv, d, max_pages, page_size, cus=256, ulps=0):
        new, kv = np.asarray(new, np.int32), np.asarray(kv, np.int32)
        desc = P.make_paged_desc(n_seqs=len(kv), n_tokens=int(new.sum()), max_new=int(new.max()), n_q_heads=hq, n_kv_heads=hkv, head_dim=d,
                                 dtype=P.BF16, n_pages=1, page_size=page_size, max_pages=max_pages)
        out = (C.c_int64 * 8)()
        fn(C.byref(desc), cus, ulps, new.ctypes.data_as(C.c_void_p), kv.ctypes.data_as(C.c_void_p), out)
        return dict(zip(("rows", "keys", "none", "spans", "cut", "parts", "slots", "workgroups"), out))
    return call


def check(r, what):
    assert not r["none"], what
    assert r["rows"] in (64, 128, 256) and r["keys"] >= 256 and r["keys"] % 64 == 0, (what, r)
    assert 0 < r["spans"] < 2 ** 31, (what, r)
    assert r["cut"] <= r["slots"], (what, r)     # every span of a cut unit has a slot of its own
    assert r["parts"] <= 4 ** 6, (what, r)       # as many levels of adding four up as a slot has counters for
    assert r["workgroups"] % 8 == 0 and r["workgroups"] > 0, (what, r)


MORE = [0, 1, 2, 63, 64, 65, 129]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("top", [1 << 24, 1 << 25, (1 << 29), (1 << 30) - 130])
@pytest.mark.parametrize("new,hq,hkv", [(4096, 32, 8), (4096, 32, 1), (260, 4, 1), (1000, 8, 2), (3000, 16, 16)])
def test_one_long_context(divide, top, new, hq, hkv, d):
    for more in MORE:
        for wide in (False, True):   # a table as wide as the context, or the widest
            pages = 1 << 14 if wide else -(-(top + more) // 65536)
            for ulps in (-1, 0, 1):
                check(divide([new], [top + more], hq, hkv, d, pages, 65536, ulps=ulps), (new, top + more, hq, hkv, d, wide, ulps))


@pytest.mark.parametrize("d", [64, 128])
def test_a_unit_of_the_chip_more_or_less(divide, d):
    """Row tiles around once, twice and four times the chip's units, where the choice of a division changes."""
    for tiles in (255, 256, 257, 511, 512, 513, 1023, 1024, 1025):
        for kv in (1, 255, 256, 257, 2500, 30000, (1 << 24) - 1, (1 << 24) + 1, (1 << 29) + 1, 1 << 30):
            for page in (1, 16, 1 << 20):
                check(divide([tiles * 256], [kv], 1, 1, d, -(-kv // page), page), (tiles, kv, page, d))


@pytest.mark.parametrize("seed", range(6))
def test_batches(divide, seed):
    """Sequences of all lengths beside each other, some empty, tables of any width; lengths past the table's end too."""
    rng = np.random.default_rng(seed)
    spread = lambda lo, hi, n=None: np.exp(rng.uniform(np.log(lo), np.log(hi), n)).astype(np.int64)
    for _ in range(1500):
        n = int(spread(1, 200))
        hkv = int(rng.choice([1, 2, 4, 8, 16]))
        hq = hkv * int(rng.choice([1, 2, 3, 4, 8, 32]))
        most = int(spread(300, 1 << 30))
        kv = np.minimum(spread(1, most + 1, n), most)
        if rng.random() < 0.5:
            kv = np.maximum(most - rng.integers(0, 200, n), 1)
        kv[rng.random(n) < 0.1] = 0
        new = np.minimum(spread(1, spread(2, 1 << 15) + 1, n), (1 << 30) // (hq * n))
        new[rng.random(n) < 0.1] = 0
        if new.max() == 0:
            new[0] = 1
        page = int(spread(1, 1 << 20))
        pages = max(-(-int(kv.max()) // page), 1)
        if rng.random() < 0.3:
            pages = min(2 * pages, (1 << 30) // page)
        pages = max(min(pages, (1 << 30) // page), 1)
        what = (seed, n, hq, hkv, most, page, pages)
        check(divide(new, kv, hq, hkv, int(rng.choice([64, 128])), pages, page, cus=int(rng.choice([32, 64, 256])), ulps=int(rng.integers(-1, 2))), what)


def test_no_rows_and_more_rows_than_there_are(divide):
    assert divide([1, 0], [5, 5], 1, 1, 64, 1, 16)["none"] == 0
    desc_rows = divide([0, 3], [0, 0], 4, 2, 128, 1, 16)
    assert not desc_rows["none"] and desc_rows["spans"] == 2     # a tile of either head, without keys


def test_the_division_of_ordinary_calls(divide):
    """The forms that the kernels' comments and the GPU tests speak of."""
    assert divide([2048], [32768], 32, 8, 128, 512, 64)["rows"] == 256
    assert divide([2048], [32768], 32, 8, 128, 512, 64)["cut"] == 0
    r = divide([1000], [64000], 8, 2, 128, 4000, 16)
    assert r["rows"] == 256 and r["parts"] > 1
    r = divide([1000], [1000], 8, 2, 128, 63, 16)
    assert r["rows"] < 256
