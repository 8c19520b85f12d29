"""Paged append and attention on the GPU against the fp64 oracle on the same bits.

Bounds of the attention, fixed before the first run.  u is half a step of the storage type (2^-8 bf16, 2^-11 half), E = 2^-24.  A
probability is rounded to the storage type for its product: u of sum p|v|/l (half: and 2^-25 of a weight that a lagging maximum keeps above 1).
A score's rounding, at most 2 head_dim E of sum|q||k| scale, is a relative one of its probability; n sums, the exponentials and the
combination of the spans cost (2 n + 64) E.  The stored o is rounded once more."""
import numpy as np
import pytest
import torch

import paper_2406_18485_amd as P
from gpu_harness import DEV
from oracle import paged_oracle as po
from oracle import rope_oracle as ro

pytestmark = pytest.mark.gpu

TORCH = {P.BF16: torch.bfloat16, P.FP16: torch.float16}
U = {P.BF16: (2.0 ** -8, 0.0), P.FP16: (2.0 ** -11, 2.0 ** -25)}
E = 2.0 ** -24


def f64(x):
    return x.detach().double().cpu().numpy()


class Case:
    """Sequences of `new` new among `kv` keys.  Slots without a key, and tokens of no sequence, hold NaN; pages lie in random order.
    `layout`: "heads" [page, head, slot, d], "tokens" [page, slot, head, d], "gaps" with NaN between the rows."""

    def __init__(self, new, kv, dtype=P.BF16, hq=4, hkv=2, d=128, page=16, causal=True, layout="heads", before=0, behind=0, spare=1, sigma=1.0,
                 max_new=None, clean=False, shared_prefix=0, seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.__dict__.update(new=new, kv=kv, dtype=dtype, hq=hq, hkv=hkv, d=d, page=page, causal=causal, clean=clean)
        n, t = len(kv), TORCH[dtype]
        self.starts = [before + sum(new[:i]) for i in range(n + 1)]
        self.tokens = self.starts[-1] + behind
        need = [-(-k // page) for k in kv]
        self.width = max(need + [1]) + spare
        total = sum(need) + 3
        order = torch.randperm(total, generator=gen).tolist()
        table, at = np.full((n, self.width + 2), -7), 0
        for b in range(n):
            table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
            same = min(shared_prefix // page, need[b], need[0])
            table[b, :same] = table[0, :same]
        self.table_np = table
        self.table = torch.tensor(table, dtype=torch.int32, device=DEV)
        self.n_pages = total
        shape = {"heads": (total, hkv, page, d), "tokens": (total, page, hkv, d), "gaps": (total, hkv, page, d + 8)}[layout]

        def cache():
            mem = torch.full(shape, float("nan"), dtype=t, device=DEV)
            return mem.transpose(1, 2) if layout == "tokens" else mem[..., :d]
        self.k_cache, self.v_cache = cache(), cache()
        for b in range(n):
            if kv[b]:
                j = np.arange(kv[b])
                pages, slots = torch.tensor(table[b, j // page], device=DEV), torch.tensor(j % page, device=DEV)
                for c in (self.k_cache, self.v_cache):
                    c[pages, :, slots] = torch.randn(kv[b], hkv, d, generator=gen).mul_(sigma).to(t).to(DEV)
        self.q = torch.full((self.tokens, hq, d), float("nan"), dtype=t, device=DEV)
        lo, hi = self.starts[0], self.starts[-1]
        self.q[lo:hi] = torch.randn(hi - lo, hq, d, generator=gen).mul_(sigma).to(t).to(DEV)
        self.seq_start = torch.tensor(self.starts, dtype=torch.int32, device=DEV)
        self.kv_len = torch.tensor(kv, dtype=torch.int32, device=DEV)
        self.scale = d ** -0.5
        self.max_new = max(new) if max_new is None else max_new
        self.reset()
        self.make_desc()

    def make_desc(self, **kw):
        self.desc = P.make_paged_desc(**{**dict(
            n_seqs=len(self.kv), n_tokens=self.tokens, max_new=self.max_new, n_q_heads=self.hq, n_kv_heads=self.hkv, head_dim=self.d,
            dtype=self.dtype, n_pages=self.n_pages, page_size=self.page, max_pages=self.width, table_stride=self.width + 2, causal=self.causal,
            softmax_scale=self.scale, flags=P.WORKSPACE_CLEAN if self.clean else 0, cache_stride=self.k_cache.stride()[:3]), **kw})
        n = max(P.paged_workspace_bytes(self.desc), 16)
        self.ws = torch.zeros(n, dtype=torch.uint8, device=DEV) if self.clean else torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)

    def reset(self):
        self.out = torch.full((self.tokens, self.hq, self.d), 7.0, device=DEV)
        self.o = torch.full((self.tokens, self.hq, self.d), 7.0, dtype=TORCH[self.dtype], device=DEV)
        self.lse = torch.full((self.tokens, self.hq), 7.0, device=DEV)

    def run(self, **kw):
        P.paged_attn(self.desc, self.q, self.k_cache, self.v_cache, self.seq_start, self.kv_len, self.table, self.out, self.o, self.lse,
                     self.ws, **kw)
        return self

    def want(self):
        kc, vc = f64(self.k_cache), f64(self.v_cache)
        args = self.scale, self.causal, self.starts, self.kv, self.table_np
        out, lse = po.attention(f64(self.q), kc, vc, *args)
        size, _ = po.attention(f64(self.q), kc, np.abs(vc), *args)
        return out, lse, size

    def check(self, finite=True):
        out, lse, size = self.want()
        got, got_o, got_lse = f64(self.out), f64(self.o), f64(self.lse)
        mine = ~np.isnan(lse)
        assert (got[~mine] == 7).all() and (got_o[~mine] == 7).all() and (got_lse[~mine] == 7).all()
        if not mine.any() or max(self.kv) == 0:
            assert np.isneginf(got_lse[mine]).all() and (got[mine] == 0).all() and (got_o[mine] == 0).all()
            return self
        out, lse, size, got, got_o, got_lse = (x[mine] for x in (out, lse, size, got, got_o, got_lse))
        blind = np.isneginf(lse)
        assert np.isneginf(got_lse[blind]).all() and (got[blind] == 0).all() and (got_o[blind] == 0).all()
        out, lse, size, got, got_o, got_lse = (x[~blind] for x in (out, lse, size, got, got_o, got_lse))
        u, small = U[self.dtype]
        n = max(self.kv + [1])
        dot = self.scale * 1.01 * np.sqrt(np.nanmax(f64(self.q) ** 2 @ np.ones(self.d)) * np.nanmax(f64(self.k_cache) ** 2 @ np.ones(self.d)))
        noise = (2 * n + 64) * E + 2 * self.d * E * dot
        off = (u + noise) * size + small * n * np.nanmax(np.abs(f64(self.v_cache)))
        err = np.abs(got - out)
        assert (err <= off).all(), (err.max(), (err / off).max())
        assert (np.abs(got_o - out) <= off + u * (np.abs(out) + off) + small).all()
        assert (np.abs(got_lse - lse) <= noise + 2 * E * np.abs(lse)).all(), np.abs(got_lse - lse).max()
        return self


LENGTHS = [  # new, kv
    ([1], [1]), ([1], [33]), ([1, 1, 1], [16, 200, 17]), ([5], [5]), ([3, 1, 7], [40, 1, 300]), ([40], [40]), ([130, 1, 70], [131, 77, 1000]),
    ([300], [345])]


@pytest.mark.parametrize("dtype", [P.BF16, P.FP16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("hq,hkv", [(4, 2), (3, 1), (2, 2)])
def test_lengths_types_and_heads(lengths, dtype, d, hq, hkv):
    Case(*lengths, dtype=dtype, d=d, hq=hq, hkv=hkv, seed=d + hq).run().check()


@pytest.mark.parametrize("page", [1, 7, 24, 128, 1000])
@pytest.mark.parametrize("layout", ["heads", "tokens", "gaps"])
@pytest.mark.parametrize("new,kv", [([1, 2], [500, 77]), ([50, 9], [500, 77])])
def test_pages_and_strides(new, kv, page, layout):
    Case(new, kv, page=page, layout=layout, seed=page).run().check()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("new,kv", [([1, 0, 2], [0, 9, 5]), ([4, 3], [2, 0]), ([0, 0], [5, 0]), ([60, 0, 50], [7, 0, 60]), ([90], [0])])
def test_rows_without_keys_and_sequences_without_tokens(new, kv, causal):
    Case(new, kv, causal=causal, before=3, behind=5).run().check()


@pytest.mark.parametrize("new", [1, 6, 200])
def test_without_a_mask(new):
    Case([new, new], [400, 37], causal=False, seed=new).run().check()


def test_more_groups_than_rows_of_a_tile():
    Case([1, 1], [70, 300], hq=40, hkv=1, seed=1).run().check()      # 40 rows of one token
    Case([2], [300], hq=16, hkv=1, seed=2).run().check()             # 32


@pytest.mark.parametrize("new,kv,page", [([1], [5000], 16), ([2, 1, 1], [9000, 300, 4100], 32), ([1], [4500], 1), ([260], [9000], 16), ([100, 1], [5000, 3000], 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_long_contexts_shared_by_workgroups(new, kv, page, d):
    c = Case(new, kv, page=page, d=d, hq=4, hkv=1, seed=page + d).run().check()
    first = c.out.clone(), c.lse.clone()
    c.reset()
    c.run()
    assert torch.equal(c.out, first[0]) and torch.equal(c.lse, first[1])


def test_many_sequences():
    rng = np.random.default_rng(0)
    Case([1] * 150, rng.integers(1, 90, 150).tolist(), hq=2, hkv=1, d=64, seed=3).run().check()
    Case([1] * 70 + [90] + [3] * 9, rng.integers(90, 120, 80).tolist(), hq=2, hkv=2, d=64, seed=4).run().check()


def test_shares_that_end_inside_units():
    """More grains than workgroups, lengths that are no multiples of a share; some sequences too short to be cut."""
    rng = np.random.default_rng(1)
    kv = rng.integers(700, 1600, 40).tolist() + rng.integers(1, 500, 30).tolist()
    c = Case([1] * 70, kv, hq=16, hkv=8, d=64, seed=20).run().check()
    first = c.out.clone()
    c.reset()
    c.run()
    assert torch.equal(c.out, first)


def reference_on_gpu(c):
    """Out, lse and attention of |v| in 64 bits, a head at a time (the sizes below are too long for the oracle)."""
    out, size = (torch.full((c.tokens, c.hq, c.d), float("nan"), dtype=torch.float64, device=DEV) for _ in range(2))
    lse = torch.full((c.tokens, c.hq), float("nan"), dtype=torch.float64, device=DEV)
    for b, (n, m) in enumerate(zip(c.new, c.kv)):
        at = slice(c.starts[b], c.starts[b] + n)
        pages = c.table[b, :-(-m // c.page)].long()
        for h in range(c.hq):
            keys, vals = (x[pages, h // (c.hq // c.hkv)].reshape(-1, c.d)[:m].double() for x in (c.k_cache, c.v_cache))
            s = c.q[at, h].double() @ keys.T * c.scale
            if c.causal:
                s.masked_fill_(torch.ones(n, m, dtype=torch.bool, device=DEV).triu(m - n + 1), float("-inf"))
            lse[at, h] = torch.logsumexp(s, -1)
            s.sub_(lse[at, h, None]).exp_()
            out[at, h], size[at, h] = s @ vals, s @ vals.abs()
    return out, lse, size


# row tiles of 64, 128 and 256 rows, whole and cut, by the lengths; tiles of 256 rows that fill the chip, at both head dimensions
FORMS = [([300], [700], 8, 2, 128), ([200, 1], [3000, 2500], 8, 2, 128), ([1000], [6000], 8, 2, 128), ([1000], [6100], 8, 2, 64), ([260], [40000], 4, 1, 128),
         ([40, 1, 33], [20000, 30000, 400], 4, 2, 64), ([2100], [2500], 32, 8, 128), ([1500, 700, 1], [1500, 3333, 900], 32, 4, 64), ([777], [5000], 96, 1, 64),
         # fewer rows than fill the chip with tiles of 256, head_dim 64, tables with room for many keys and for few
         ([700], [4800], 32, 8, 64), ([520, 9, 1], [2500, 4500, 100], 32, 4, 64), ([1, 0, 1100, 33], [9000, 0, 1100, 2000], 16, 16, 64), ([700], [2000], 32, 8, 64)]


@pytest.mark.parametrize("new,kv,hq,hkv,d", FORMS)
@pytest.mark.parametrize("dtype", [P.BF16, P.FP16])
def test_long_chunks_in_every_form(new, kv, hq, hkv, d, dtype):
    c = Case(new, kv, dtype=dtype, hq=hq, hkv=hkv, d=d, page=48, seed=21).run()
    out, lse, size = reference_on_gpu(c)
    u, small = U[dtype]
    dot = c.scale * 1.01 * (c.q.double().norm(dim=-1).max() * c.k_cache.double().nan_to_num().norm(dim=-1).max()).item()
    noise = (2 * max(kv) + 64) * E + 2 * d * E * dot
    off = (u + noise) * size + small * max(kv) * c.v_cache.double().nan_to_num().abs().max().item()
    assert ((c.out.double() - out).abs() <= off).all()
    assert ((c.o.double() - out).abs() <= off + u * (out.abs() + off) + small).all()
    assert ((c.lse.double() - lse).abs() <= noise + 2 * E * lse.abs()).all()
    first = c.out.clone()
    c.reset()
    c.run()
    assert torch.equal(c.out, first)
    # an infinity among the last values: the last token alone sees it
    b = 0
    page, slot = int(c.table_np[b, (kv[b] - 1) // c.page]), (kv[b] - 1) % c.page
    c.v_cache[page, :, slot, 1] = float("inf")
    c.reset()
    c.run()
    last = c.starts[b + 1] - 1
    assert (c.out[last, :, 1] == float("inf")).all()
    c.out[last, :, 1] = first[last, :, 1]
    assert torch.equal(c.out, first)


def test_large_scores_move_the_maximum():
    for new in ([1], [100]):
        Case(new, [700], sigma=6.0, seed=5).run().check()


def test_shared_pages():
    c = Case([1, 1, 2], [200, 170, 90], shared_prefix=64, seed=6)
    c.run().check()


@pytest.mark.parametrize("new", [[3], [64]])
def test_masked_values_that_are_not_finite_have_no_effect(new):
    c = Case(new, [100], d=64, seed=7).run()
    want = c.out.clone(), c.lse.clone()
    last = 99
    page, slot = int(c.table_np[0, last // c.page]), last % c.page
    c.v_cache[page, 0, slot, 3] = float("inf")
    c.v_cache[page, 0, slot, 40] = float("-inf")
    c.v_cache[page, 1, slot, 9] = float("nan")
    c.reset()
    c.run()
    assert torch.equal(c.out[:-1], want[0][:-1]) and torch.equal(c.lse, want[1])   # only the last token sees that key
    last_row = c.out[-1]
    assert (last_row[:2, 3] == float("inf")).all() and (last_row[:2, 40] == float("-inf")).all() and torch.isnan(last_row[2:, 9]).all()
    last_row[:2, 3] = want[0][-1, :2, 3]
    last_row[:2, 40] = want[0][-1, :2, 40]
    last_row[2:, 9] = want[0][-1, 2:, 9]
    assert torch.equal(last_row, want[0][-1])
    # a key of that kind
    c.k_cache[page, :, slot, 5] = float("nan")
    c.v_cache[page, :, slot] = 1.0
    c.reset()
    c.run()
    assert torch.equal(c.out[:-1], want[0][:-1]) and torch.isnan(c.out[-1]).all() and torch.isnan(c.lse[-1]).all()


@pytest.mark.parametrize("new,kv", [([4, 1], [90, 40]), ([80, 60], [90, 70]), ([1, 1], [3000, 40])])
def test_pages_outside_the_cache_give_nan_to_the_rows_that_see_them(new, kv):
    c = Case(new, kv, seed=8).run()
    want = c.out.clone(), c.lse.clone()
    for bad in (-1, c.n_pages, 2 ** 31 - 1, -2 ** 31):
        first = kv[0] - 1 - (kv[0] - 1) % c.page      # the page of the first sequence's last key
        c.table[0, first // c.page] = bad
        c.reset()
        c.run()
        sees = c.starts[1] - min(new[0], kv[0] - first)
        assert torch.isnan(c.out[sees:c.starts[1]]).all() and torch.isnan(c.lse[sees:c.starts[1]]).all()
        rest = [i for i in range(c.tokens) if not sees <= i < c.starts[1]]
        assert torch.equal(c.out[rest], want[0][rest]) and torch.equal(c.lse[rest], want[1][rest])


def test_lengths_past_the_page_table_give_nan_and_bad_starts_access_nothing():
    c = Case([1, 2], [64, 40], spare=0, seed=9).run()
    want = c.out.clone()
    c.kv_len[0] = 2 ** 31 - 1
    c.reset()
    c.run()
    assert torch.isnan(c.out[0]).all() and torch.isnan(c.lse[0]).all() and torch.equal(c.out[1:], want[1:])
    c.kv_len[0] = -5
    c.reset()
    c.run()
    assert (c.out[0] == 0).all() and torch.isneginf(c.lse[0]).all() and torch.equal(c.out[1:], want[1:])
    for starts in ([-9, 1, 99], [0, 2 ** 31 - 1, 3], [3, 2, 1], [-2 ** 31, -1, -1]):
        c.seq_start.copy_(torch.tensor(starts, dtype=torch.int32))
        c.run()
    torch.cuda.synchronize()


def test_no_more_than_max_new_tokens_of_a_sequence():
    c = Case([3, 1], [50, 20], max_new=2, seed=10).run()
    full = Case([3, 1], [50, 20], seed=10).run()
    assert torch.equal(c.out[:2], full.out[:2]) and torch.equal(c.out[3:], full.out[3:]) and (c.out[2] == 7).all() and (c.lse[2] == 7).all()


def test_either_result_alone_and_their_strides():
    c = Case([2, 40], [60, 90], seed=11).run()
    out, o, lse = c.out.clone(), c.o.clone(), c.lse.clone()
    for which in ("out", "o"):
        c.reset()
        keep = getattr(c, which)
        P.paged_attn(c.desc, c.q, c.k_cache, c.v_cache, c.seq_start, c.kv_len, c.table, c.out if which == "out" else None,
                     c.o if which == "o" else None, c.lse, c.ws)
        assert torch.equal(keep, out if which == "out" else o) and torch.equal(c.lse, lse)
    # head-major results with room between them, from queries that are part of a projection
    big = torch.full((c.hq, c.tokens, c.d + 8), 5.0, device=DEV)
    packed = torch.full((c.tokens, c.hq + 4, c.d), float("nan"), dtype=torch.bfloat16, device=DEV)
    packed[:, :c.hq] = c.q
    view = big[..., :c.d].transpose(0, 1)
    c.make_desc(o_stride=view.stride()[:2], q_stride=packed.stride()[:2])
    P.paged_attn(c.desc, packed, c.k_cache, c.v_cache, c.seq_start, c.kv_len, c.table, view, None, c.lse, c.ws)
    assert torch.equal(view, out) and (big[..., c.d:] == 5).all()


def test_a_cache_of_more_than_4_gib():
    """Pages 2^31 bytes apart and more: offsets that pass 32 bits, in elements too."""
    gen = torch.Generator().manual_seed(12)
    hkv, page, d, far = 2, 16, 64, (1 << 31) + 64
    mem = [torch.empty(far + hkv * page * d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    caches = [m.as_strided((2, hkv, page, d), (far, page * d, d, 1)) for m in mem]
    small = [torch.randn(2, hkv, page, d, generator=gen).to(torch.bfloat16).to(DEV) for _ in range(2)]
    for c, s in zip(caches, small):
        c.copy_(s)
    q = torch.randn(16, 12, d, generator=gen).to(torch.bfloat16).to(DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    table = torch.tensor([[1, 0], [0, 1]], **i32)
    for new in (1, 8):   # 6 and 48 rows; no slot is written twice
        got = []
        for cache in (caches, small):
            desc = P.make_paged_desc(n_seqs=2, n_tokens=2 * new, n_q_heads=12, n_kv_heads=hkv, head_dim=d, dtype=P.BF16, n_pages=2,
                                     page_size=page, max_pages=2, cache_stride=cache[0].stride()[:3])
            out, lse = torch.empty(2 * new, 12, d, device=DEV), torch.empty(2 * new, 12, device=DEV)
            k, v = q[:2 * new, :hkv].contiguous(), q[:2 * new, 2:].contiguous()
            P.paged_append(desc, None, k, v, None, None, torch.ones(d // 2, device=DEV), None, torch.tensor([0, new, 2 * new], **i32),
                           torch.tensor([32, 25], **i32), table, None, *cache)
            P.paged_attn(desc, q, *cache, torch.tensor([0, new, 2 * new], **i32), torch.tensor([32, 25], **i32), table, out, None, lse)
            got.append((out, lse))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
        assert torch.equal(caches[0], small[0]) and torch.equal(caches[1], small[1])


def test_another_stream_and_replays_that_follow_the_lengths():
    c = Case([1, 1], [3000, 500], hq=4, hkv=1, spare=2, clean=True, seed=13)
    lengths = [[3000, 500], [2990, 1], [300, 499], [1, 2]]
    want = []
    for kv in lengths:
        c.kv_len.copy_(torch.tensor(kv, dtype=torch.int32))
        c.reset()
        c.run()
        want.append((c.out.clone(), c.lse.clone()))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run()
    side.synchronize()
    assert torch.equal(c.out, want[-1][0])
    for clean in (True, False):
        c.clean = clean
        c.make_desc()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.run()
        for _ in range(2):
            for kv, (out, lse) in zip(lengths, want):
                c.kv_len.copy_(torch.tensor(kv, dtype=torch.int32))
                c.out.fill_(3.0)
                graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(c.out, out) and torch.equal(c.lse, lse)
    assert (c.ws[:P.WORKSPACE_HEAD] == 0).all()


def test_parts_of_a_context_merge_to_the_whole():
    """A context whose pages lie on two ranks: the earlier part without a mask, the later one causal, merged by the running update."""
    c = Case([2, 20], [700, 400], page=32, seed=14).run()
    first = [320, 96]      # keys on the other rank: whole pages
    parts = []
    for causal, kv, at in ((False, first, [0, 0]), (True, [k - f for k, f in zip(c.kv, first)], [f // c.page for f in first])):
        table = torch.stack([torch.roll(c.table[b, :c.width], -at[b]) for b in range(2)]).contiguous()
        desc = P.make_paged_desc(n_seqs=2, n_tokens=c.tokens, n_q_heads=c.hq, n_kv_heads=c.hkv, head_dim=c.d, dtype=c.dtype, n_pages=c.n_pages,
                                 page_size=c.page, max_pages=c.width, causal=causal)
        out, lse = torch.empty_like(c.out), torch.empty_like(c.lse)
        ws = torch.empty(max(P.paged_workspace_bytes(desc), 16), dtype=torch.uint8, device=DEV)
        P.paged_attn(desc, c.q, c.k_cache, c.v_cache, c.seq_start, torch.tensor(kv, dtype=torch.int32, device=DEV), table, out, None, lse, ws)
        parts.append((out, lse))
    (out, lse), (out2, lse2) = parts
    P.lse_merge(c.tokens * c.hq, c.d, out, lse, out2, lse2)
    c.out, c.lse = out, lse
    c.o = out.to(TORCH[c.dtype])
    c.check()


# ---- append --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [P.BF16, P.FP16])
@pytest.mark.parametrize("d,rot", [(128, 128), (64, 32), (128, 0)])
@pytest.mark.parametrize("norm,inter", [(False, False), (True, False), (True, True)])
@pytest.mark.parametrize("given", [False, True])
def test_append_against_the_oracle(dtype, d, rot, norm, inter, given):
    new, kv = [1, 0, 30, 5, 2], [40, 9, 30, 200, 1]     # the last one's first token has no slot
    c = Case(new, kv, dtype=dtype, d=d, hq=6, hkv=2, page=24, layout="tokens", before=2, behind=3, seed=15)
    gen = torch.Generator().manual_seed(16)
    t = TORCH[dtype]
    k, v = (torch.randn(c.tokens, 2, d, generator=gen).to(t).to(DEV) for _ in range(2))
    wq, wk = (1 + 0.3 * torch.randn(d, generator=gen).to(DEV) if norm else None for _ in range(2))
    f = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float().to(DEV)
    pos = torch.randint(-10, 1 << 20, (c.tokens,), generator=gen, dtype=torch.int32) if given else None
    before = f64(c.k_cache), f64(c.v_cache)
    q_out = torch.full_like(c.q, 7.0)
    desc = P.make_paged_desc(n_seqs=5, n_tokens=c.tokens, n_q_heads=6, n_kv_heads=2, head_dim=d, dtype=dtype, n_pages=c.n_pages, page_size=24,
                             max_pages=c.width, table_stride=c.width + 2, rot_dim=rot, eps=1e-5,
                             flags=(P.QK_NORM if norm else 0) | (P.ROPE_INTERLEAVED if inter else 0), cache_stride=c.k_cache.stride()[:3])
    P.paged_append(desc, c.q, k, v, wq, wk, f, None if pos is None else pos.to(DEV), c.seq_start, c.kv_len, c.table, q_out, c.k_cache, c.v_cache)
    w = lambda x: None if x is None else f64(x)
    kc, vc = po.append(*before, f64(k), f64(v), w(wk), 1e-5, None if pos is None else pos.numpy(), f64(f), inter, norm, c.starts, kv, c.table_np)
    got_k, got_v = f64(c.k_cache), f64(c.v_cache)
    assert np.array_equal(got_v, vc, equal_nan=True)
    assert np.array_equal(np.isnan(got_k), np.isnan(kc))
    u, small = U[dtype]
    # (the norm-and-rotation bound of the rope tests, with |n_a| + |n_b| below sqrt 2 times the row's norm: at most sqrt d max|w|, or |k|)
    size = 1.5 * (np.sqrt(d) * f64(wk).__abs__().max() if norm else np.sqrt((f64(k) ** 2).sum(-1)).max())
    ok = ~np.isnan(kc)
    assert (np.abs(got_k - kc)[ok] <= (32 * E * size + u * (np.abs(kc) + 32 * E * size) + small)[ok]).all()
    # queries as by the rotation alone
    lo, hi = c.starts[0], c.starts[-1]
    slots = np.concatenate([np.arange(m - n, m) for n, m in zip(new, kv)])
    want = ro.rope_forward(f64(c.q)[lo:hi], w(wq), 1e-5, (slots if pos is None else pos.numpy()[lo:hi])[:, None], f64(f), inter, norm)
    size = 1.5 * (np.sqrt(d) * f64(wq).__abs__().max() if norm else np.sqrt((f64(c.q)[lo:hi] ** 2).sum(-1)).max())
    assert (np.abs(f64(q_out)[lo:hi] - want) <= 32 * E * size + u * (np.abs(want) + 32 * E * size) + small).all()
    assert (q_out[:lo] == 7).all() and (q_out[hi:] == 7).all()


def test_append_drops_what_has_no_page_and_bad_starts_access_nothing():
    c = Case([3, 2], [20, 40], seed=17)
    gen = torch.Generator().manual_seed(18)
    k, v = (torch.randn(5, 2, 128, generator=gen).to(torch.bfloat16).to(DEV) for _ in range(2))
    desc = P.make_paged_desc(n_seqs=2, n_tokens=5, n_q_heads=4, n_kv_heads=2, head_dim=128, dtype=P.BF16, n_pages=c.n_pages, page_size=16,
                             max_pages=c.width, table_stride=c.width + 2, rot_dim=0)
    before = c.k_cache.clone(), c.v_cache.clone()

    def call():
        P.paged_append(desc, None, k, v, None, None, None, None, c.seq_start, c.kv_len, c.table, None, c.k_cache, c.v_cache)
        torch.cuda.synchronize()
    same = lambda: all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(before, (c.k_cache, c.v_cache)))
    for bad in (-1, c.n_pages, 2 ** 31 - 1):
        c.table.fill_(bad)
        call()
        assert same()
    c.table.fill_(0)
    for kv in ([-5, -9], [2 ** 31 - 1, 2 ** 31 - 1], [0, 0]):
        c.kv_len.copy_(torch.tensor(kv, dtype=torch.int32))
        call()
        assert same()
    for starts in ([-9, -5, -1], [9, 9, 99], [2 ** 31 - 1, 3, 0]):
        c.seq_start.copy_(torch.tensor(starts, dtype=torch.int32))
        call()
        assert same()


def test_a_prompt_and_decoding_steps_together():
    """A prompt in two chunks, then token by token, appended and attended to in a captured step whose lengths move on; and the same
    sequence in one go through the rotation and the unmasked steps' own forward, causal with one chunk pair."""
    hq, hkv, d, page, total, prompt = 4, 2, 128, 16, 96, 84
    gen = torch.Generator().manual_seed(19)
    mk = lambda h: torch.randn(1, total, h, d, generator=gen).to(torch.bfloat16).to(DEV)
    q, k, v = mk(hq), mk(hkv), mk(hkv)
    wq, wk = (1 + 0.2 * torch.randn(d, generator=gen).to(DEV) for _ in range(2))
    f = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float().to(DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    width = total // page
    table = torch.randperm(width, generator=gen).to(**i32)[None].contiguous()
    k_cache, v_cache = (torch.full((width, hkv, page, d), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    out, lse = torch.empty(total, hq, d, device=DEV), torch.empty(total, hq, device=DEV)

    def step(n, qs, ks, vs, q_rot, kv_len, out, lse):
        desc = P.make_paged_desc(n_seqs=1, n_tokens=n, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=P.BF16, n_pages=width, page_size=page,
                                 max_pages=width, eps=1e-5)
        desc.flags = P.QK_NORM
        start = torch.tensor([0, n], **i32)

        def run():
            desc.flags = P.QK_NORM
            P.paged_append(desc, qs, ks, vs, wq, wk, f, None, start, kv_len, table, q_rot, k_cache, v_cache)
            desc.flags = 0
            P.paged_attn(desc, q_rot, k_cache, v_cache, start, kv_len, table, out, None, lse)
        return run
    q_rot = torch.empty(total, hq, d, dtype=torch.bfloat16, device=DEV)
    for lo, hi in ((0, 50), (50, prompt)):
        step(hi - lo, q[0, lo:hi], k[0, lo:hi], v[0, lo:hi], q_rot[lo:hi], torch.tensor([hi], **i32), out[lo:hi], lse[lo:hi])()
    one = [x[0, :1].clone() for x in (q, k, v)]
    kv_len, q1, o1, l1 = torch.tensor([prompt], **i32), torch.empty_like(one[0]), torch.empty(1, hq, d, device=DEV), torch.empty(1, hq, device=DEV)
    run = step(1, *one, q1, kv_len, o1, l1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for t in range(prompt, total):
        for dst, src in zip(one, (q, k, v)):
            dst.copy_(src[0, t:t + 1])
        kv_len.fill_(t + 1)
        graph.replay()
        out[t], lse[t], q_rot[t] = o1[0], l1[0], q1[0]
    # in one go
    half = total // 2
    rd = P.make_rope_desc(batch=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, len=total, dtype=P.BF16, eps=1e-5, flags=P.QK_NORM,
                          chunk_len=half, chunk=(0, 1), q_stride=(0, d, hq * d), k_stride=(0, d, hkv * d))
    qr, kr = (torch.empty(1, h, total, d, dtype=torch.bfloat16, device=DEV) for h in (hq, hkv))
    P.qk_rope_fwd(rd, q, k, wq, wk, f, None, qr, kr)
    assert torch.equal(qr[0].transpose(0, 1), q_rot)
    vv = v.transpose(1, 2).contiguous()
    sd = P.make_desc(batch=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, q_len=total, kv_len=total, dtype=P.BF16, softmax_scale=d ** -0.5,
                     causal=True, chunk_len=half, q_chunk=(0, 1), kv_chunk=(0, 1))
    whole, whole_lse = torch.empty(1, hq, total, d, device=DEV), torch.empty(1, hq, total, device=DEV)
    P.attn_step_fwd(sd, qr, kr, vv, whole, whole_lse)
    assert (whole[0].transpose(0, 1) - out).abs().max() <= 2 * 2.0 ** -8 * vv.float().abs().max()   # u of sum p|v|, of both
    assert (whole_lse[0].T - lse).abs().max() <= 1e-4
