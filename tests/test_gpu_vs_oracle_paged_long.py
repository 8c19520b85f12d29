"""Paged calls on the GPU where a context has more parts than are added up at a time, and where a group of lanes appends many heads.
Bounds as in the tests of short calls (test_gpu_vs_oracle_paged)."""
import numpy as np
import pytest
import torch

import paper_2406_18485_amd as P
from gpu_harness import DEV
from oracle import paged_oracle as po
from oracle import rope_oracle as ro
from test_gpu_vs_oracle_paged import E, TORCH, U, Case, f64, reference_on_gpu

pytestmark = pytest.mark.gpu

PART, FAN = 256, 64     # keys of a part of a context that has the chip to itself, up to 131072 of them; parts that are added up at a time


def check(c):
    out, lse, size = reference_on_gpu(c)
    blind = torch.isneginf(lse)       # rows that see no key (the reference's softmax of nothing is NaN)
    assert torch.equal(blind, torch.isneginf(c.lse)) and (c.out[blind] == 0).all() and (c.o[blind] == 0).all()
    out[blind], size[blind], lse[blind] = 0, 0, float("-inf")
    u, small = U[c.dtype]
    dot = c.scale * 1.01 * (c.q.double().norm(dim=-1).max() * c.k_cache.double().nan_to_num().norm(dim=-1).max()).item()
    noise = (2 * max(c.kv) + 64) * E + 2 * c.d * E * dot
    off = (u + noise) * size + small * max(c.kv) * c.v_cache.double().nan_to_num().abs().max().item()
    assert ((c.out.double() - out).abs() <= off).all()
    assert ((c.o.double() - out).abs() <= off + u * (out.abs() + off) + small).all()
    assert ((c.lse.double() - lse).abs()[~blind] <= (noise + 2 * E * lse.abs())[~blind]).all()
    assert (c.ws[:P.WORKSPACE_HEAD] == 0).all()       # every counter is back at zero
    first = c.out.clone(), c.lse.clone()
    c.reset()
    c.run()
    assert torch.equal(c.out, first[0]) and torch.equal(c.lse, first[1])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq", [1, 8, 32])
@pytest.mark.parametrize("kv", [PART * (FAN - 1) + 1, PART * FAN, PART * FAN + 1, PART * (FAN + 1), 2 * PART * FAN, 2 * PART * FAN + 1, 4 * PART * FAN - 3])
def test_parts_around_what_is_added_up_at_a_time(kv, hq, d):
    """63, 64 (one level), 65 (a lone last part), 66, 128, 129 and 256 parts."""
    check(Case([1], [kv], hq=hq, hkv=1, d=d, page=64, clean=True, seed=hq + d).run())


@pytest.mark.parametrize("dtype", [P.BF16, P.FP16])
@pytest.mark.parametrize("d", [64, 128])
def test_long_contexts_of_unequal_lengths(d, dtype):
    # apart from each other: every unit begins with a share of its own
    check(Case([1, 1, 2], [70001, 30000, 17000], dtype=dtype, hq=8, hkv=1, d=d, page=48, clean=True, seed=1).run())
    # 2559 grains of 64 keys in shares of 5: the second unit begins inside one
    check(Case([1, 1], [1001 * 64, 1558 * 64], dtype=dtype, hq=4, hkv=1, d=d, page=256, clean=True, seed=2).run())
    # and with sequences that are not cut between them
    check(Case([1, 2, 1, 1, 3, 1], [20000, 100, 41000, 512, 1, 33333], dtype=dtype, hq=8, hkv=2, d=d, page=16, clean=True, seed=3).run())


def test_rows_that_see_less_than_the_longest():
    """Drafted tokens at the border of a part, and more new tokens than are asked for."""
    check(Case([4], [PART * (FAN + 1) + 2], hq=4, hkv=1, d=128, page=64, clean=True, seed=4).run())
    c = Case([6], [PART * FAN + 4], hq=4, hkv=1, d=64, page=64, max_new=2, clean=True, seed=5).run()
    full = Case([6], [PART * FAN + 4], hq=4, hkv=1, d=64, page=64, clean=True, seed=5)
    out, lse, size = reference_on_gpu(full)
    noise = (2 * full.kv[0] + 64) * E
    assert ((c.out.double() - out).abs()[:2] <= (U[P.BF16][0] + noise + 1e-5) * size[:2]).all() and (c.out[2:] == 7).all()
    assert ((c.lse.double() - lse).abs()[:2] <= 1e-4).all() and (c.ws[:P.WORKSPACE_HEAD] == 0).all()


def test_replays_between_one_level_and_two():
    c = Case([1, 1], [70000, 40000], hq=4, hkv=1, d=64, page=64, clean=True, seed=6)
    lengths = [[70000, 40000], [PART * FAN, PART * FAN], [PART * FAN + 1, 5], [300, 40000], [1, 0], [70000, 39999]]
    want = []
    for kv in lengths:
        c.kv_len.copy_(torch.tensor(kv, dtype=torch.int32))
        c.reset()
        c.run()
        want.append((c.out.clone(), c.lse.clone()))
    torch.cuda.synchronize()
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


@pytest.mark.parametrize("dtype,d,rot,norm,inter", [(P.BF16, 128, 128, True, False), (P.FP16, 64, 32, False, True)])
def test_append_of_many_tokens(dtype, d, rot, norm, inter):
    """Several heads a group of lanes: of q, of k and of v."""
    new, kv, hq, hkv = [7001, 1, 2300, 4099], [9000, 50, 2300, 4100], 9, 3
    c = Case(new, kv, dtype=dtype, d=d, hq=hq, hkv=hkv, page=48, before=1, behind=2, seed=7)
    lanes = d // 16
    assert -(-c.tokens // (256 // lanes)) * (hq + 2 * hkv) >= 2 * 4 * torch.cuda.get_device_properties(0).multi_processor_count
    gen = torch.Generator().manual_seed(8)
    k, v = (torch.randn(c.tokens, hkv, d, generator=gen).to(TORCH[dtype]).to(DEV) for _ in range(2))
    wq, wk = (1 + 0.3 * torch.randn(d, generator=gen).to(DEV) if norm else None for _ in range(2))
    f = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().to(DEV)
    before = f64(c.k_cache), f64(c.v_cache)
    q_out = torch.full_like(c.q, 7.0)
    desc = P.make_paged_desc(n_seqs=len(kv), n_tokens=c.tokens, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=dtype, n_pages=c.n_pages, page_size=48,
                             max_pages=c.width, table_stride=c.width + 2, rot_dim=rot, eps=1e-5,
                             flags=(P.QK_NORM if norm else 0) | (P.ROPE_INTERLEAVED if inter else 0))
    P.paged_append(desc, c.q, k, v, wq, wk, f, None, c.seq_start, c.kv_len, c.table, q_out, c.k_cache, c.v_cache)
    w = lambda x: None if x is None else f64(x)
    kc, vc = po.append(*before, f64(k), f64(v), w(wk), 1e-5, None, f64(f), inter, norm, c.starts, kv, c.table_np)
    got_k, got_v = f64(c.k_cache), f64(c.v_cache)
    assert np.array_equal(got_v, vc, equal_nan=True) and np.array_equal(np.isnan(got_k), np.isnan(kc))
    u, small = U[dtype]

    def close(got, want, x, weight):
        size = 1.5 * (np.sqrt(d) * np.abs(f64(weight)).max() if norm else np.sqrt((f64(x) ** 2).sum(-1)).max())
        assert (np.abs(got - want) <= 32 * E * size + u * (np.abs(want) + 32 * E * size) + small).all()
    ok = ~np.isnan(kc)
    close(got_k[ok], kc[ok], k, wk)
    lo, hi = c.starts[0], c.starts[-1]
    slots = np.concatenate([np.arange(m - n, m) for n, m in zip(new, kv)])
    close(f64(q_out)[lo:hi], ro.rope_forward(f64(c.q)[lo:hi], w(wq), 1e-5, slots[:, None], f64(f), inter, norm), c.q[lo:hi], wq)
    assert (q_out[:lo] == 7).all() and (q_out[hi:] == 7).all()


@pytest.mark.parametrize("dtype", [P.BF16, P.FP16])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("rot", [0, 32])
def test_appended_infinities_and_nan_in_elements_that_are_not_rotated(dtype, rot, inter):
    c = Case([5], [12], dtype=dtype, d=64, hq=4, hkv=2, seed=9)
    k, v = torch.randn(5, 2, 64, device=DEV).to(TORCH[dtype]), torch.randn(5, 2, 64, device=DEV).to(TORCH[dtype])
    for x in (c.q, k):
        x[0, :, rot], x[1, :, 63], x[3, :, rot + 5] = float("inf"), float("-inf"), float("nan")
    q_out = torch.full_like(c.q, 7.0)
    desc = P.make_paged_desc(n_seqs=1, n_tokens=5, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=dtype, n_pages=c.n_pages, page_size=16,
                             max_pages=c.width, table_stride=c.width + 2, rot_dim=rot, flags=P.ROPE_INTERLEAVED if inter else 0)
    f = torch.ones(max(rot // 2, 1), device=DEV)
    P.paged_append(desc, c.q, k, v, None, None, f, None, c.seq_start, c.kv_len, c.table, q_out, c.k_cache, c.v_cache)
    slots = c.k_cache[int(c.table_np[0, 0]), :, 7:12].transpose(0, 1)
    same = lambda a, b: torch.equal(a[..., rot:].nan_to_num(nan=77.0), b[..., rot:].nan_to_num(nan=77.0))
    assert same(q_out, c.q) and same(slots, k)
    assert torch.isfinite(q_out[..., :rot]).all() and torch.isfinite(slots[..., :rot]).all()


def test_queries_of_a_sequence_whose_length_is_negative_are_rotated_as_with_none():
    """A negative kv_len counts as 0: its new tokens lie before the first slot."""
    c = Case([4, 3], [0, 9], hq=4, hkv=2, d=128, seed=10)
    k, v = (torch.randn(7, 2, 128, device=DEV).to(torch.bfloat16) for _ in range(2))
    desc = P.make_paged_desc(n_seqs=2, n_tokens=7, n_q_heads=4, n_kv_heads=2, head_dim=128, dtype=P.BF16, n_pages=c.n_pages, page_size=16,
                             max_pages=c.width, table_stride=c.width + 2)
    f = (10000.0 ** (-torch.arange(0, 128, 2, dtype=torch.float64) / 128)).float().to(DEV)
    got = []
    for kv in (0, -1, -1000, -2 ** 31):
        c.kv_len[0] = kv
        q_out = torch.full_like(c.q, 7.0)
        P.paged_append(desc, c.q, k, v, None, None, f, None, c.seq_start, c.kv_len, c.table, q_out, c.k_cache, c.v_cache)
        got.append(q_out)
    assert all(torch.equal(x, got[0]) for x in got)
    want = ro.rope_forward(f64(c.q)[:4], None, 0.0, np.arange(-4, 0)[:, None], f64(f), False, False)
    assert np.abs(f64(got[0])[:4] - want).max() <= 2.0 ** -8 * np.abs(want).max() + 1e-5


@pytest.mark.parametrize("dtype", [P.BF16, P.FP16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,hq,hkv", [(1, 8, 1), (7, 8, 2), (300, 4, 1), (1100, 32, 4)])
def test_many_small_probabilities_beside_a_large_one(new, hq, hkv, d, dtype):
    """One key that takes nearly all, and some 10^5 whose probabilities, 2^-23 to 2^-27 of its, have a per cent together.

    A probability's rounding is u of itself, or half a step below the type's normal numbers: half, 2^-25, where the largest is 2^7 at least.
    The rest of the bound is that of the short calls."""
    kv = 120000
    c = Case([new], [kv], dtype=dtype, hq=hq, hkv=hkv, d=d, page=64, clean=True, seed=11)
    gen = torch.Generator(device=DEV).manual_seed(12)
    pages, slots = torch.tensor(c.table_np[0, np.arange(kv) // 64], device=DEV), torch.arange(kv, device=DEV) % 64
    # q all ones but for a little; scores of -0.5 to 0.5 a key, and one of 17 (log2: 24.5)
    c.q.copy_(1 + 0.01 * torch.randn(c.q.shape, device=DEV, generator=gen))
    keys = 0.3 * torch.randn(kv, hkv, d, device=DEV, generator=gen)
    keys -= keys.mean(-1, keepdim=True)
    keys += (torch.rand(kv, hkv, 1, device=DEV, generator=gen) - 0.5) / (d * c.scale)
    keys[kv // 3] = 17.0 / (d * c.scale)
    c.k_cache[pages, :, slots] = keys.to(TORCH[dtype])
    values = 1 + 0.1 * torch.randn(kv, hkv, d, device=DEV, generator=gen)
    values[kv // 3] = 0
    c.v_cache[pages, :, slots] = values.to(TORCH[dtype])
    c.run()
    out, lse, size = reference_on_gpu(c)
    assert 1e-3 < out.mean() < 2e-2
    u = U[dtype][0]
    dot = c.scale * 1.01 * (c.q.double().norm(dim=-1).max() * keys.double().norm(dim=-1).max()).item()
    noise = (2 * kv + 64) * E + 2 * d * E * dot
    off = (u + noise) * size + (kv * 2.0 ** -32 * 1.6 if dtype == P.FP16 else 0)      # (|v| below 1.6)
    assert ((c.out.double() - out).abs() <= off).all(), ((c.out.double() - out).abs() / off).max()
    assert ((c.lse.double() - lse).abs() <= noise + 2 * E * lse.abs()).all()


@pytest.mark.parametrize("dtype", [P.BF16, P.FP16])
@pytest.mark.parametrize("new,kv,hq,hkv,d,page", [([1], [1000], 8, 8, 128, 16), ([1, 1, 1], [300, 4000, 7], 16, 2, 64, 24), ([5, 3], [4000, 900], 12, 2, 128, 32),
                                                  ([1, 2], [30000, 17], 8, 1, 128, 64)])
def test_few_rows_keep_both_pieces_of_a_probability(new, kv, hq, hkv, d, page, dtype):
    """The second piece rounds what the first leaves: u of u of sum p|v|/l (half: and 2^-25 of what is 2^7 at least)."""
    c = Case(new, kv, dtype=dtype, hq=hq, hkv=hkv, d=d, page=page, clean=True, seed=13).run()
    out, lse, size = reference_on_gpu(c)
    u = U[dtype][0]
    dot = c.scale * 1.01 * (c.q.double().norm(dim=-1).max() * c.k_cache.double().nan_to_num().norm(dim=-1).max()).item()
    noise = (2 * max(kv) + 64) * E + 2 * d * E * dot
    off = (u * u + noise) * size + (max(kv) * 2.0 ** -32 * c.v_cache.double().nan_to_num().abs().max() if dtype == P.FP16 else 0)
    assert ((c.out.double() - out).abs() <= off).all(), ((c.out.double() - out).abs() / off).max()


@pytest.mark.parametrize("new", [[1] * 4200, [1] * 4197 + [0, 70, 2], [0] * 290 + [1, 0, 2, 0, 0, 3, 0, 0, 1, 0], [0] * 290 + [40, 0, 2, 0, 0, 3, 0, 0, 1, 0]])
def test_thousands_of_sequences(new):
    """More than a wave has lanes for 64 at a time; and more than there are tokens."""
    rng = np.random.default_rng(14)
    kv = [int(rng.integers(1, 100)) if n == 1 else n + int(rng.integers(0, 60)) for n in new]
    c = Case(new, kv, hq=2, hkv=1, d=64, seed=15).run().check()
    gen = torch.Generator().manual_seed(16)
    # and appended: every sequence's tokens are found
    k, v = (torch.randn(c.tokens, 1, 64, generator=gen).to(torch.bfloat16).to(DEV) for _ in range(2))
    desc = P.make_paged_desc(n_seqs=len(kv), n_tokens=c.tokens, n_q_heads=2, n_kv_heads=1, head_dim=64, dtype=P.BF16, n_pages=c.n_pages, page_size=16,
                             max_pages=c.width, table_stride=c.width + 2, rot_dim=0)
    want_k, want_v = c.k_cache.clone(), c.v_cache.clone()
    P.paged_append(desc, None, k, v, None, None, None, None, c.seq_start, c.kv_len, c.table, None, c.k_cache, c.v_cache)
    seq = np.repeat(np.arange(len(new)), new)
    pos = np.concatenate([np.arange(m - n, m) for n, m in zip(new, kv)])
    pages, slots = torch.tensor(c.table_np[seq, pos // 16], device=DEV), torch.tensor(pos % 16, device=DEV)
    want_k[pages, 0, slots], want_v[pages, 0, slots] = k[:, 0], v[:, 0]
    assert torch.equal(c.k_cache.view(torch.int16), want_k.view(torch.int16)) and torch.equal(c.v_cache.view(torch.int16), want_v.view(torch.int16))


@pytest.mark.parametrize("dtype", [P.BF16, P.FP16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,kv,hq,hkv", [([1], [1000], 8, 2), ([4], [5000], 8, 1), ([1, 3], [40000, 700], 4, 1), ([120], [900], 4, 1)])
def test_infinite_values_that_rows_see(new, kv, hq, hkv, d, dtype):
    """In the middle of the context: a column of one, of both signs, of a NaN; all else as it was."""
    c = Case(new, kv, dtype=dtype, hq=hq, hkv=hkv, d=d, page=32, clean=True, seed=17).run()
    want = c.out.clone(), c.lse.clone()
    odd = [(3, 10, "inf"), (3, kv[0] // 2, "inf"), (9, kv[0] // 3, "-inf"), (11, 77, "inf"), (11, kv[0] // 2, "-inf"), (40, 200, "nan"), (41, 0, "inf"), (d - 1, 333, "-inf")]
    for col, key, x in odd:
        c.v_cache[int(c.table_np[0, key // c.page]), :, key % c.page, col] = float(x)
    c.reset()
    c.run()
    mine = slice(c.starts[0], c.starts[1])
    for col, x in ((3, "inf"), (9, "-inf"), (41, "inf"), (d - 1, "-inf")):
        assert (c.out[mine, :, col] == float(x)).all() and (c.o[mine, :, col] == float(x)).all(), col
        c.out[mine, :, col] = want[0][mine, :, col]
    for col in (11, 40):
        assert torch.isnan(c.out[mine, :, col]).all() and torch.isnan(c.o[mine, :, col]).all(), col
        c.out[mine, :, col] = want[0][mine, :, col]
    assert torch.equal(c.out, want[0]) and torch.equal(c.lse, want[1])


@pytest.mark.parametrize("new,kv,hq,d", [([40], [200000], 1, 64), ([40], [100000], 1, 128), ([260], [200000], 1, 128), ([40, 1], [100000, 300], 1, 64), ([900], [80000], 8, 64),
                                         ([33], [30000], 1, 64)])
@pytest.mark.parametrize("dtype", [P.BF16, P.FP16])
def test_many_rows_whose_parts_are_added_up_in_several_levels(new, kv, hq, d, dtype):
    """241, 224, 51, 121, 8 and 118 parts of a unit on a chip of 256 units, four at a time: two to four levels."""
    check(Case(new, kv, dtype=dtype, hq=hq, hkv=1, d=d, page=48, clean=True, seed=18).run())


def test_many_rows_replayed_between_divisions():
    c = Case([60, 40], [100000, 40000], hq=2, hkv=1, d=64, page=64, clean=True, seed=19)
    lengths = [[100000, 40000], [60, 40000], [100000, 40], [300, 200], [4000, 90], [59, 0], [100000, 39999]]
    want = []
    for kv in lengths:
        c.kv_len.copy_(torch.tensor(kv, dtype=torch.int32))
        c.reset()
        c.run()
        want.append((c.out.clone(), c.lse.clone()))
    torch.cuda.synchronize()
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


def test_one_workspace_for_calls_of_both_kinds():
    """Few rows, many rows and few again, in one captured step, with counters that nobody clears."""
    few = Case([1, 2], [30000, 4000], hq=8, hkv=2, d=64, page=64, clean=True, seed=20)
    many = Case([300, 40], [30000, 4000], hq=8, hkv=2, d=64, page=64, clean=True, seed=21)
    want = []
    for c in (few, many):
        c.run()
        want.append((c.out.clone(), c.lse.clone()))
    ws = few.ws if few.ws.numel() > many.ws.numel() else many.ws
    few.ws = many.ws = ws.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for c in (few, many, few):
            c.run()
    for _ in range(3):
        for c in (few, many):      # (the captured calls' own tensors)
            c.out.fill_(3.0)
            c.lse.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        for c, (out, lse) in zip((few, many), want):
            assert torch.equal(c.out, out) and torch.equal(c.lse, lse)
        assert (ws[:P.WORKSPACE_HEAD] == 0).all()


@pytest.mark.parametrize("dtype", [P.BF16, P.FP16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,hq", [([1], 4), ([100], 1), ([300], 8)])
def test_infinite_values_of_keys_with_hardly_any_weight(new, hq, d, dtype):
    """2^-40 of the largest, nothing in half: the result is infinite all the same."""
    kv = [new[0] + 400]
    c = Case(new, kv, dtype=dtype, hq=hq, hkv=1, d=d, page=32, clean=True, seed=22)
    c.q.fill_(1.0)
    place = lambda key: (int(c.table_np[0, key // c.page]), slice(None), key % c.page)
    for key in range(kv[0]):
        c.k_cache[place(key)] = 28.0 / (d * c.scale) if key == 1 else 0.0
    c.run()
    want = c.out.clone(), c.lse.clone()
    for key, col, x in ((5, 5, "inf"), (9, 33, "-inf"), (13, 40, "nan")):   # (the same tile, so that the largest counts)
        c.v_cache[(*place(key), col)] = float(x)
    c.reset()
    c.run()
    assert (c.out[..., 5] == float("inf")).all() and (c.out[..., 33] == float("-inf")).all() and torch.isnan(c.out[..., 40]).all()
    for col in (5, 33, 40):
        c.out[..., col] = want[0][..., col]
    assert torch.equal(c.out, want[0]) and torch.equal(c.lse, want[1])


@pytest.mark.parametrize("dtype", [P.BF16, P.FP16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [2, 200])
def test_values_that_are_none_of_them_finite(new, d, dtype):
    """All NaN; all infinite, of one sign in even columns and of both in odd ones."""
    c = Case([new], [3000], dtype=dtype, hq=4, hkv=1, d=d, page=32, clean=True, seed=23).run()
    lse = c.lse.clone()
    for what in ("nan", "inf"):
        c.v_cache.fill_(float(what))
        if what == "inf":
            c.v_cache[:, :, ::2, 1::2] = float("-inf")
        c.reset()
        c.run()
        assert torch.isnan(c.out[..., 1::2]).all() and torch.equal(c.lse, lse)
        assert torch.isnan(c.out[..., ::2]).all() if what == "nan" else (c.out[..., ::2] == float("inf")).all()
