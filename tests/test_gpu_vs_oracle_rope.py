"""Norm and rotation on the GPU against the fp64 oracle on the same bits.

Bounds, fixed before the first run.  u is half a step of the storage type relative to the value (2^-8 bf16, 2^-11 half with
2^-25 below its normal numbers, 2^-24 fp32), E = 2^-24.  Forward: an output is c n_a - s n_b; the norm's factor carries the rounding of some
25 sums and a reciprocal root, the cosine and sine one of 2 pi 2^-25 for the reduced angle and two of their own, then three
operations: below 32 E (|n_a| + |n_b|) together, and the storage type's rounding.  Backward: dx = r (h - hat mean(h hat)): the same for g, and
some 25 sums of the mean: below 64 E r (|h_a| + |h_b| + |hat| mean|h hat|).  A weight's gradient: at most `rows` sums of terms that carry
32 E: below (rows + 64) E sum|g||hat|."""
import numpy as np
import pytest
import torch

import oracle as orc
import paper_2406_18485_amd as P
from gpu_harness import DEV
from oracle import rope_oracle as ro
from paper_2406_18485_amd.ring import RingReplay, RingShape

pytestmark = pytest.mark.gpu

TORCH = {P.BF16: torch.bfloat16, P.FP16: torch.float16, P.FP32: torch.float32}
U = {P.BF16: (2.0 ** -8, 0.0), P.FP16: (2.0 ** -11, 2.0 ** -25), P.FP32: (2.0 ** -24, 0.0)}
E = 2.0 ** -24
EPS = 1e-5


def freqs(rot):
    return (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float().to(DEV)


def f64(x):
    return x.detach().double().cpu().numpy()


def draw(gen, shape, dtype):
    return torch.randn(shape, generator=gen).to(TORCH[dtype]).to(DEV)


class Case:
    """One set of inputs; `layout`: "heads" [b,h,n,d], "tokens" [b,n,h,d] in one packed projection, "gaps" with NaN between rows."""

    def __init__(self, dtype, b, n, hq, hkv, d, rot, norm=True, inter=False, layout="heads", where="plain", weights=True, seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.__dict__.update(dtype=dtype, b=b, n=n, hq=hq, hkv=hkv, d=d, rot=rot, norm=norm, inter=inter)
        if layout == "tokens":
            x = draw(gen, (b, n, hq + 2 * hkv, d), dtype).transpose(1, 2)
            self.q, self.k = x[:, :hq], x[:, hq:hq + hkv]
        elif layout == "gaps":
            def gaps(h):
                x = torch.full((b, n, h, d + 16), float("nan"), dtype=TORCH[dtype], device=DEV)
                x[..., :d] = draw(gen, (b, n, h, d), dtype)
                return x[..., :d].transpose(1, 2)
            self.q, self.k = gaps(hq), gaps(hkv)
        else:
            self.q, self.k = draw(gen, (b, hq, n, d), dtype), draw(gen, (b, hkv, n, d), dtype)
        self.wq, self.wk = (1 + 0.3 * torch.randn(d, generator=gen).to(DEV) if norm and weights else None for _ in range(2))
        self.f = freqs(rot)
        self.positions, chunk = None, {}
        if where == "plain":
            self.pos = np.broadcast_to(np.arange(n), (b, n))
        elif where == "zigzag":
            cp, rank = 32, 5
            self.pos = np.broadcast_to(orc.zigzag_positions(cp, rank, n // 2), (b, n))
            chunk = dict(chunk_len=n // 2, chunk=(rank, 2 * cp - 1 - rank))
        else:   # given, in no order, some negative, up to two million
            self.pos = np.random.default_rng(seed).integers(-100, 2_000_000, (b, n))
            self.positions = torch.tensor(self.pos, dtype=torch.int32, device=DEV)
        self.q_out, self.k_out = (torch.full((b, h, n, d), float("nan"), dtype=TORCH[dtype], device=DEV) for h in (hq, hkv))
        self.dqo, self.dko = (torch.randn(b, h, n, d, generator=gen).to(DEV) for h in (hq, hkv))
        self.dq, self.dk = (self.like(x) for x in (self.q, self.k))
        self.dwq, self.dwk = (torch.full((d,), 7.0, device=DEV) if norm else None for _ in range(2))
        self.desc = P.make_rope_desc(batch=b, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, rot_dim=rot, len=n, dtype=dtype, eps=EPS,
                                     flags=(P.QK_NORM if norm else 0) | (P.ROPE_INTERLEAVED if inter else 0),
                                     q_stride=self.q.stride()[:3], k_stride=self.k.stride()[:3], **chunk)
        self.ws = torch.full((max(P.qk_rope_workspace_bytes(self.desc), 16),), 0xFF, dtype=torch.uint8, device=DEV)

    @staticmethod
    def like(x):
        """Memory of its own in x's shape and strides (a gradient has its tensor's)."""
        span = 1 + sum(max(s - 1, 0) * st for s, st in zip(x.shape, x.stride()))
        return torch.full((span,), 7.0, dtype=x.dtype, device=DEV).as_strided(x.shape, x.stride())

    def fwd(self, **kw):
        P.qk_rope_fwd(self.desc, self.q, self.k, self.wq, self.wk, self.f, self.positions, self.q_out, self.k_out, **kw)

    def bwd(self, **kw):
        P.qk_rope_bwd(self.desc, self.q, self.k, self.wq, self.wk, self.f, self.positions, self.dqo, self.dko, self.dq, self.dk,
                      self.dwq, self.dwk, self.ws, **kw)

    def check_fwd(self):
        for x, w, y, h in ((self.q, self.wq, self.q_out, self.hq), (self.k, self.wk, self.k_out, self.hkv)):
            if h == 0:
                continue
            pos = self.pos[:, None]
            want = ro.rope_forward(f64(x), None if w is None else f64(w), EPS, pos, f64(self.f), self.inter, self.norm)
            size = self.pair_sum(np.abs(ro.rope_forward(f64(x), None if w is None else f64(w), EPS, 0 * pos, f64(self.f), self.inter, self.norm)))
            self.close(f64(y), want, 32 * E * size, "forward")

    def check_bwd(self):
        for x, w, g, dx, dw, h in ((self.q, self.wq, self.dqo, self.dq, self.dwq, self.hq), (self.k, self.wk, self.dko, self.dk, self.dwk, self.hkv)):
            if h == 0:
                continue
            pos, w64 = self.pos[:, None], np.ones(self.d) if w is None else f64(w)
            want, want_dw = ro.rope_backward(f64(x), w64, EPS, pos, f64(self.f), f64(g), self.inter, self.norm)
            gabs = self.pair_sum(np.abs(f64(g)))
            if self.norm:
                r = 1 / np.sqrt((f64(x) ** 2).mean(-1, keepdims=True) + EPS)
                hat = np.abs(f64(x)) * r
                habs = gabs * np.abs(w64)
                size = r * (habs + hat * (habs * hat).mean(-1, keepdims=True))
                terms = (gabs * hat).reshape(-1, self.d).sum(0)
                rows = self.b * self.n * h
                assert (np.abs(f64(dw) - want_dw) <= (rows + 64) * E * terms).all(), np.abs(f64(dw) - want_dw).max()
            else:
                size = gabs
            self.close(f64(dx), want, 64 * E * size, "backward")

    def pair_sum(self, x):
        y = np.array(x)
        a, b = ro.pairs(self.rot, self.inter)
        y[..., a] = y[..., b] = x[..., a] + x[..., b]
        return y

    def close(self, got, want, off, what):
        u, small = U[self.dtype]
        bad = ~(np.abs(got - want) <= off + u * (np.abs(want) + off) + small)
        assert not bad.any(), (what, int(bad.sum()), bad.size, np.abs(got - want).max())


SHAPES = [  # b, n, hq, hkv, d, rot
    (1, 1, 1, 1, 64, 64), (2, 37, 4, 2, 128, 128), (3, 5, 5, 1, 128, 64), (1, 130, 9, 3, 64, 32), (2, 9, 3, 1, 80, 48), (1, 33, 2, 2, 256, 256),
    (1, 7, 1, 1, 16, 16), (2, 8, 2, 1, 96, 0), (1, 2, 70, 2, 128, 128)]


@pytest.mark.parametrize("dtype", [P.BF16, P.FP16, P.FP32])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("inter", [False, True])
def test_forward_and_backward_against_the_oracle(shape, dtype, inter):
    c = Case(dtype, *shape, inter=inter, layout="tokens", where="given", seed=sum(shape))
    c.fwd()
    c.bwd()
    c.check_fwd()
    c.check_bwd()


@pytest.mark.parametrize("norm,weights", [(False, False), (True, False), (True, True)])
@pytest.mark.parametrize("where", ["plain", "zigzag", "given"])
@pytest.mark.parametrize("layout", ["heads", "tokens", "gaps"])
def test_layouts_positions_and_the_norm(layout, where, norm, weights):
    c = Case(P.BF16, 2, 46, 6, 2, 128, 128, norm=norm, layout=layout, where=where, weights=weights, seed=3)
    c.fwd()
    c.bwd()
    c.check_fwd()
    c.check_bwd()


@pytest.mark.parametrize("hq,hkv", [(4, 0), (0, 3)])
def test_queries_or_keys_alone(hq, hkv):
    c = Case(P.FP16, 2, 21, hq, hkv, 64, 64, seed=4)
    if hq == 0:
        c.q = c.q_out = c.dqo = c.dq = c.dwq = None
    else:
        c.k = c.k_out = c.dko = c.dk = c.dwk = None
    c.fwd()
    c.bwd()
    c.check_fwd()
    c.check_bwd()


def test_many_tokens_whose_sums_are_spread_over_workgroups():
    c = Case(P.BF16, 1, 3001, 8, 8, 64, 64, layout="tokens", seed=5)
    c.fwd()
    c.bwd()
    c.check_fwd()
    c.check_bwd()
    first = [x.clone() for x in (c.dq, c.dk, c.dwq, c.dwk)]
    c.ws.fill_(0x7F)
    c.bwd()
    assert all(torch.equal(a, b) for a, b in zip(first, (c.dq, c.dk, c.dwq, c.dwk)))   # bit-reproducible


def test_in_place_and_what_lies_between_rows_stays():
    c = Case(P.BF16, 2, 46, 6, 2, 128, 128, seed=6)
    c.fwd()
    want = c.q_out.clone(), c.k_out.clone()
    q, k = c.q.clone(), c.k.clone()
    P.qk_rope_fwd(c.desc, q, k, c.wq, c.wk, c.f, None, q, k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    # into token-major memory with room between the heads
    room = torch.full((2, 46, 8, 144), 5.0, dtype=torch.bfloat16, device=DEV)
    out = room[..., :128].transpose(1, 2)
    d = P.make_rope_desc(batch=2, n_q_heads=6, n_kv_heads=2, head_dim=128, len=46, dtype=P.BF16, eps=EPS, flags=P.QK_NORM,
                         q_out_stride=out[:, :6].stride()[:3], k_out_stride=out[:, 6:].stride()[:3])
    P.qk_rope_fwd(d, c.q, c.k, c.wq, c.wk, c.f, None, out[:, :6], out[:, 6:])
    assert torch.equal(out[:, :6], want[0]) and torch.equal(out[:, 6:], want[1])
    assert (room[..., 128:] == 5.0).all()


def test_no_tokens():
    c = Case(P.BF16, 1, 8, 2, 1, 64, 64, seed=7)
    d = P.make_rope_desc(batch=1, n_q_heads=2, n_kv_heads=1, head_dim=64, len=0, dtype=P.BF16, eps=EPS, flags=P.QK_NORM)
    P.qk_rope_fwd(d, c.q, c.k, c.wq, c.wk, c.f, None, c.q_out, c.k_out)
    assert torch.isnan(c.q_out).all()
    P.qk_rope_bwd(d, c.q, c.k, c.wq, c.wk, c.f, None, c.dqo, c.dko, c.dq, c.dk, c.dwq, c.dwk, c.ws)
    assert (c.dwq == 0).all() and (c.dwk == 0).all() and (c.dq == 7).all()


def test_rows_of_zeros_infinities_and_nan_stay_in_their_row():
    c = Case(P.BF16, 1, 4, 2, 1, 64, 64, seed=8)
    c.fwd()
    want = c.q_out.clone()
    c.q[0, 0, 1] = 0.0
    c.q[0, 0, 2, 3] = float("inf")
    c.q[0, 1, 3, 3] = float("nan")
    c.fwd()
    assert (c.q_out[0, 0, 1] == 0).all()
    assert torch.isnan(c.q_out[0, 1, 3]).all()
    assert torch.equal(c.q_out[0, 0, 0], want[0, 0, 0]) and torch.equal(c.q_out[0, 1, :3], want[0, 1, :3])


def test_gradient_against_differences_of_the_kernel():
    """Directional derivative in fp32: the losses' rounding, E x 16 on every |g y| at most, over 2 h, and h^2 times a third derivative
    that rows of norm 8 keep below the gradient's own size."""
    c = Case(P.FP32, 1, 12, 2, 1, 64, 32, where="given", seed=9)
    gen = torch.Generator().manual_seed(10)
    v, h = torch.randn(c.q.shape, generator=gen).to(DEV), 2.0 ** -6

    def loss(q):
        P.qk_rope_fwd(c.desc, q, c.k, c.wq, c.wk, c.f, c.positions, c.q_out, c.k_out)
        return (c.q_out.double() * c.dqo.double()).sum().item()

    c.bwd()
    want = (c.dq.double() * v.double()).sum().item()
    got = (loss(c.q + h * v) - loss(c.q - h * v)) / (2 * h)
    noise = 16 * E * (c.q_out.double() * c.dqo.double()).abs().sum().item() / (2 * h)
    assert abs(got - want) <= noise + h * h * (c.dq.double() * v.double()).abs().sum().item(), (got, want, noise)


def test_another_stream_and_graph_replays():
    c = Case(P.BF16, 1, 700, 4, 1, 128, 128, layout="tokens", where="zigzag", seed=11)
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    outs = lambda: (c.q_out, c.k_out, c.dq, c.dk, c.dwq, c.dwk)
    want = [x.clone() for x in outs()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for x in outs():
            x.fill_(3.0)
        c.fwd()
        c.bwd()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.fwd()
        c.bwd()
    for _ in range(3):
        for x in outs():
            x.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs(), want))


def test_wrong_types_and_places_are_refused():
    c = Case(P.BF16, 1, 8, 2, 1, 64, 64, where="given", seed=12)
    with pytest.raises(TypeError, match="q is torch.float16"):
        P.qk_rope_fwd(c.desc, c.q.half(), c.k, c.wq, c.wk, c.f, c.positions, c.q_out, c.k_out)
    with pytest.raises(TypeError, match="positions is torch.int64"):
        P.qk_rope_fwd(c.desc, c.q, c.k, c.wq, c.wk, c.f, c.positions.long(), c.q_out, c.k_out)
    with pytest.raises(ValueError, match="k_out is on cpu"):
        P.qk_rope_fwd(c.desc, c.q, c.k, c.wq, c.wk, c.f, c.positions, c.q_out, c.k_out.cpu())


@pytest.mark.parametrize("rank", [0, 2])
def test_rotation_around_the_ring_against_the_oracle(rank):
    """A training step's attention from the projections on: every rank's keys normed and rotated at its zigzag positions, the ring's
    forward and backward, the gradients carried back through rotation and norm.  The ring's own bound of 2e-2 on dq, dk; through the norm
    they grow by at most r max|w| (twice, for the projection off the row): r <= 2, |w| <= 2."""
    cp, hq, hkv, d, c_len = 4, 4, 2, 64, 48
    L, S = 2 * c_len, 2 * 4 * c_len
    gen = torch.Generator().manual_seed(20)
    raw_q = draw(gen, (1, hq, S, d), P.BF16)      # the whole sequence, natural order
    raw_k, v = draw(gen, (1, hkv, S, d), P.BF16), draw(gen, (1, hkv, S, d), P.BF16)
    d_o = (0.5 * torch.randn(1, hq, S, d, generator=gen)).to(torch.bfloat16).to(DEV)
    wq, wk = (1 + 0.2 * torch.randn(d, generator=gen).to(DEV) for _ in range(2))
    f = freqs(d)
    mine = lambda x, r: x[:, :, torch.tensor(orc.zigzag_positions(cp, r, c_len), device=DEV)].contiguous()
    rep = RingReplay(RingShape(cp=cp, w=cp, rank=rank, hq=hq, hkv=hkv, d=d, c=c_len, dtype=P.BF16, scale=d ** -0.5), DEV)

    def desc(r):
        return P.make_rope_desc(batch=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, len=L, chunk_len=c_len, chunk=(r, 2 * cp - 1 - r),
                                dtype=P.BF16, eps=EPS, flags=P.QK_NORM)
    q, k = torch.empty(1, hq, L, d, dtype=torch.bfloat16, device=DEV), torch.empty(cp, 1, hkv, L, d, dtype=torch.bfloat16, device=DEV)
    other = torch.empty_like(q)
    for r in range(cp):
        P.qk_rope_fwd(desc(r), mine(raw_q, r), mine(raw_k, r), wq, wk, f, None, q if r == rank else other, k[r])
    vs = torch.stack([mine(v, r) for r in range(cp)])
    rep.forward(q, k, vs)
    rep.backward(q, k, vs, mine(d_o, rank))
    dq, dk = torch.empty_like(q), torch.empty_like(k[0])
    dwq, dwk = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    ws = torch.empty(P.qk_rope_workspace_bytes(desc(rank)), dtype=torch.uint8, device=DEV)
    P.qk_rope_bwd(desc(rank), mine(raw_q, rank), mine(raw_k, rank), wq, wk, f, None, rep.dq, rep.dk[rank], dq, dk, dwq, dwk, ws)

    # the oracle, on the rotated rows as the kernels rounded them, then on what its own gradients say
    pos = orc.zigzag_positions(cp, rank, c_len)
    keys = np.concatenate([f64(k[r])[0] for r in range(cp)], axis=1)
    kpos = np.concatenate([orc.zigzag_positions(cp, r, c_len) for r in range(cp)])
    vals = np.concatenate([f64(vs[r])[0] for r in range(cp)], axis=1)
    out, lse = orc.attention_forward(f64(q)[0], keys, vals, pos, kpos, d ** -0.5)
    assert np.abs(f64(rep.out)[0] - out).max() <= 2e-2
    gq, gk, *_ = orc.attention_backward(f64(q)[0], keys, vals, f64(mine(d_o, rank))[0], pos, kpos, d ** -0.5)
    gk = gk[:, rank * L:(rank + 1) * L]
    for raw, w, g, got, got_dw in ((raw_q, wq, gq, dq, dwq), (raw_k, wk, gk, dk, dwk)):
        x = f64(mine(raw, rank))[0]
        want, want_dw = ro.rope_backward(x, f64(w), EPS, pos[None], f64(f), g)
        assert 1 / np.sqrt((x ** 2).mean(-1)).max() >= 0.5
        assert np.abs(f64(got)[0] - want).max() <= 2 * 2 * 2 * 2e-2
        # (every row's gradient off by up to 2e-2 in random directions, sums of rows of them)
        assert np.abs(f64(got_dw) - want_dw).max() <= 2e-2 * np.abs(x).max() * np.sqrt(x.shape[0] * x.shape[1])
