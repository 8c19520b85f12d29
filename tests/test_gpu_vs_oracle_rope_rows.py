"""Norm and rotation on the GPU where a group of lanes has many rows, and where a row's numbers are at the ends of their range.
Bounds as in the tests of single rows (test_gpu_vs_oracle_rope)."""
import numpy as np
import pytest
import torch

import paper_2406_18485_amd as P
from gpu_harness import DEV
from oracle import rope_oracle as ro
from test_gpu_vs_oracle_rope import E, TORCH, U, Case, f64

pytestmark = pytest.mark.gpu


def rows_per_unit(c):
    """Rows of lane groups (tokens of a workgroup x heads) for every unit of the chip."""
    lanes = 1 << (c.d // (8 if c.dtype == P.FP32 else 16) - 1).bit_length()
    blocks = -(-c.b * c.n // (256 // lanes))
    return blocks * (c.hq + c.hkv) / torch.cuda.get_device_properties(0).multi_processor_count


# heads that a group's share does not divide, of which it has some of q and some of k; a last block of few tokens
MANY = [(P.BF16, 3, 2333, 9, 3, 128, 128, False), (P.FP16, 2, 3499, 11, 2, 128, 64, True), (P.FP32, 2, 1501, 9, 3, 128, 128, False),
        (P.FP32, 1, 1301, 16, 1, 256, 32, True), (P.BF16, 1, 12001, 13, 5, 64, 64, True)]


@pytest.mark.parametrize("dtype,b,n,hq,hkv,d,rot,inter", MANY)
def test_groups_of_many_heads_and_blocks(dtype, b, n, hq, hkv, d, rot, inter):
    c = Case(dtype, b, n, hq, hkv, d, rot, inter=inter, layout="tokens", where="given", seed=n)
    assert rows_per_unit(c) > 4    # more than a row for every group, forward (4 a unit) and backward (3)
    c.fwd()
    c.bwd()
    c.check_fwd()
    c.check_bwd()
    first = [x.clone() for x in (c.dq, c.dk, c.dwq, c.dwk)]
    c.ws.fill_(0x7F)
    c.bwd()
    assert all(torch.equal(a, x) for a, x in zip(first, (c.dq, c.dk, c.dwq, c.dwk)))   # bit-reproducible


@pytest.mark.parametrize("dtype", [P.BF16, P.FP32])
def test_groups_of_many_heads_in_place(dtype):
    c = Case(dtype, 2, 3499, 9, 3, 128, 128, layout="heads", seed=1)
    assert rows_per_unit(c) > 4
    c.fwd()
    q, k = c.q.clone(), c.k.clone()
    P.qk_rope_fwd(c.desc, q, k, c.wq, c.wk, c.f, None, q, k)
    assert torch.equal(q, c.q_out) and torch.equal(k, c.k_out)
    # gradients over the forward's inputs
    c.bwd()
    want = c.dq.clone(), c.dk.clone(), c.dwq.clone(), c.dwk.clone()
    P.qk_rope_bwd(c.desc, c.q, c.k, c.wq, c.wk, c.f, None, c.dqo, c.dko, c.q, c.k, c.dwq, c.dwk, c.ws)
    assert all(torch.equal(a, x) for a, x in zip(want, (c.q, c.k, c.dwq, c.dwk)))


def test_a_group_with_rows_of_one_side_alone():
    for hq, hkv in ((11, 0), (0, 11)):
        c = Case(P.BF16, 3, 2333, hq, hkv, 128, 128, seed=2)
        assert rows_per_unit(c) > 4
        if hq == 0:
            c.q = c.q_out = c.dqo = c.dq = c.dwq = None
        else:
            c.k = c.k_out = c.dko = c.dk = c.dwk = None
        c.fwd()
        c.bwd()
        c.check_fwd()
        c.check_bwd()


@pytest.mark.parametrize("dtype", [P.BF16, P.FP16, P.FP32])
@pytest.mark.parametrize("d,rot", [(64, 32), (128, 0), (80, 48), (16, 0)])
@pytest.mark.parametrize("inter", [False, True])
def test_infinities_and_nan_in_elements_that_are_not_rotated(dtype, d, rot, inter):
    """They pass as they are, and so do their neighbours."""
    c = Case(dtype, 1, 9, 3, 1, d, rot, norm=False, inter=inter, seed=3)
    odd = [(0, rot, float("inf")), (1, d - 1, float("-inf")), (2, rot + 3, float("nan"))]
    for i, at, x in odd:
        c.q[0, :, i, at] = x
        c.dqo[0, :, i, at] = x
    c.fwd()
    c.bwd()
    assert torch.equal(c.q_out[..., rot:].nan_to_num(nan=77.0), c.q[..., rot:].nan_to_num(nan=77.0))
    assert torch.equal(c.dq[..., rot:].nan_to_num(nan=77.0), c.dqo[..., rot:].to(TORCH[dtype]).nan_to_num(nan=77.0))
    for i, at, x in odd:
        c.q[0, :, i, at] = 0
        c.dqo[0, :, i, at] = 0
    want = c.q_out.clone(), c.dq.clone()
    c.fwd()
    c.bwd()
    assert torch.equal(c.q_out[..., :rot], want[0][..., :rot]) and torch.equal(c.dq[..., :rot], want[1][..., :rot])


@pytest.mark.parametrize("dtype", [P.BF16, P.FP32])
@pytest.mark.parametrize("size", [1e-14, 3e-16])
def test_gradient_of_small_rows_without_eps(dtype, size):
    """The norm's factor is some 1e14 and 1e15, its cube past the largest float; the gradient itself is not."""
    c = Case(dtype, 1, 40, 3, 2, 64, 64, seed=4)
    c.q.mul_(size)
    c.k.mul_(size)
    c.desc.eps = 0.0
    c.fwd()
    c.bwd()
    for x, w, y, g, dx, dw in ((c.q, c.wq, c.q_out, c.dqo, c.dq, c.dwq), (c.k, c.wk, c.k_out, c.dko, c.dk, c.dwk)):
        want, want_dw = ro.rope_backward(f64(x), f64(w), 0.0, c.pos[:, None], f64(c.f), f64(g), False, True)
        gabs = c.pair_sum(np.abs(f64(g)))
        r = 1 / np.sqrt((f64(x) ** 2).mean(-1, keepdims=True))
        hat, habs = np.abs(f64(x)) * r, gabs * np.abs(f64(w))
        off = 64 * E * r * (habs + hat * (habs * hat).mean(-1, keepdims=True))
        assert (np.abs(f64(dx) - want) <= off + U[dtype][0] * (np.abs(want) + off)).all()
        assert (np.abs(f64(dw) - want_dw) <= (x.shape[1] * 40 + 64) * E * (gabs * hat).reshape(-1, 64).sum(0)).all()
        out = ro.rope_forward(f64(x), f64(w), 0.0, c.pos[:, None], f64(c.f), False, True)
        off = 32 * E * c.pair_sum(np.abs(f64(w)) * hat)
        assert (np.abs(f64(y) - out) <= off + U[dtype][0] * (np.abs(out) + off)).all()


def test_sine_and_cosine_in_32_bits():
    """Of rows whose pairs are (1, 0), which come out as the cosine and the sine themselves.  They carry their own rounding, E / 2 of at most 1,
    and that of the last operation, E / 2, and E at the most for the reduced angle and the series between them."""
    n = 20000
    pos = torch.randint(-2_000_000, 2_000_000, (1, n), generator=torch.Generator().manual_seed(5), dtype=torch.int32)
    q = torch.zeros(1, 1, n, 128, device=DEV)
    q[..., :64] = 1
    f = (10000.0 ** (-torch.arange(0, 128, 2, dtype=torch.float64) / 128)).float()
    out = torch.empty_like(q)
    desc = P.make_rope_desc(batch=1, n_q_heads=1, n_kv_heads=0, head_dim=128, len=n, dtype=P.FP32)
    P.qk_rope_fwd(desc, q, None, None, None, f.to(DEV), pos.to(DEV), out, None)
    angle = pos[0].double()[:, None] * f.double()
    off = (out[0, 0].double().cpu() - torch.cat((angle.cos(), angle.sin()), -1)).abs()
    assert off.max() <= 2 * E, off.max() / E
