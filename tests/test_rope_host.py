"""The norm-and-rotation oracle against what it is defined by, and what the calls refuse before anything is launched."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2406_18485_amd as P
from oracle import rope_oracle as ro

FREQ = 1.0 / 10000.0 ** (np.arange(0, 8, 2) / 8.0)


@pytest.mark.parametrize("interleaved", [False, True])
def test_forward_is_the_rotation_matrix_on_the_normed_row(interleaved):
    rng = np.random.default_rng(0)
    x, w = rng.standard_normal((3, 12)), rng.standard_normal(12)
    pos = np.array([0, 5, 1 << 20])
    y = ro.rope_forward(x, w, 1e-3, pos, FREQ, interleaved)
    for r in range(3):
        n = w * x[r] / np.sqrt(sum(v * v for v in x[r]) / 12 + 1e-3)
        assert np.allclose(y[r], ro.rotation_matrix(pos[r], FREQ, 12, interleaved) @ n, atol=1e-12)
    assert np.allclose(y[0], w * x[0] / np.sqrt((x[0] ** 2).mean() + 1e-3))   # position 0 is not turned


def test_scores_depend_on_the_distance_alone_and_the_rest_passes():
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 12))
    turn = lambda x, p: ro.rope_forward(x[None], None, 0, np.array([p]), FREQ, norm=False)[0]
    assert np.isclose(turn(q, 107) @ turn(k, 100), turn(q, 7) @ turn(k, 0), atol=1e-12)
    assert np.array_equal(turn(q, 99)[8:], q[8:])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_backward_against_differences_and_autograd(norm, interleaved):
    rng = np.random.default_rng(2)
    x, w, g = rng.standard_normal((4, 12)), rng.standard_normal(12), rng.standard_normal((4, 12))
    pos = np.array([3, 0, 77, 12345])
    loss = lambda x, w: (g * ro.rope_forward(x, w, 1e-2, pos, FREQ, interleaved, norm)).sum()
    dx, dw = ro.rope_backward(x, w, 1e-2, pos, FREQ, g, interleaved, norm)
    h = 1e-5
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = h
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * h) - dx[i]) < 1e-8
    if not norm:
        assert dw is None
        return
    for i in range(12):
        e = np.zeros(12)
        e[i] = h
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * h) - dw[i]) < 1e-8
    xt, wt = torch.tensor(x, requires_grad=True), torch.tensor(w, requires_grad=True)
    n = xt * torch.rsqrt((xt * xt).mean(-1, keepdim=True) + 1e-2) * wt
    m = torch.tensor(np.stack([ro.rotation_matrix(p, FREQ, 12, interleaved) for p in pos]))
    (torch.matmul(m, n[..., None])[..., 0] * torch.tensor(g)).sum().backward()
    assert np.allclose(xt.grad.numpy(), dx, atol=1e-10) and np.allclose(wt.grad.numpy(), dw, atol=1e-10)


# ---- what is refused.  The pointers are never read: every call fails before a launch
GOOD = dict(batch=2, n_q_heads=4, n_kv_heads=2, head_dim=128, len=64, dtype=P.BF16, flags=P.QK_NORM, eps=1e-5)
PTR = 0x1000


def _desc(**kw):
    return P.make_rope_desc(**{**GOOD, **kw})


def _fwd(d, q=PTR, k=PTR, wq=PTR, wk=PTR, f=PTR, pos=None, qo=PTR, ko=PTR):
    P.qk_rope_fwd(d, q, k, wq, wk, f, pos, qo, ko, stream=0)


def _bwd(d, q=PTR, k=PTR, wq=PTR, wk=PTR, f=PTR, pos=None, dqo=PTR, dko=PTR, dq=PTR, dk=PTR, dwq=PTR, dwk=PTR, ws=PTR, n=1 << 30):
    P.qk_rope_bwd(d, q, k, wq, wk, f, pos, dqo, dko, dq, dk, dwq, dwk, ws, n, stream=0)


def _refused(call, code):
    with pytest.raises(P.LoongError) as e:
        call()
    assert e.value.code == code and P.last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=7), P.E_DTYPE), (dict(batch=-1), P.E_SHAPE), (dict(len=-1), P.E_SHAPE), (dict(n_q_heads=0, n_kv_heads=0), P.E_SHAPE),
    (dict(n_q_heads=-2), P.E_SHAPE), (dict(head_dim=72), P.E_UNSUPPORTED), (dict(head_dim=272), P.E_UNSUPPORTED),
    (dict(head_dim=0), P.E_UNSUPPORTED), (dict(rot_dim=24), P.E_UNSUPPORTED), (dict(rot_dim=144), P.E_UNSUPPORTED),
    (dict(rot_dim=-16), P.E_UNSUPPORTED), (dict(flags=1), P.E_UNSUPPORTED), (dict(eps=-1.0), P.E_SHAPE), (dict(eps=float("nan")), P.E_SHAPE),
    (dict(chunk_len=31), P.E_SHAPE), (dict(chunk_len=-32), P.E_SHAPE), (dict(chunk_len=32, chunk=(-1, 2)), P.E_SHAPE),
    (dict(q_stride=(-8, 128, 128)), P.E_SHAPE), (dict(k_stride=(128, 132, 128)), P.E_ALIGN), (dict(q_out_stride=(128, 128, 4)), P.E_ALIGN),
    (dict(batch=1 << 16, len=1 << 16), P.E_UNSUPPORTED),
])
def test_descriptors_that_are_refused(kw, code):
    d = _desc(**kw)
    _refused(lambda: _fwd(d), code)
    _refused(lambda: _bwd(d), code)
    _refused(lambda: P.qk_rope_workspace_bytes(d), code)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), P.E_NULL), (dict(ko=None), P.E_NULL), (dict(f=None), P.E_NULL), (dict(k=PTR + 8), P.E_ALIGN), (dict(qo=PTR + 2), P.E_ALIGN),
    (dict(wq=PTR + 4), P.E_ALIGN), (dict(pos=PTR + 2), P.E_ALIGN)])
def test_forward_arguments_that_are_refused(kw, code):
    _refused(lambda: _fwd(_desc(), **kw), code)


@pytest.mark.parametrize("kw,code", [
    (dict(dqo=None), P.E_NULL), (dict(dk=None), P.E_NULL), (dict(ws=None), P.E_NULL), (dict(ws=PTR + 8), P.E_ALIGN), (dict(n=16), P.E_SHAPE),
    (dict(dq=PTR + 8), P.E_ALIGN), (dict(dwk=PTR + 1), P.E_ALIGN)])
def test_backward_arguments_that_are_refused(kw, code):
    _refused(lambda: _bwd(_desc(), **kw), code)


def test_weight_gradients_need_the_norm_and_the_heads():
    _refused(lambda: _bwd(_desc(flags=0)), P.E_UNSUPPORTED)
    _refused(lambda: _bwd(_desc(n_kv_heads=0)), P.E_UNSUPPORTED)
    assert P.qk_rope_workspace_bytes(_desc(flags=0)) == 0
    assert P.qk_rope_workspace_bytes(_desc()) > 0


def test_tensors_that_no_kernel_may_read_are_refused():
    x = torch.zeros(2, 4, 64, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="q is on cpu"):
        _fwd(_desc(), q=x)


@pytest.mark.parametrize("kw,text", [
    (dict(wq=torch.ones(64)), "128 are read"), (dict(f=torch.ones(63)), "64 are read"), (dict(pos=torch.zeros(2, 63, dtype=torch.int32)), "128 are read"),
    (dict(pos=torch.zeros(64, 2, dtype=torch.int32).T), "not contiguous")])
def test_weights_and_positions_that_are_too_short_are_refused(kw, text):
    with pytest.raises(ValueError, match=text):
        _fwd(_desc(), **kw)
    with pytest.raises(ValueError, match=text):
        _bwd(_desc(), **kw)


def test_nothing_to_do_is_no_error():
    _fwd(_desc(len=0))
    _fwd(_desc(batch=0))
    _fwd(_desc(n_kv_heads=0, len=0), k=None, ko=None, wk=None)
    assert C.sizeof(P.binding.RopeDesc) == 12 * 4 + 12 * 8
