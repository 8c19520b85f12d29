"""The paged oracle against plain attention, and what the paged calls refuse before anything is launched."""
import ctypes as C

import numpy as np
import pytest
import torch

import oracle as orc
import paper_2406_18485_amd as P
from oracle import paged_oracle as po
from oracle import rope_oracle as ro


def test_oracle_over_scattered_pages_is_plain_causal_attention():
    rng = np.random.default_rng(0)
    hq, hkv, d, page, n, scale = 4, 2, 8, 3, 11, 0.4
    q, k, v = rng.standard_normal((n, hq, d)), rng.standard_normal((n, hkv, d)), rng.standard_normal((n, hkv, d))
    f = 1.0 / 100.0 ** (np.arange(0, d, 2) / d)
    table = [[5, 0, 3, 1, -1], [2, 4, 6, 7, -1]]
    kc, vc = (np.full((8, hkv, page, d), np.nan) for _ in range(2))
    # twice the same tokens, in one go and in two
    kc, vc = po.append(kc, vc, np.concatenate([k, k[:4]]), np.concatenate([v, v[:4]]), None, 0, None, f, False, False, [0, n, n + 4], [n, 4], table)
    kc, vc = po.append(kc, vc, k[4:], v[4:], None, 0, None, f, False, False, [0, 0, n - 4], [n, n], table)
    assert np.isnan(kc[1, :, 2:]).all() and not np.isnan(kc[1, :, :2]).any()
    out, lse = po.attention(np.concatenate([q, q[5:]]), kc, vc, scale, True, [0, n, 2 * n - 5], [n, n], table)
    keys = np.stack([ro.rope_forward(k[j], None, 0, j, f, norm=False) for j in range(n)], 1)
    want, want_lse = orc.attention_forward(q.transpose(1, 0, 2), keys, v.transpose(1, 0, 2), np.arange(n), np.arange(n), scale)
    assert np.allclose(out[:n], want.transpose(1, 0, 2)) and np.allclose(lse[:n], want_lse.T)
    assert np.array_equal(out[n:], out[5:n]) and np.array_equal(lse[n:], lse[5:n])


PTR = 0x1000
GOOD = dict(n_seqs=3, n_tokens=20, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=P.BF16, n_pages=64, page_size=16, max_pages=32)


def _desc(**kw):
    return P.make_paged_desc(**{**GOOD, **kw})


def _append(d, **kw):
    a = dict(q=PTR, k=PTR, v=PTR, q_weight=None, k_weight=None, inv_freq=PTR, positions=None, seq_start=PTR, kv_len=PTR, page_table=PTR,
             q_out=PTR, k_cache=PTR, v_cache=PTR)
    a.update(kw)
    P.paged_append(d, **a, stream=0)


def _attn(d, **kw):
    a = dict(q=PTR, k_cache=PTR, v_cache=PTR, seq_start=PTR, kv_len=PTR, page_table=PTR, out=PTR, o=PTR, lse=PTR, workspace=PTR,
             workspace_bytes=1 << 40)
    a.update(kw)
    P.paged_attn(d, **a, stream=0)


def _refused(call, code):
    with pytest.raises(P.LoongError) as e:
        call()
    assert e.value.code == code and P.last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=9), P.E_DTYPE), (dict(dtype=P.FP32), P.E_UNSUPPORTED), (dict(n_seqs=-1), P.E_SHAPE), (dict(n_tokens=-1), P.E_SHAPE),
    (dict(max_new=-1), P.E_SHAPE), (dict(n_q_heads=0), P.E_SHAPE), (dict(n_kv_heads=0), P.E_SHAPE), (dict(n_kv_heads=3), P.E_UNSUPPORTED),
    (dict(head_dim=96), P.E_UNSUPPORTED), (dict(page_size=0), P.E_SHAPE), (dict(page_size=(1 << 24) + 1), P.E_UNSUPPORTED),
    (dict(n_pages=-1), P.E_SHAPE), (dict(max_pages=-1), P.E_SHAPE), (dict(flags=2), P.E_UNSUPPORTED), (dict(n_tokens=1 << 28), P.E_UNSUPPORTED),
    (dict(n_seqs=(1 << 20) + 1), P.E_UNSUPPORTED), (dict(max_pages=1 << 27), P.E_UNSUPPORTED),
    (dict(cache_stride=(4096, 2048, 1 << 31)), P.E_UNSUPPORTED), (dict(q_stride=(1024, 132)), P.E_ALIGN), (dict(kv_stride=(-8, 128)), P.E_SHAPE),
    (dict(cache_stride=(4096, 2048, 4)), P.E_ALIGN), (dict(o_stride=(1 << 41, 128)), P.E_SHAPE), (dict(table_stride=-1), P.E_SHAPE)])
def test_descriptors_that_are_refused(kw, code):
    d = _desc(**kw)
    _refused(lambda: _append(d), code)
    _refused(lambda: _attn(d), code)
    _refused(lambda: P.paged_workspace_bytes(d), code)


@pytest.mark.parametrize("kw,code", [
    (dict(rot_dim=136), P.E_UNSUPPORTED), (dict(rot_dim=8), P.E_UNSUPPORTED), (dict(flags=P.QK_NORM, eps=-1.0), P.E_SHAPE),
    (dict(flags=P.QK_NORM, eps=float("inf")), P.E_SHAPE), (dict(flags=P.WORKSPACE_CLEAN), P.E_UNSUPPORTED)])
def test_append_descriptors_that_are_refused(kw, code):
    _refused(lambda: _append(_desc(**kw)), code)


@pytest.mark.parametrize("kw,code", [
    (dict(softmax_scale=0.0), P.E_SHAPE), (dict(softmax_scale=float("nan")), P.E_SHAPE), (dict(flags=P.QK_NORM), P.E_UNSUPPORTED),
    (dict(n_pages=0), P.E_SHAPE)])
def test_attention_descriptors_that_are_refused(kw, code):
    _refused(lambda: _attn(_desc(**kw)), code)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), P.E_NULL), (dict(q_out=None), P.E_NULL), (dict(v=None), P.E_NULL), (dict(inv_freq=None), P.E_NULL),
    (dict(page_table=None), P.E_NULL), (dict(k_cache=PTR + 8), P.E_ALIGN), (dict(k_weight=PTR + 4), P.E_ALIGN), (dict(kv_len=PTR + 2), P.E_ALIGN)])
def test_append_arguments_that_are_refused(kw, code):
    _refused(lambda: _append(_desc(), **kw), code)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), P.E_NULL), (dict(lse=None), P.E_NULL), (dict(out=None, o=None), P.E_NULL), (dict(seq_start=None), P.E_NULL),
    (dict(o=PTR + 8), P.E_ALIGN), (dict(workspace=PTR + 8), P.E_ALIGN), (dict(lse=PTR + 2), P.E_ALIGN)])
def test_attention_arguments_that_are_refused(kw, code):
    _refused(lambda: _attn(_desc(), **kw), code)


def test_nothing_to_do_is_no_error():
    for kw in (dict(n_seqs=0), dict(n_tokens=0)):
        _append(_desc(**kw))
        _attn(_desc(**kw))
    _attn(_desc(max_new=0))


def test_workspace_only_where_a_context_can_be_shared():
    assert P.paged_workspace_bytes(_desc(max_new=1, max_pages=16)) == 0            # 256 keys: one span
    few, many = P.paged_workspace_bytes(_desc(max_new=1, max_pages=4096)), P.paged_workspace_bytes(_desc(n_tokens=4000, max_pages=4096))
    assert P.WORKSPACE_HEAD < few < many < 1 << 28
    assert C.sizeof(P.binding.PagedDesc) == 15 * 4 + 4 + 8 * (1 + 6 + 3)


def test_tensors_that_no_kernel_may_read_are_refused():
    with pytest.raises(ValueError, match="page_table is on cpu"):
        _attn(_desc(), page_table=torch.zeros(3, 32, dtype=torch.int32))


@pytest.mark.parametrize("name,x,text", [
    ("seq_start", torch.zeros(3, dtype=torch.int32), "4 are read"), ("kv_len", torch.zeros(6, dtype=torch.int32)[::2], "not contiguous"),
    ("page_table", torch.zeros(2, 32, dtype=torch.int32), "3 rows of 32 are read"),
    ("page_table", torch.zeros(3, 40, dtype=torch.int32), "strides"), ("lse", torch.zeros(20, 7), "160 are read")])
def test_tables_that_are_too_short_are_refused(name, x, text):
    with pytest.raises(ValueError, match=text):
        _attn(_desc(), **{name: x})
