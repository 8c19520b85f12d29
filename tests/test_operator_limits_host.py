"""Descriptors at the ends of their ranges: what the calls around the step refuse, before anything is launched or read."""
import subprocess
import sys

import pytest

import paper_2406_18485_amd as P
from test_paged_host import _append, _attn
from test_rope_host import _bwd, _fwd, _refused

PTR = 0x1000
TINY = (16, 16, 16)


def rope(hq, hkv, n):
    return P.make_rope_desc(batch=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=16, len=n, dtype=P.BF16, flags=P.QK_NORM, eps=1e-5, q_stride=TINY,
                            k_stride=TINY, q_out_stride=TINY, k_out_stride=TINY)


def paged(hq, hkv, n):
    return P.make_paged_desc(n_seqs=1, n_tokens=n, n_q_heads=hq, n_kv_heads=hkv, head_dim=64, dtype=P.BF16, n_pages=1, page_size=16, max_pages=1,
                             q_stride=(64, 64), kv_stride=(64, 64), o_stride=(64, 64), cache_stride=(64, 64, 64))


MANY = [(2 ** 31 - 1, 1), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 30, 2 ** 30), ((1 << 20) + 1, 1)]


def refuse_many_heads():
    for hq, hkv in MANY:
        for n in (0, 1, 64):
            print(hq, hkv, n, flush=True)
            r, p = rope(hq, hkv, n), paged(hq, hkv, n)
            for call in (lambda: _fwd(r), lambda: _bwd(r), lambda: P.qk_rope_workspace_bytes(r), lambda: _append(p), lambda: _attn(p),
                         lambda: P.paged_workspace_bytes(p)):
                _refused(call, P.E_UNSUPPORTED)


def test_more_heads_than_the_launches_count():
    """In a process of its own: such numbers have ended it."""
    code = f"import sys; sys.path[:0] = {sys.path!r}; import test_operator_limits_host as t; t.refuse_many_heads()"
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stdout[-200:], r.stderr[-2000:])


@pytest.mark.parametrize("i", range(3))
@pytest.mark.parametrize("stride", [0, 8])
def test_results_whose_rows_lie_on_each_other(i, stride):
    """Rows of a result that share memory would be written by several workgroups at once.  Inputs may be broadcast."""
    good = dict(batch=2, n_q_heads=4, n_kv_heads=2, head_dim=128, len=64, dtype=P.BF16)
    over = [4 * 64 * 128, 64 * 128, 128]
    over[i] = stride
    no_weights = dict(wq=None, wk=None)
    for name in ("q", "k"):
        _refused(lambda: _fwd(P.make_rope_desc(**good, **{name + "_out_stride": over}), **no_weights), P.E_SHAPE)
        _refused(lambda: _bwd(P.make_rope_desc(**good, **{name + "_stride": over}), **no_weights, dwq=None, dwk=None, ws=None), P.E_SHAPE)
    good = dict(n_seqs=3, n_tokens=20, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=P.BF16, n_pages=64, page_size=16, max_pages=32)
    over = [2 * 16 * 128, 16 * 128, 128]
    over[i] = stride
    _refused(lambda: _append(P.make_paged_desc(**good, cache_stride=over)), P.E_SHAPE)
    if i < 2:
        over = [8 * 128, 128]
        over[i] = stride
        _refused(lambda: _append(P.make_paged_desc(**good, o_stride=over)), P.E_SHAPE)
        _refused(lambda: _attn(P.make_paged_desc(**good, o_stride=over)), P.E_SHAPE)


def test_a_stride_that_is_not_used_may_be_anything():
    """Of one batch element, head, token or page; and of a call with nothing to do."""
    one = P.make_rope_desc(batch=1, n_q_heads=1, n_kv_heads=1, head_dim=128, len=0, dtype=P.BF16, q_stride=(0, 0, 0), q_out_stride=(0, 0, 0))
    _fwd(one, wq=None, wk=None)
    _bwd(one, wq=None, wk=None, dwq=None, dwk=None, ws=None)
    none = P.make_paged_desc(n_seqs=0, n_tokens=0, n_q_heads=1, n_kv_heads=1, head_dim=128, dtype=P.BF16, n_pages=1, page_size=1, max_pages=1,
                             cache_stride=(0, 0, 0), o_stride=(0, 0))
    _append(none)
    _attn(none)
