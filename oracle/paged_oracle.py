"""A paged cache and attention over it, in fp64 numpy: sequence by sequence, slot by slot."""
from __future__ import annotations

import numpy as np

from .ring_attention_oracle import attention_forward
from .rope_oracle import rope_forward


def slots_of(seq: int, n_keys: int, page_table, page_size: int):
    """(page, slot) of a sequence's keys 0 .. n_keys - 1."""
    return [(int(page_table[seq][j // page_size]), j % page_size) for j in range(n_keys)]


def append(k_cache, v_cache, k, v, weight, eps, positions, inv_freq, interleaved, norm, seq_start, kv_len, page_table):
    """Copies of the caches [page, kv head, slot, d] with the new tokens [token, kv head, d] in their slots.
    positions: of every token, or None: the slot's number."""
    kc, vc = np.array(k_cache, np.float64), np.array(v_cache, np.float64)
    for b in range(len(kv_len)):
        n = seq_start[b + 1] - seq_start[b]
        where = slots_of(b, kv_len[b], page_table, kc.shape[2])
        for i in range(n):
            t, j = seq_start[b] + i, kv_len[b] - n + i
            if j < 0:
                continue
            page, slot = where[j]
            pos = j if positions is None else positions[t]
            kc[page, :, slot] = rope_forward(k[t], weight, eps, pos, inv_freq, interleaved, norm)
            vc[page, :, slot] = v[t]
    return kc, vc


def attention(q, k_cache, v_cache, scale, causal, seq_start, kv_len, page_table):
    """(out [token, q head, d], lse [token, q head]); rows of no sequence are NaN."""
    out = np.full(q.shape, np.nan)
    lse = np.full(q.shape[:2], np.nan)
    for b in range(len(kv_len)):
        lo, hi = seq_start[b], seq_start[b + 1]
        if hi == lo:
            continue
        where = slots_of(b, kv_len[b], page_table, k_cache.shape[2])
        pages, slots = (np.array([w[i] for w in where], int) for i in (0, 1))
        keys = np.asarray(k_cache, np.float64)[pages, :, slots].transpose(1, 0, 2)
        vals = np.asarray(v_cache, np.float64)[pages, :, slots].transpose(1, 0, 2)
        pos_k = np.arange(kv_len[b])
        pos_q = np.arange(kv_len[b] - (hi - lo), kv_len[b])
        rows = np.asarray(q, np.float64)[lo:hi].transpose(1, 0, 2)
        o, s = attention_forward(rows, keys, vals, pos_q, pos_k, scale, causal)
        out[lo:hi], lse[lo:hi] = o.transpose(1, 0, 2), s.T
    return out, lse
