"""Oracle of generating with a paged key / value cache: rotary positions with several axes, appending to the cache, attention of
one new token per sequence. TEST INFRASTRUCTURE: fp64 numpy loops written from the definitions stated with the entry points in
include/hydra_attn.h (hydra_rope_axes, hydra_kv_append, hydra_mla_kv_append, hydra_attn_decode), shares nothing with the CUDA
library.

Pins (tests/test_oracle_paged_cache.py): one axis = oracle.mla_ops.rope, equal positions on all axes too; a rotation by hand;
inverse after forward = identity and the inverse is the adjoint; a cache filled token by token = filled at once; attention over
the cache = the last row of oracle.attn_fwd on the same keys; missing pages = those keys left out.
"""
from __future__ import annotations

import numpy as np


def axis_of_pairs(axis_pairs):
    return [a for a, n in enumerate(axis_pairs) for _ in range(n)]


def rope_axes(x, positions, offset: int, axis_pairs, theta: float, inverse: bool = False) -> np.ndarray:
    """x [T, h, d], positions [axes, T]."""
    y = np.array(x, dtype=np.float64)
    dim = 2 * sum(axis_pairs)
    for i, axis in enumerate(axis_of_pairs(axis_pairs)):
        for t in range(y.shape[0]):
            angle = float(positions[axis][t]) * float(theta) ** (-2.0 * i / dim) * (-1.0 if inverse else 1.0)
            a, b = y[t, :, offset + 2 * i].copy(), y[t, :, offset + 2 * i + 1].copy()
            y[t, :, offset + 2 * i] = a * np.cos(angle) - b * np.sin(angle)
            y[t, :, offset + 2 * i + 1] = a * np.sin(angle) + b * np.cos(angle)
    return y


def place(page_table, seq_lens, cu_new, n_pages: int, page_size: int, t: int):
    """(sequence, index in it, page, row of the page) of new token t, or None if it has no place."""
    if cu_new is None:
        if t >= len(seq_lens):
            return None
        b, at = t, int(seq_lens[t]) - 1
    else:
        own = [b for b in range(len(seq_lens)) if cu_new[b] <= t < cu_new[b + 1]]
        if not own:
            return None
        b = own[0]
        at = int(seq_lens[b]) - int(cu_new[b + 1]) + t
    if at < 0 or at >= page_table.shape[1] * page_size:
        return None
    page = int(page_table[b, at // page_size])
    return (b, at, page, at % page_size) if 0 <= page < n_pages else None


def kv_append(k_pages, v_pages, page_table, seq_lens, k, v, positions, cu_new, rope=None):
    """k [T, hk, d_qk], v [T, hk, d_v]; rope: None or (theta, offset, axis_pairs). Returns the new (k_pages, v_pages)."""
    k_out, v_out = np.array(k_pages, dtype=np.float64), np.array(v_pages, dtype=np.float64)
    for t in range(k.shape[0]):
        where = place(page_table, seq_lens, cu_new, k_out.shape[0], k_out.shape[2], t)
        if where is None:
            continue
        _, at, page, row = where
        kt = np.asarray(k[t:t + 1], dtype=np.float64)
        if rope is not None:
            theta, offset, axis_pairs = rope
            pos = [[at]] if positions is None else [[p[t]] for p in positions]
            kt = rope_axes(kt, pos, offset, axis_pairs, theta)
        k_out[page, :, row] = kt[0]
        v_out[page, :, row] = v[t]
    return k_out, v_out


def mla_rows(kv_up, k_pe, d_nope: int):
    """The rows that hydra_mla_kv_append stores, before the rotation: k [T, h, d_nope + rope], v [T, h, d_v]."""
    T, h, _ = kv_up.shape
    pe = np.broadcast_to(np.asarray(k_pe)[:, None, :], (T, h, k_pe.shape[1]))
    return np.concatenate([kv_up[:, :, :d_nope], pe], axis=2), kv_up[:, :, d_nope:]


def decode(q, k_pages, v_pages, page_table, seq_lens, scale: float):
    """q [n, h, d_qk] -> out [n, h, d_v], lse [h, n]."""
    n, h, _ = q.shape
    n_pages, hk, page_size, _ = k_pages.shape
    out = np.zeros((n, h, v_pages.shape[3]))
    lse = np.full((h, n), -np.inf)
    for b in range(n):
        length = min(max(int(seq_lens[b]), 0), page_table.shape[1] * page_size)
        at = np.arange(length)
        page = np.asarray(page_table[b])[at // page_size]
        there = (page >= 0) & (page < n_pages)
        page, row = page[there], (at % page_size)[there]
        if not len(page):
            continue
        for a in range(h):
            k = np.asarray(k_pages[page, a // (h // hk), row], dtype=np.float64)
            v = np.asarray(v_pages[page, a // (h // hk), row], dtype=np.float64)
            s = scale * (k @ np.asarray(q[b, a], dtype=np.float64))
            p = np.exp(s - s.max())
            out[b, a] = p @ v / p.sum()
            lse[a, b] = s.max() + np.log(p.sum())
    return out, lse
