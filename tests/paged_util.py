"""Helpers of the GPU tests of generation: caches with scattered pages, guarded buffers, error bounds."""
from __future__ import annotations

import numpy as np
import torch

import hydra_workloads as hw

THETA = 10000.0
DV = 128
GUARD = 4096


def bits(rng, *shape, scale=1.0):
    return hw.f32_to_bf16_bits((scale * rng.standard_normal(shape)).astype(np.float32))


def dev(b):
    from paper_2609_34318_b200.runner import bits_to_tensor
    return bits_to_tensor(b)


def to_bits(t):
    from paper_2609_34318_b200.runner import tensor_to_bits
    return tensor_to_bits(t)


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def guarded(shape, dtype, fill=float("nan")):
    """A buffer between two bands of sentinel bytes, and the function that checks the bands."""
    nbytes = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
    room = (nbytes + 255) // 256 * 256
    raw = torch.full((room + 2 * GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
    t = raw[GUARD:GUARD + nbytes].view(dtype).view(shape)
    t.fill_(fill)

    def check():
        assert bool((raw[:GUARD] == 0xA5).all()) and bool((raw[GUARD + nbytes:] == 0xA5).all()), "written outside the buffer"
    return t, check


def scattered_table(lengths, page, rng, spare=3, extra_columns=1, free=-1):
    """Page table of sequences whose pages lie anywhere among `spare` free ones; (table, number of pages)."""
    need = [-(-max(n, 0) // page) for n in lengths]
    ids = rng.permutation(sum(need) + spare)
    table = np.full((len(lengths), max(need + [0]) + extra_columns), free, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    return table, sum(need) + spare


def decode_bounds(q, k_pages, page_table, seq_lens, scale, vmax):
    """How far out [n, h, 1] (apart from its own rounding) and lse [h, n] may be from the definition. A score is a sum of d products
    that are exact in fp32; every addition is off by at most eps = 2^-23 of the largest partial sum, which sum |q_i k_i| bounds
    (whichever order, and if a step truncates), and the scale, a product of two rounded factors, by 3 eps / 2 more: ds = (d + 2)
    eps scale max_j sum_i |q_i k_i|. exp2 of the special-function unit is off by 2^-22 relative, and its argument, the difference of a
    score and a running maximum, by eps / 2 of them, at most 2 |s|; probabilities enter the product with v in two bf16, off
    by 2^-17. So a probability is off by a factor within r = 2 ds + 2^-22 + 2^-16 + 2 eps |s| (the sum of them by no more), O by 2 r max|v|, and by the
    fp32 sums of O and of the join, n eps relative at most (n terms a thread adds, under 300 here), LSE by r + 8 eps |lse|."""
    n, h, d = q.shape
    n_pages, hk, page, _ = k_pages.shape
    eps = 2.0 ** -23
    out, lse = np.zeros((n, h, 1)), np.zeros((h, n))
    for b in range(n):
        at = np.arange(min(max(int(seq_lens[b]), 0), page_table.shape[1] * page))
        pg = page_table[b][at // page]
        ok = (pg >= 0) & (pg < n_pages)
        pg, row = pg[ok], (at % page)[ok]
        for a in range(h):
            k = k_pages[pg, a // (h // hk), row]
            if not len(k):
                continue
            s_abs = scale * (np.abs(k) @ np.abs(q[b, a])).max()
            s = scale * np.abs(k @ q[b, a]).max()
            ds = (d + 2) * eps * s_abs
            r = 2 * ds + 2.0 ** -22 + 2.0 ** -16 + 2 * eps * s * 1.5
            out[b, a] = (2 * r + 300 * eps) * vmax
            lse[a, b] = r + 8 * eps * (s + np.log(len(k)) + 1)
    return out, lse


def check_decode(out, lse, ref_out, ref_lse, bound_out, bound_lse):
    """Within the bounds plus half a bf16 step of the result."""
    got, got_l = f64(out), lse.cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isneginf(got_l), np.isneginf(ref_lse))
    assert np.isfinite(got).all()
    over = np.abs(got - ref_out) - (bound_out + 2.0 ** -8 * np.abs(ref_out) * (1 + 2.0 ** -8))
    assert over.max(initial=0.0) <= 0.0, (float(over.max()), float(np.abs(got - ref_out).max()))
    fin = np.isfinite(ref_lse)
    over = np.abs(got_l[fin] - ref_lse[fin]) - bound_lse[fin]
    assert over.max(initial=0.0) <= 0.0, (float(over.max()), float(np.abs(got_l[fin] - ref_lse[fin]).max()))
