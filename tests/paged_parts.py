"""Long problems of hydra_attn_decode on which a single misread slice of 16 keys shows, wherever it lies. Two kinds:

* "weights": q so small that all keys have nearly the same probability; v is one-hot, key j has its 1 in column (j // 16) % 128.
  Column c of O is the weight of the slices that bear c: a slice that is lost, or taken in another's place, changes its column by
  one part in as many as there are slices of c.
* "chosen": eight keys of every query head, at ends of the sequence, next to borders of slices and anywhere, hold nearly all of its
  probability, and v is random: O is their mean, and a row of v that meets another key's probability changes it by a large part.

What a sum of terms is off by is bounded by what each of them is off by and by the additions, relative to the sum of their absolute
values (`Parts.solve`): no cancellation is made up for by a bound as wide as the largest v, and at the lengths used half a bf16 step
of the result is nearly all of the tolerance. tests/test_paged_parts.py plants mistakes in the definition and sees them refused.
"""
from __future__ import annotations

import numpy as np

import hydra_workloads as hw
from paged_util import DV, bits, scattered_table

SLICE = 16                      # keys of a slice of a tile
ROWS = 997                      # rows of k and v that repeat (a prime: no two tiles have the same)
BLOCKS = 148
CHUNK = 1 << 15
EPS = 2.0 ** -23

# lengths, query heads, K / V heads, d, page, pages that are not there (sequence, column). Every form of the kernel: units of one, two
# and four K / V heads, up to 8, 16 and 32 query heads of one, more than 32; shares of under 32 tiles of 64 rows per thread block (of
# one piece), of 32 to 63 (four pieces) and of 64 or more (five); rows of 2 to some 300 parts.
CASES = {
    "one_head": ([100000, 3, 50001], 1, 1, 192, 64, ()),                             # 2345 tiles, share 16
    "four_kv_heads": ([40000, 36001, 0, 90], 4, 4, 192, 64, ((0, 300),)),            # 4757, 33
    "four_of_two": ([30001, 10000], 16, 8, 128, 16, ()),                             # 2 units of 2501: 5002, 34
    "two_of_eight": ([80000, 76543], 16, 2, 192, 8, ((1, 1000), (1, 1001))),         # 4892, 34
    "group_of_8": ([150001, 160000], 8, 1, 128, 64, ()),                             # 4844, 33
    "group_of_9": ([9000, 8001, 700], 9, 1, 128, 16, ()),                            # 278, 2
    "group_of_12": ([150000, 90000, 70001], 12, 1, 192, 64, ((2, 0),)),              # 4846, 33
    "group_of_16": ([200000, 5, 190001, 0, 220007], 16, 1, 128, 64, ((4, 2000),)),   # 9533, 65
    "group_of_16_two": ([70000, 80017], 32, 2, 192, 16, ()),                         # 2 units of 2345: 4690, 32
    "group_of_17": ([9000, 8000], 17, 1, 192, 24, ()),                               # 266, 2: up to 71 parts
    "group_of_24": ([100000, 70, 110000], 24, 1, 192, 64, ((0, 1),)),                # 3284, 23
    "group_of_32": ([160000, 160001], 32, 1, 128, 64, ()),                           # 5001, 34: up to 300 parts
    "group_of_32_short": ([30000], 32, 1, 192, 64, ()),                              # 469, 4: 118 parts
    "group_of_40": ([41000, 40001], 80, 2, 128, 64, ((0, 640),)),                    # 4 units of 1267: 5068, 35
}
KINDS = ("weights", "chosen")


class Parts:
    def __init__(self, name, kind):
        lengths, self.h, self.hk, self.d, self.page, missing = CASES[name]
        self.kind, d, page, n, g = kind, self.d, self.page, len(lengths), self.h // self.hk
        rng = np.random.default_rng(sum(lengths) + KINDS.index(kind))
        self.lens = np.asarray(lengths, dtype=np.int32)
        self.table, self.n_pages = scattered_table(lengths, page, rng)
        self.scale = float(np.float32(d ** -0.5))
        self.qb = bits(rng, n, self.h, d, scale=2.0 ** -6 if kind == "weights" else 1.0)
        self.q = hw.bf16_bits_to_f64(self.qb)
        place = np.arange(self.n_pages * page)
        rows = lambda step, width, scale: bits(rng, ROWS, self.hk, width, scale=scale)[place * step % ROWS].reshape(
            self.n_pages, page, self.hk, width).swapaxes(1, 2).copy()
        self.kb = rows(1, d, 1.0 if kind == "weights" else 2.0 ** -4)
        self.vb = np.zeros((self.n_pages, self.hk, page, DV), dtype=np.uint16) if kind == "weights" else rows(31, DV, 1.0)
        self.chosen = {}
        for b, length in enumerate(lengths):
            at = np.arange(length)
            pg, row = self.table[b][at // page], at % page
            if kind == "weights":
                self.vb[pg, :, row, at // SLICE % DV] = 0x3F80      # 1.0
                continue
            for a in range(self.h if length else 0):
                border = rng.integers(1, max(2, length // SLICE), 3) * SLICE
                mine = np.concatenate([[a, length - 1 - a], border - rng.integers(0, 2, 3), rng.integers(0, length, 3)])
                mine = np.unique(np.clip(mine, 0, length - 1))
                unit = self.q[b, a] / (self.q[b, a] @ self.q[b, a])
                score = 14.0 + 0.3 * rng.standard_normal((len(mine), 1))
                self.kb[pg[mine], a // g, row[mine]] = hw.f32_to_bf16_bits((score / self.scale * unit).astype(np.float32))
                self.chosen[b, a] = mine
        for b, col in missing:
            self.table[b, col] = -1
        unit_kv = next(m for m in (4, 2, 1) if m == 1 or (self.hk % m == 0 and m * g <= 16))
        self.tile_keys = 64 // unit_kv
        self.units = self.hk // unit_kv * -(-g // 32)
        self.share = -(-int(sum(-(-x // self.tile_keys) for x in lengths)) * self.units // BLOCKS)

    def keys(self, b):
        """Places of sequence b that count."""
        at = np.arange(int(self.lens[b]))
        pg = self.table[b][at // self.page]
        return at[(pg >= 0) & (pg < self.n_pages)]

    def solve(self, b, mistakes=()):
        """In 64 bits, of sequence b: [out [h, d_v] of the definition, and of every mistake], lse [h], how far out and lse may be from the
        first (out apart from its own rounding). A mistake gives, of the places that count, those that v is taken from (-1: none)."""
        h, d, g, at = self.h, self.d, self.h // self.hk, self.keys(b)
        outs, lse = [np.zeros((h, DV)) for _ in range(1 + len(mistakes))], np.full(h, -np.inf)
        bound_out, bound_lse = np.zeros((h, DV)), np.zeros(h)
        if not len(at):
            return outs, lse, bound_out, bound_lse
        sources = [at] + [m(at) for m in mistakes]
        rows = lambda x, kv, where: hw.bf16_bits_to_f64(x[self.table[b][where // self.page], kv, where % self.page])
        # additions one after the other that an element of O or of the sum of probabilities sees: two products of 16 keys per tile of
        # the block's share, the warps and parts that are joined
        additions = 32 * self.share + 64
        for kv in range(self.hk):
            heads = slice(kv * g, (kv + 1) * g)
            q = self.q[b, heads]
            s, s_abs = np.empty((g, len(at))), np.zeros(g)
            for i in range(0, len(at), CHUNK):
                k = rows(self.kb, kv, at[i:i + CHUNK])
                s[:, i:i + CHUNK] = self.scale * (q @ k.T)
                s_abs = np.maximum(s_abs, self.scale * (np.abs(q) @ np.abs(k).T).max(1))
            top, s_max = s.max(1, keepdims=True), np.abs(s).max(1)
            p = np.exp(s - top)
            total = p.sum(1)
            p /= total[:, None]
            lse[heads] = top[:, 0] + np.log(total)
            # A score is off by (d + 2) EPS of its products' absolute sum, the exponential by 2^-22 and its argument's rounding, a
            # probability enters the product with v in two bf16 (2^-17), and up to 16 factors 2^(m - m') are applied when the running
            # maximum is raised and parts are joined (2^-18). Twice that, for the probability and for the sum it is divided by.
            r = (d + 2) * EPS * s_abs + 2.0 ** -22 + 3 * EPS * s_max + 2.0 ** -17 + 2.0 ** -18
            bound_lse[heads] = 2 * r + additions * EPS + 8 * EPS * (s_max + np.log(len(at)) + 1)
            off = (2 * r + 2 * additions * EPS)[:, None]
            for o, src in zip(outs, sources):
                w = p if src is at else np.where(src < 0, 0.0, p)
                if self.kind == "weights":
                    for a in range(g):
                        o[kv * g + a] = np.bincount(src // SLICE % DV, weights=w[a], minlength=DV)
                    if src is at:
                        bound_out[heads] = off * o[heads]
                    continue
                for i in range(0, len(at), CHUNK):
                    v = rows(self.vb, kv, np.maximum(src[i:i + CHUNK], 0))
                    o[heads] += w[:, i:i + CHUNK] @ v
                    if src is at:
                        bound_out[heads] += off * (w[:, i:i + CHUNK] @ np.abs(v))
        return outs, lse, bound_out, bound_lse


def excess(out, lse, ref_out, ref_lse, bound_out, bound_lse):
    """How much further out and lse (64-bit arrays of the values that a call gave) are from the definition than the bounds and half a
    bf16 step of the result allow: at most 0 where they are right."""
    if not np.isfinite(out).all() or not np.array_equal(np.isneginf(lse), np.isneginf(ref_lse)):
        return np.inf, np.inf
    over = np.abs(out - ref_out) - (bound_out * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref_out))
    fin = np.isfinite(ref_lse)
    return float(over.max(initial=-np.inf)), float((np.abs(lse[fin] - ref_lse[fin]) - bound_lse[fin]).max(initial=-np.inf))
