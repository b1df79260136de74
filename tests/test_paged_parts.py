"""The checks of tests/test_gpu_attn_decode_parts.py refuse what a kernel could do wrong: the mistakes are planted in the definition,
at the lengths and head layouts that are used there."""
import numpy as np
import pytest

import hydra_workloads as hw
from paged_parts import CASES, KINDS, SLICE, Parts, excess

bf16 = lambda x: hw.bf16_bits_to_f64(hw.f32_to_bf16_bits(x.astype(np.float32)))


def lost(first, count):
    return lambda at: np.where((at >= first) & (at < first + count), -1, at)


def taken_from(first, count, other):
    def places(at):
        there = set(at.tolist())
        out = at.copy()
        for j in range(count):
            if first + j in there and other + j in there:
                out[np.searchsorted(at, first + j)] = other + j
        return out
    return places


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", CASES)
def test_a_slice_that_is_lost_or_misplaced_is_refused(name, kind):
    p = Parts(name, kind)
    rng = np.random.default_rng(7)
    for b in {int(np.argmax(p.lens)), int(np.argsort(p.lens)[-2]) if len(p.lens) > 1 else 0}:
        n = int(p.lens[b])
        if n < 2 * SLICE:
            continue
        if kind == "weights":
            # any slice: the first, the last whole one, a tile's, others
            slices = [0, n // SLICE - 1] + rng.integers(0, n // SLICE, 4).tolist()
            slices = [s for s in slices if np.isin(np.arange(s * SLICE, (s + 1) * SLICE), p.keys(b)).all()]
            mistakes = [lost(s * SLICE, SLICE) for s in slices] + [taken_from(s * SLICE, SLICE, s * SLICE + (SLICE if s == 0 else -SLICE))
                                                                   for s in slices]
        else:
            # one row of any chosen key, and the rows of its slice in another order
            keys = [j for a in range(0, p.h, max(1, p.h // 4)) for j in p.chosen[b, a].tolist()[::3] if j in p.keys(b)]
            mistakes = [lost(j, 1) for j in keys] + [taken_from(j, 1, j ^ 1) for j in keys if (j ^ 1) in p.keys(b)]
        outs, lse, bound_out, bound_lse = p.solve(b, mistakes)
        over = excess(bf16(outs[0]), lse.astype(np.float32).astype(np.float64), outs[0], lse, bound_out, bound_lse)
        assert max(over) <= 0.0
        assert len(mistakes) >= 4
        for wrong in outs[1:]:
            assert excess(bf16(wrong), lse, outs[0], lse, bound_out, bound_lse)[0] > 0.0
        # and parts of a row that are joined with factors that are off by a hundredth
        off = outs[0] * np.where(rng.random(outs[0].shape[0]) < 0.5, 1.01, 0.99)[:, None]
        assert excess(bf16(off), lse, outs[0], lse, bound_out, bound_lse)[0] > 0.0
        assert excess(bf16(outs[0]), lse + 0.01, outs[0], lse, bound_out, bound_lse)[1] > 0.0


def test_the_cases_reach_every_number_of_pieces():
    shares = {name: Parts(name, "weights").share for name in CASES}
    assert min(shares.values()) < 4 and sum(32 <= s < 64 for s in shares.values()) >= 6 and max(shares.values()) >= 64
