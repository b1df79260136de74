"""The largest sizes that the operators of generation take: a table of 2^30 tokens, rows behind the first 2^32 elements."""
import numpy as np
import pytest
import torch

import hydra_workloads as hw
import paper_2609_34318_b200 as P
from oracle import paged_cache as C
from paged_util import DV, THETA, bits, check_decode, decode_bounds, dev, f64, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,h", [(24, 1), (64, 17)])
def test_a_sequence_of_2_30_tokens_of_which_few_pages_are_there(page, h):
    """Pages at both ends, in the middle and where a piece of the work may begin; the last one ends inside the sequence's last tile."""
    rng = np.random.default_rng(page)
    columns, d, hk = 2 ** 30 // page, 128, 1
    length = columns * page - 3
    at = np.unique(np.concatenate([[0, 1, columns // 2, columns - 2, columns - 1], rng.integers(0, columns, 40)]))
    n_pages = len(at) + 2
    ids = rng.permutation(n_pages)[:len(at)].astype(np.int32)
    table = torch.full((1, columns), -1, dtype=torch.int32, device="cuda")
    table[0, torch.from_numpy(at).cuda()] = i32(ids)
    qb, kb, vb = bits(rng, 1, h, d), bits(rng, n_pages, hk, page, d), bits(rng, n_pages, hk, page, DV)
    cache = P.paged_cache(dev(kb), dev(vb), table, i32([length]))
    out, lse = torch.empty(1, h, DV, dtype=torch.bfloat16, device="cuda"), torch.empty(h, 1, device="cuda")
    ws = torch.zeros(P.hydra_workspace_bytes_decode(h, hk), dtype=torch.uint8, device="cuda")
    scale = float(np.float32(d ** -0.5))
    P.hydra_attn_decode(dev(qb), cache, h, scale, out, lse, ws)
    assert P.hydra_poll_status(ws) == (0, -1)
    q, k, v = (hw.bf16_bits_to_f64(x) for x in (qb, kb, vb))
    small, lens = ids[None, :], np.array([len(at) * page - 3])      # the same keys as one short sequence
    check_decode(out, lse, *C.decode(q, k, v, small, lens, scale), *decode_bounds(q, k, small, lens, scale, np.abs(v).max()))


def test_rows_behind_the_first_2_32_elements():
    """Rotated to another place and in place, and read by an append: the rows of the last tokens."""
    rng = np.random.default_rng(1)
    h, d, last = 8, 128, 40
    T = 2 ** 32 // (h * d) + last
    x, y = (torch.empty(T, h, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert (T - last) * h * d == 2 ** 32
    tail = bits(rng, last, h, d)
    x[-last:] = dev(tail)
    pos = torch.zeros(2, T, dtype=torch.int32, device="cuda")
    p = rng.integers(0, 262144, (2, last)).astype(np.int32)
    pos[:, -last:] = i32(p)
    spec = P.rope_spec(THETA, d, 0, [24, 40])
    P.hydra_rope_axes(x, pos, T, h, d, spec, False, y)
    short, want = dev(tail), torch.empty(last, h, d, dtype=torch.bfloat16, device="cuda")
    P.hydra_rope_axes(short, i32(p), last, h, d, spec, False, want)
    ref = C.rope_axes(hw.bf16_bits_to_f64(tail), p, 0, [24, 40], THETA)
    assert np.abs(f64(want) - ref).max() <= 2.0 ** -8 * np.abs(ref).max() * (1 + 2.0 ** -8)
    assert torch.equal(y[-last:], want)
    page, n_pages = 16, 4                           # the tokens before the last ones are of a sequence without pages
    kp, vp = (torch.zeros(n_pages, h, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = P.paged_cache(kp, vp, i32([[-1] * 3, [3, 1, 0]]), i32([T - last, last]))
    P.hydra_kv_append(x, y, pos, i32([0, T - last, T]), T, spec, cache)
    at = torch.arange(last, device="cuda")
    pages = i32([3, 1, 0]).long()[at // page]
    assert torch.equal(kp[pages, :, at % page], want) and torch.equal(vp[pages, :, at % page], want)
    assert not kp[2].any() and not vp[2].any()
    P.hydra_rope_axes(x, pos, T, h, d, spec, False, x)
    assert torch.equal(x[-last:], want)
