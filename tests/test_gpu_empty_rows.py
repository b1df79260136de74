"""Padded batches: any number of rows without a key, or without a new token, between two that have some. What they cost does not
grow with their number as a walk from row to row would (a dependent load each)."""
import numpy as np
import pytest
import torch

import paper_2609_34318_b200 as P
from oracle import paged_cache as C
from paged_util import DV, bits, check_decode, decode_bounds, dev, i32

import hydra_workloads as hw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("empty", [0, 1, 31, 40, 1000, 1 << 18])
@pytest.mark.parametrize("units", [1, 3])
def test_a_piece_goes_on_behind_empty_rows(empty, units):
    """148 shares of two or more tiles, one of which ends a sequence and begins the next one that has keys. With 2^18 empty rows in
    between a dependent load for each of them took 40 ms, longer than the other warps wait here."""
    rng = np.random.default_rng(empty + units)
    d, page, hk = 128, 64, units                    # one K / V head a unit (an odd number of them), tiles of 64 keys
    lengths = [64 * 149 - 5, 64 * 2 + 9, 64]
    rows = [empty, 2 * empty + 1, 2 * empty + 2]
    n = 3 * empty + 3                               # empty rows in front, between the first two, and behind
    need = [-(-x // page) for x in lengths]
    ids = rng.permutation(sum(need) + 2).astype(np.int32)
    small = np.full((3, max(need)), -1, dtype=np.int32)
    for i, (b, m) in enumerate(zip(rows, need)):
        small[i, :m], ids = ids[:m], ids[m:]
    qb, kb, vb = bits(rng, 3, hk, d), bits(rng, sum(need) + 2, hk, page, d), bits(rng, sum(need) + 2, hk, page, DV)
    table = torch.full((n, max(need)), -1, dtype=torch.int32, device="cuda")
    lens, q = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, hk, d, dtype=torch.bfloat16, device="cuda")
    table[rows], lens[rows], q[rows] = i32(small), i32(lengths), dev(qb)
    out = torch.full((n, hk, DV), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((hk, n), float("nan"), device="cuda")
    ws = torch.zeros(P.hydra_workspace_bytes_decode(hk, hk), dtype=torch.uint8, device="cuda")
    cache = P.paged_cache(dev(kb), dev(vb), table, lens)
    scale = float(np.float32(d ** -0.5))
    P.hydra_attn_decode(q, cache, hk, scale, out, lse, ws)      # (what a device does once comes before the short waits)
    torch.cuda.synchronize()
    out.fill_(float("nan")), lse.fill_(float("nan"))
    P.hydra_set_wait_limit_ns(20_000_000)
    try:
        P.hydra_attn_decode(q, cache, hk, scale, out, lse, ws)
        status = P.hydra_poll_status(ws)
    finally:
        P.hydra_set_wait_limit_ns(2_000_000_000)
    assert status == (0, -1)
    qf, kf, vf = (hw.bf16_bits_to_f64(x) for x in (qb, kb, vb))
    ref = C.decode(qf, kf, vf, small, np.array(lengths), scale)
    check_decode(out[rows], lse[:, rows], *ref, *decode_bounds(qf, kf, small, np.array(lengths), scale, np.abs(vf).max()))
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[rows] = False
    assert not out[rest].any() and torch.isneginf(lse[:, rest]).all()


@pytest.mark.parametrize("pad", [0, 7])
@pytest.mark.parametrize("empty", [0, 1, 3, 4, 5, 6, 40, 1000, 1 << 20])
@pytest.mark.parametrize("first,last", [(2501, 2500), (5001, 0), (0, 5001), (2500, 2501)])
def test_new_tokens_behind_rows_without_one(empty, first, last, pad):
    """Two or more tokens to a warp, of two sequences or of one and of none (behind the last one), with rows that append nothing in
    front, between and behind. With 2^20 of them a walk takes 58 ms."""
    rng = np.random.default_rng(empty + first)
    d, dv, page, lead = 16, 8, 64, min(empty, 33)
    n, rows, T = lead + 2 * empty + 2, [lead, lead + empty + 1], first + last + pad
    new = np.zeros(n, dtype=np.int64)
    new[rows] = first, last
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    columns = -(-max(first, last) // page)
    n_pages = 2 * columns + 1
    ids = rng.permutation(n_pages).astype(np.int32)
    small = ids[:2 * columns].reshape(2, columns)
    table = torch.full((n, columns), int(ids[-1]), dtype=torch.int32, device="cuda")        # a page of its own: nothing may land there
    lens = torch.zeros(n, dtype=torch.int32, device="cuda")
    table[rows], lens[rows] = i32(small), i32([first, last])
    k, v = dev(bits(rng, T, 1, d)), dev(bits(rng, T, 1, dv))
    kp, vp = (torch.zeros(n_pages, 1, page, w, dtype=torch.bfloat16, device="cuda") for w in (d, dv))
    want_k, want_v = kp.clone(), vp.clone()
    for i, (t0, count) in enumerate([(0, first), (first, last)]):
        at = torch.arange(count, device="cuda")
        pages = i32(small[i]).long()[at // page]
        want_k[pages, 0, at % page], want_v[pages, 0, at % page] = k[t0:t0 + count, 0], v[t0:t0 + count, 0]
    cache, cud = P.paged_cache(kp, vp, table, lens), i32(cu)
    P.hydra_kv_append(k, v, None, cud, T, None, cache)
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    P.hydra_kv_append(k, v, None, cud, T, None, cache)
    end.record()
    torch.cuda.synchronize()
    assert start.elapsed_time(end) < 10.0
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v)
