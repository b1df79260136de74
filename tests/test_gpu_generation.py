"""The operators of generation together, as they would be used: a prompt's queries rotated, its keys and values appended to the
paged cache, prefilled with hydra_attn_fwd_dims, then token by token rotate, append, attend. Every step's (out, lse) must be the
last row of causal attention over the whole sequence so far, by the oracle on the rows that the library itself stored."""
import numpy as np
import pytest
import torch

import hydra_workloads as hw
import oracle
from gpu_util import TOL_LSE, TOL_REL
from oracle import paged_cache as C
from paged_util import DV, THETA, bits, check_decode, decode_bounds, dev, f64, i32, scattered_table, to_bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("h,hk,d,mla,axes", [(4, 4, 192, True, [32]), (16, 2, 128, False, [16, 24, 24]), (8, 1, 192, False, [8, 12, 12])])
def test_prefill_and_steps(h, hk, d, mla, axes, captured):
    import paper_2609_34318_b200 as P
    rng = np.random.default_rng(h)
    prompts, steps, page = [70, 1, 200], 5, 16
    n, T0 = len(prompts), sum(prompts)
    rot = 2 * sum(axes)
    spec, scale = P.rope_spec(THETA, rot, d - rot, axes), float(np.float32(d ** -0.5))
    total = [p + steps for p in prompts]
    table, n_pages = scattered_table(total, page, rng)
    kp = torch.full((n_pages, hk, page, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    vp = torch.full((n_pages, hk, page, DV), float("nan"), dtype=torch.bfloat16, device="cuda")
    seq_lens = i32(prompts)
    cache = P.paged_cache(kp, vp, i32(table), seq_lens)

    def inputs(count):
        kv = [dev(bits(rng, count, hk, d - rot + DV)), dev(bits(rng, count, rot))] if mla else \
            [dev(bits(rng, count, hk, d)), dev(bits(rng, count, hk, DV))]
        return dev(bits(rng, count, h, d)), kv
    append = P.hydra_mla_kv_append if mla else P.hydra_kv_append
    index = np.concatenate([np.arange(p) for p in prompts])
    position = lambda at: np.stack([at, at // 7, at % 5][:len(axes)]).astype(np.int32)

    # the prompts
    cu = hw.cu_seqlens(prompts)
    q, kv = inputs(T0)
    pos = i32(position(index))
    P.hydra_rope_axes(q, pos, T0, h, d, spec, False, q)
    append(*kv, pos, i32(cu), T0, spec, cache)
    table_d = torch.from_numpy(table).cuda().long()

    def stored(b, length):
        at = torch.arange(length, device="cuda")
        pages = table_d[b][at // page]
        return kp[pages, :, at % page], vp[pages, :, at % page]
    k, v = (torch.cat([stored(b, p)[i] for b, p in enumerate(prompts)]) for i in (0, 1))
    out, lse = torch.empty(T0, h, DV, dtype=torch.bfloat16, device="cuda"), torch.empty(h, T0, device="cuda")
    fwd_ws = torch.zeros(P.hydra_workspace_bytes_dims(P.HYDRA_WS_FWD, cu, h, hk, d, DV), dtype=torch.uint8, device="cuda")
    P.hydra_attn_fwd_dims(q, k, v, cu, h, hk, d, DV, None, True, scale, out, lse, None, None, 0, fwd_ws)
    # the decode of the prompts' last tokens is the last row of that forward (both within their tolerance of the same rows)
    ws = torch.zeros(P.hydra_workspace_bytes_decode(h, hk), dtype=torch.uint8, device="cuda")
    o1, l1 = torch.empty(n, h, DV, dtype=torch.bfloat16, device="cuda"), torch.empty(h, n, device="cuda")
    last = torch.from_numpy(cu[1:].astype(np.int64) - 1).cuda()
    P.hydra_attn_decode(q[last].contiguous(), cache, h, scale, o1, l1, ws)
    torch.cuda.synchronize()
    assert np.abs(f64(o1) - f64(out[last])).max() <= TOL_REL * np.abs(f64(out[last])).max()
    assert np.abs(l1.cpu().numpy() - lse[:, last].cpu().numpy()).max() <= TOL_LSE

    # token by token
    q1, kv1 = inputs(n)
    qr, pos1 = torch.empty_like(q1), i32(position(np.zeros(n, dtype=np.int64)))

    def step():
        P.hydra_rope_axes(q1, pos1, n, h, d, spec, False, qr)
        append(*kv1, pos1, None, n, spec, cache)
        P.hydra_attn_decode(qr, cache, h, scale, o1, l1, ws)
    graph = None
    if captured:
        graph = torch.cuda.CUDAGraph()
        seq_lens.zero_()                            # (nothing is stored)
        step()
        torch.cuda.synchronize()
        assert not o1.any() and torch.isneginf(l1).all()
        with torch.cuda.graph(graph):
            step()
    for i in range(steps):
        fresh_q, fresh_kv = inputs(n)
        q1.copy_(fresh_q)
        for a, b in zip(kv1, fresh_kv):
            a.copy_(b)
        seq_lens.copy_(i32([p + i + 1 for p in prompts]))
        pos1.copy_(i32(position(np.array([p + i for p in prompts]))))
        graph.replay() if graph else step()
        assert P.hydra_poll_status(ws) == (0, -1)
        for b in range(n):
            length = prompts[b] + i + 1
            kb, vb = (to_bits(x) for x in stored(b, length))
            qb = np.zeros((length, h, d), dtype=np.uint16)
            qb[-1] = to_bits(qr[b])
            ref_o, ref_l = oracle.attn_fwd_gqa(qb, kb, vb, hw.cu_seqlens([length]), True, np.float32(scale))
            assert np.abs(f64(o1[b]) - ref_o[-1]).max() <= 2.0 ** -8 * np.abs(ref_o[-1]).max() + 1e-3
            assert np.abs(l1[:, b].cpu().numpy() - ref_l[:, -1]).max() <= TOL_LSE


def test_pages_behind_the_first_2_32_elements():
    """The last pages of a cache whose K alone has 4.3e9 elements (8.6 GB): what the appends store there, the attention reads."""
    import paper_2609_34318_b200 as P
    rng = np.random.default_rng(17)
    hk, h, d, page, lengths = 4, 8, 192, 64, [130, 1, 70]
    n_pages = 2 ** 32 // (hk * page * d) + 8
    kp = torch.empty(n_pages, hk, page, d, dtype=torch.bfloat16, device="cuda")
    vp = torch.empty(n_pages, hk, page, DV, dtype=torch.bfloat16, device="cuda")
    assert kp.numel() > 2 ** 32 and vp.numel() > 2 ** 31
    small, used = scattered_table(lengths, page, rng, spare=0)
    table = np.where(small < 0, -1, n_pages - 1 - small).astype(np.int32)
    T = sum(lengths)
    kb, vb, qb = bits(rng, T, hk, d), bits(rng, T, hk, DV), bits(rng, 3, h, d)
    cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    cache = P.paged_cache(kp, vp, i32(table), i32(lengths))
    P.hydra_kv_append(dev(kb), dev(vb), None, i32(cu), T, None, cache)
    up, pe = bits(rng, 1, hk, 128 + DV), bits(rng, 1, 64)           # the last token of the third sequence once more, from the MLA form
    P.hydra_mla_kv_append(dev(up), dev(pe), None, i32([0, 0, 0, 1]), 1, P.rope_spec(THETA, 64, 128), cache)
    out, lse = torch.empty(3, h, DV, dtype=torch.bfloat16, device="cuda"), torch.empty(h, 3, device="cuda")
    ws = torch.zeros(P.hydra_workspace_bytes_decode(h, hk), dtype=torch.uint8, device="cuda")
    scale = float(np.float32(d ** -0.5))
    P.hydra_attn_decode(dev(qb), cache, h, scale, out, lse, ws)
    assert P.hydra_poll_status(ws) == (0, -1)
    last = torch.arange(used, device="cuda").neg() + n_pages - 1
    k, v = f64(kp[last]), f64(vp[last])             # page p of the small table
    for b in range(3):
        for j in range(lengths[b] - (b == 2)):
            at, row = small[b][j // page], j % page
            assert np.array_equal(k[at, :, row], hw.bf16_bits_to_f64(kb[cu[b] + j])) and np.array_equal(v[at, :, row], hw.bf16_bits_to_f64(vb[cu[b] + j]))
    row = k[small[2][69 // page], :, 69 % page]
    assert np.array_equal(row[:, :128], hw.bf16_bits_to_f64(up)[0, :, :128]) and (row[:, 128:] == row[:1, 128:]).all()
    q = hw.bf16_bits_to_f64(qb)
    count = np.zeros_like(k[:, :1, :, :1])
    for b in range(3):
        for j in range(lengths[b]):
            count[small[b][j // page], :, j % page] = 1
    k, v = np.where(count > 0, k, 0.0), np.where(count > 0, v, 0.0)
    ref = C.decode(q, k, v, small, np.array(lengths, dtype=np.int32), scale)
    check_decode(out, lse, *ref, *decode_bounds(q, k, small, lengths, scale, np.abs(v).max()))
