"""Rotation, appends and attention on a stream that is not the current one: given as an argument, or current where the tensors are
another's. The inputs arrive on that stream behind half a millisecond of waiting: a launch anywhere else reads what was there before."""
import numpy as np
import pytest
import torch

import paper_2609_34318_b200 as P
from paged_util import DV, THETA, bits, dev, i32, scattered_table

pytestmark = pytest.mark.gpu

CYCLES = 1_000_000              # of the SM clock (at most 1965 MHz)


@pytest.mark.parametrize("given", [True, False])
def test_a_step_on_another_stream(given):
    rng = np.random.default_rng(3)
    lengths, h, hk, d, page = [40, 1, 17], 4, 2, 192, 16
    n, spec = len(lengths), P.rope_spec(THETA, 64, 128)
    table, n_pages = scattered_table(lengths, page, rng)
    inputs = [dev(bits(rng, n, h, d)), dev(bits(rng, n, hk, 128 + DV)), dev(bits(rng, n, 64)), dev(bits(rng, n, hk, d)), dev(bits(rng, n, hk, DV)),
              i32(np.arange(n)[None] * 7 + 1)]
    pages = [dev(bits(rng, n_pages, hk, page, w)) for w in (d, DV)]

    def step(q, up, pe, k, v, pos, kp, vp, stream):
        cache = P.paged_cache(kp, vp, td, ld)
        turned, out, lse = torch.empty_like(q), torch.empty(n, h, DV, dtype=q.dtype, device="cuda"), torch.empty(h, n, device="cuda")
        results = []
        for append in (lambda: P.hydra_mla_kv_append(up, pe, pos, None, n, spec, cache, stream=stream),
                       lambda: P.hydra_kv_append(k, v, pos, None, n, spec, cache, stream=stream)):
            P.hydra_rope_axes(q, pos, n, h, d, spec, False, turned, stream=stream)
            append()
            P.hydra_attn_decode(turned, cache, h, 0.07, out, lse, ws, stream=stream)
            with torch.cuda.stream(stream or torch.cuda.current_stream()):
                results += [x.clone() for x in (turned, kp, vp, out, lse)]
        return results
    td, ld = i32(table), i32(lengths)
    ws = torch.zeros(P.hydra_workspace_bytes_decode(h, hk), dtype=torch.uint8, device="cuda")
    want = step(*inputs, *[x.clone() for x in pages], None)
    torch.cuda.synchronize()
    late = [torch.zeros_like(x) for x in inputs + pages]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(CYCLES)
        for x, y in zip(late, inputs + pages):
            x.copy_(y)
        if not given:
            got = step(*late, None)
    if given:
        got = step(*late, side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
