"""hydra_attn_decode of long sequences, cut into parts: every form of the kernel, with pieces that are popped and rows of hundreds of
parts, on inputs where a slice of 16 keys that is lost, doubled or met by another key's probability shows (tests/paged_parts.py)."""
import numpy as np
import pytest
import torch

import paper_2609_34318_b200 as P
from paged_parts import CASES, KINDS, Parts, excess
from paged_util import DV, dev, f64, guarded, i32

pytestmark = pytest.mark.gpu


class Call:
    def __init__(self, p):
        self.p, n = p, len(p.lens)
        self.q, self.cache = dev(p.qb), P.paged_cache(dev(p.kb), dev(p.vb), i32(p.table), i32(p.lens))
        self.out, self.check_out = guarded((n, p.h, DV), torch.bfloat16)
        self.lse, self.check_lse = guarded((p.h, n), torch.float32)
        self.ws, self.check_ws = guarded((P.hydra_workspace_bytes_decode(p.h, p.hk),), torch.uint8, fill=0xFF)

    def run(self):
        P.hydra_attn_decode(self.q, self.cache, self.p.h, self.p.scale, self.out, self.lse, self.ws)

    def guards(self):
        assert P.hydra_poll_status(self.ws) == (0, -1)
        self.check_out(), self.check_lse(), self.check_ws()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", CASES)
def test_every_slice_of_every_part(name, kind):
    c = Call(Parts(name, kind))
    c.run()
    c.guards()
    out, lse = f64(c.out), c.lse.cpu().numpy().astype(np.float64)
    for b in range(len(c.p.lens)):
        outs, ref_lse, bound_out, bound_lse = c.p.solve(b)
        over = excess(out[b], lse[:, b], outs[0], ref_lse, bound_out, bound_lse)
        assert max(over) <= 0.0, (b, over)


@pytest.mark.parametrize("name", ["group_of_8", "group_of_16", "group_of_32", "group_of_40"])
def test_calls_in_turn_repeat_bit_for_bit(name):
    """Of two problems in one workspace, eager and recorded: who runs a popped piece, and what the workspace holds, changes nothing."""
    a, b = Call(Parts(name, "chosen")), Call(Parts("group_of_24", "weights"))
    bytes_a, bytes_b = a.ws.nbytes, b.ws.nbytes
    shared = a.ws if bytes_a >= bytes_b else b.ws
    a.ws = b.ws = shared
    wants, graphs = [], []
    for c in (a, b):
        c.run()
        torch.cuda.synchronize()
        wants.append((c.out.clone(), c.lse.clone()))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            c.run()
    for i in range(8):
        for c, graph, (out, lse) in zip((a, b), graphs, wants):
            c.out.fill_(float("nan")), c.lse.fill_(float("nan"))
            graph.replay() if i % 2 else c.run()
            assert torch.equal(c.out, out) and torch.equal(c.lse, lse)
    a.guards(), b.guards()
