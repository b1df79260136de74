"""The status that a call of hydra_attn_decode without a sequence leaves, in a workspace that held anything."""
import pytest
import torch

import paper_2609_34318_b200 as P
from paged_util import DV, guarded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("fill", [0, 0x05, 0xFF])
def test_a_call_without_a_sequence_has_a_status_of_its_own(fill, captured):
    """Filled with one byte, a status block says that the call of the number it holds has failed."""
    h, hk, d = 4, 2, 192
    k, v = torch.zeros(3, hk, 16, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, hk, 16, DV, dtype=torch.bfloat16, device="cuda")
    cache = P.paged_cache(k, v, torch.zeros(0, 4, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"))
    q, out, lse = (torch.empty(0, h, w, dtype=torch.bfloat16, device="cuda") for w in (d, DV, 1))
    ws, check_ws = guarded((P.hydra_workspace_bytes_decode(h, hk),), torch.uint8, fill=0)
    call = lambda: P.hydra_attn_decode(q, cache, h, 0.1, out, lse.float(), ws)
    if captured:
        graph = torch.cuda.CUDAGraph()
        call()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            call()
    for _ in range(2):
        ws.fill_(fill)
        graph.replay() if captured else call()
        assert P.hydra_poll_status(ws) == (0, -1)
        check_ws()
