"""hydra_attn_decode against its definition in 64 bits (oracle/paged_cache.py), element by element, within bounds derived from the
number formats (tests/paged_util.py): lengths from none and one to several per thread block, every grouping, pages that end inside
a tile, missing pages, rows of anything where nothing counts; strides, streams, captured calls, the waits that run out."""
import numpy as np
import pytest
import torch

import hydra_workloads as hw
from oracle import paged_cache as C
from paged_util import DV, bits, check_decode, decode_bounds, dev, f64, guarded, i32, scattered_table

pytestmark = pytest.mark.gpu


class Problem:
    def __init__(self, lengths, h, hk, d, page, seed=0, q_scale=1.0, garbage=True, spare=3, table=None, seq_lens=None, **kw):
        import paper_2609_34318_b200 as P
        self.P, self.h, self.hk, self.d, self.page = P, h, hk, d, page
        rng = np.random.default_rng(seed)
        self.table, self.n_pages = scattered_table(lengths, page, rng, spare=spare, **kw)
        if table is not None:
            self.table = table(self.table, self.n_pages)
        self.lens = np.asarray(lengths if seq_lens is None else seq_lens, dtype=np.int32)
        n = len(lengths)
        qb = bits(rng, n, h, d, scale=q_scale)
        kb, vb = bits(rng, self.n_pages, hk, page, d), bits(rng, self.n_pages, hk, page, DV)
        self.q, self.k, self.v = (hw.bf16_bits_to_f64(x) for x in (qb, kb, vb))
        if garbage:                                 # rows that nobody's keys are: NaN and infinities of both signs
            mine = np.zeros((self.n_pages, page), dtype=bool)
            for b in range(n):
                at = np.arange(min(max(int(self.lens[b]), 0), self.table.shape[1] * page))
                pg = self.table[b][at // page]
                ok = (pg >= 0) & (pg < self.n_pages)
                mine[pg[ok], (at % page)[ok]] = True
            bad = np.array([0x7FC0, 0x7F80, 0xFF80, 0xFFFF], dtype=np.uint16)
            for x in (kb, vb):
                x.swapaxes(1, 2)[~mine] = bad[rng.integers(0, 4, x.swapaxes(1, 2)[~mine].shape)]
        self.scale = float(np.float32(d ** -0.5))
        self.qd, self.kd, self.vd, self.td, self.ld = dev(qb), dev(kb), dev(vb), i32(self.table), i32(self.lens)
        self.cache = P.paged_cache(self.kd, self.vd, self.td, self.ld)
        self.out, self.check_out = guarded((n, h, DV), torch.bfloat16)
        self.lse, self.check_lse = guarded((h, n), torch.float32)
        self.ws, self.check_ws = guarded((P.hydra_workspace_bytes_decode(h, hk),), torch.uint8, fill=0xFF)

    def run(self, q=None, **kw):
        self.P.hydra_attn_decode(self.qd if q is None else q, self.cache, self.h, self.scale, self.out, self.lse, self.ws, **kw)

    def verify(self):
        assert self.P.hydra_poll_status(self.ws) == (0, -1)
        for c in (self.check_out, self.check_lse, self.check_ws):
            c()
        ref = C.decode(self.q, self.k, self.v, self.table, self.lens, self.scale)
        check_decode(self.out, self.lse, *ref, *decode_bounds(self.q, self.k, self.table, self.lens, self.scale, np.abs(self.v).max()))


def solve(*args, **kw):
    p = Problem(*args, **kw)
    p.run()
    p.verify()
    return p


@pytest.mark.parametrize("d", [192, 128])
@pytest.mark.parametrize("h,hk", [(4, 4), (1, 1), (16, 2), (12, 1), (16, 1), (24, 1), (33, 1), (80, 2)])
def test_every_grouping(d, h, hk):
    solve([1, 17, 64, 65, 0, 300], h, hk, d, 16, seed=h)


@pytest.mark.parametrize("page", [8, 16, 24, 48, 64, 72, 128, 256])
@pytest.mark.parametrize("lengths", [[1], [63, 64, 65], [15, 16, 17, 127, 128, 129, 200]])
def test_pages_that_end_inside_a_tile(page, lengths):
    solve(lengths, 4, 2, 192, page, seed=page)
    solve(lengths, 2, 2, 128, page, seed=page + 1)


@pytest.mark.parametrize("lengths", [[0], [0, 0, 0], [0, 5, 0], [1] * 200, [3] * 700, [0] * 500 + [40] + [0] * 500 + [9]])
def test_empty_rows_and_many_sequences(lengths):
    solve(lengths, 4, 2, 128, 8, seed=len(lengths))


@pytest.mark.parametrize("lengths,h,hk", [([20000], 2, 1), ([9473], 4, 4), ([5000, 1, 3000, 64], 8, 8), ([700] * 40, 4, 4),
                                          ([64 * 148], 1, 1), ([64 * 149 + 1], 1, 1), ([64] * 147, 1, 1), ([64] * 149, 1, 1)])
def test_pairs_cut_between_thread_blocks(lengths, h, hk):
    """One part per block, many parts of one pair, pairs that begin and end inside a block's run."""
    solve(lengths, h, hk, 192, 64, seed=sum(lengths))


@pytest.mark.parametrize("share,rest,h,hk", [(31, 100, 4, 4), (32, 0, 4, 4), (33, 7, 1, 1), (63, 40, 2, 2), (64, 0, 8, 4), (65, 147, 1, 1), (130, 1, 2, 2)])
def test_shares_that_are_run_in_pieces(share, rest, h, hk):
    """Long enough for every thread block's share of the tiles to be cut and its last pieces popped, at the shares where the number of
    pieces changes; call after call on two problems in turn, every result bit for bit the first one."""
    tile = 64 // hk                                 # keys; one unit per sequence, 148 shares of `share` tiles
    tiles = 148 * share - rest
    lengths = [tile * (tiles // 2) - 3, 5, tile * (tiles // 3), 0, tile * 7 + 1]
    lengths.append(tile * (tiles - sum(-(-n // tile) for n in lengths)) - tile // 2)
    p = Problem(lengths, h, hk, 128, 64, seed=share, garbage=False)
    other = Problem([n // 2 for n in lengths], h, hk, 128, 64, seed=share + 1, garbage=False)
    p.run()
    p.verify()
    first, first_l = p.out.clone(), p.lse.clone()
    for _ in range(10):
        other.run()
        p.out.fill_(float("nan"))
        p.run()
        assert torch.equal(p.out, first) and torch.equal(p.lse, first_l)
    other.verify()


def test_missing_pages_and_lengths_outside_the_table():
    def table(t, n):
        t[0, 1] = -1                                # in the middle
        t[1, 0] = n                                 # the first
        t[2, :] = -7                                # all of them: a row without a key
        t[3, 2:4] = 2 ** 31 - 1
        t[4, 4] = -2 ** 31                          # the last
        return t
    solve([80, 80, 80, 200, 80], 4, 2, 192, 16, table=table, seed=1)
    # longer than the table: what has no place does not count; negative: nothing does
    solve([100, 100, 100], 4, 4, 128, 16, seed=2, extra_columns=0, seq_lens=[2 ** 31 - 1, -5, 113])


def test_sequences_that_share_pages():
    def table(t, n):
        t[1, :3] = t[0, :3]
        t[2] = t[0]
        return t
    solve([100, 70, 100, 20], 4, 1, 192, 16, table=table, seed=3, garbage=False)


def test_large_scores_raise_the_running_maximum():
    p = Problem([700, 130], 8, 2, 128, 16, seed=4, q_scale=12.0)
    p.run()
    p.verify()
    # and rising ones: keys along one direction, ever longer
    p = Problem([512], 2, 1, 128, 64, seed=5, garbage=False)
    order = p.table[0, :8]
    ramp = np.zeros((p.n_pages, 1, 64, 128), dtype=np.float32)
    ramp[order, 0, :, 0] = np.arange(512).reshape(8, 64) * 0.25
    p.kd.copy_(dev(hw.f32_to_bf16_bits(ramp)))
    p.k = f64(p.kd)
    for sign in (1.0, -1.0):
        p.qd.zero_()
        p.qd[..., 0] = 16.0 * sign
        p.q = f64(p.qd)
        p.run()
        p.verify()


def test_rows_of_a_fused_projection_and_a_workspace_of_anything():
    p = Problem([65, 300, 0, 7], 4, 2, 192, 16, seed=6)
    wide = torch.full((4, 4 * 192 + 40), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + 4 * 192] = p.qd.view(4, -1)
    q = wide[:, 8:8 + 4 * 192].unflatten(1, (4, 192))
    for fill in (0, 0x55, 0xFF):
        p.ws.fill_(fill)
        p.out.fill_(float("nan"))
        p.run(q=q)
        p.verify()


def test_results_do_not_depend_on_timing_or_on_what_ran_before():
    p = Problem([3000, 100, 1], 4, 2, 192, 64, seed=7)
    p.run()
    torch.cuda.synchronize()
    first, first_l = p.out.clone(), p.lse.clone()
    other = Problem([50] * 30, 4, 2, 192, 64, seed=8)
    for i in range(20):
        other.run()
        p.out.fill_(float("nan"))
        p.run()
        assert torch.equal(p.out, first) and torch.equal(p.lse, first_l)


def test_two_streams_at_once():
    ps = [Problem([2000 + 500 * i, 9], 4, 4, 192, 16, seed=20 + i) for i in range(3)]
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    for _ in range(10):
        for p, s in zip(ps, streams):
            p.run(stream=s)
    torch.cuda.synchronize()
    for p in ps:
        p.verify()


def test_a_captured_call_follows_lengths_and_table():
    p = Problem([200, 0, 90, 1500], 4, 2, 128, 16, seed=9, garbage=False)
    p.run()                                         # what a device does once comes before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run()
    for lens in ([200, 0, 90, 1500], [1, 0, 89, 3], [0, 0, 0, 0], [150, 0, 1, 1501]):
        p.lens = np.asarray(lens, dtype=np.int32)
        p.ld.copy_(i32(lens))
        p.table[0, 2] = -1 if lens[0] == 150 else p.table[0, 2]
        p.td.copy_(i32(p.table))
        p.out.fill_(float("nan"))
        p.lse.fill_(float("nan"))
        graph.replay()
        p.verify()


def test_captured_calls_that_share_a_workspace_and_run_in_pieces():
    """The pieces are counted in the workspace: two recorded calls and one that is not use the same, one after the other."""
    a, b = Problem([16 * 148 * 40, 700, 0], 4, 4, 128, 64, seed=30, garbage=False), Problem([9000, 16 * 148 * 33], 4, 4, 192, 16, seed=31, garbage=False)
    b.ws, b.check_ws = a.ws, a.check_ws
    wants, graphs = [], []
    for p in (a, b):
        p.run()
        p.verify()
        wants.append((p.out.clone(), p.lse.clone()))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            p.run()
    for i in range(10):
        for p in (a, b):
            p.out.fill_(float("nan"))
        graphs[0].replay()
        graphs[1].replay()
        if i % 3 == 0:
            a.run()
        for p, (out, lse) in zip((a, b), wants):
            assert torch.equal(p.out, out) and torch.equal(p.lse, lse)
    a.verify()


def test_refused_calls_launch_nothing():
    import paper_2609_34318_b200 as P
    p = Problem([10], 4, 2, 192, 16, seed=10)
    n0 = P.hydra_launch_count()
    assert P.hydra_attn_decode(p.qd, p.cache, 3, p.scale, p.out, p.lse, p.ws, check=False) == P.HYDRA_ERR_INVALID_ARG
    assert P.hydra_attn_decode(p.qd, p.cache, 4, -1.0, p.out, p.lse, p.ws, check=False) == P.HYDRA_ERR_INVALID_ARG
    assert P.hydra_attn_decode(p.qd, p.cache, 4, p.scale, p.out, p.lse, p.ws, workspace_bytes=64, check=False) == \
        P.HYDRA_ERR_WORKSPACE_TOO_SMALL
    with pytest.raises(P.HydraError):
        P.hydra_attn_decode(p.qd, p.cache, 3, p.scale, p.out, p.lse, p.ws)
    with pytest.raises(ValueError):
        P.hydra_attn_decode(p.qd.transpose(1, 2), p.cache, 4, p.scale, p.out, p.lse, p.ws)
    assert P.hydra_launch_count() == n0
    assert torch.isnan(p.out.float()).all()


def test_waits_that_run_out_leave_a_status_and_the_next_call_is_right():
    """The loading warp idles for 3 ms and loads nothing, the other warps' waits run out after 0.5 ms: the kernel returns by itself."""
    import paper_2609_34318_b200 as P
    p = Problem([900, 40], 4, 2, 192, 16, seed=11)
    P.hydra_set_wait_limit_ns(500_000)
    P.hydra_debug_stall(P.HYDRA_STALL_DECODE, 3_000_000)
    try:
        p.run()
        status, detail = P.hydra_poll_status(p.ws)
    finally:
        P.hydra_debug_stall(P.HYDRA_STALL_DECODE, 0)
        P.hydra_set_wait_limit_ns(2_000_000_000)
    assert status == P.HYDRA_ERR_DEVICE_TIMEOUT and 0 <= detail < 148
    p.run()
    p.verify()
