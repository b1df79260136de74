"""hydra_kv_append and hydra_mla_kv_append against their definition in 64 bits: every row of the cache, rows that nothing was
stored in bit for bit as they were; rotated columns within half a bf16 step (and 2^-21 of the inputs' scale, see the rotation's test)."""
import numpy as np
import pytest
import torch

import hydra_workloads as hw
from oracle import paged_cache as C
from paged_util import THETA, bits, dev, f64, guarded, i32, scattered_table, to_bits

pytestmark = pytest.mark.gpu


class Append:
    """New tokens of sequences that hold `cached` tokens already; `pad` rows behind the last sequence."""

    def __init__(self, new, cached, hk, d, dv, page, axis_pairs, mla=False, pad=0, own_positions=True, one_each=False, seed=0,
                 table=None, fused=False, offset=None, seq_lens=None):
        import paper_2609_34318_b200 as P
        self.P, self.mla = P, mla
        rng = np.random.default_rng(seed)
        self.lens = np.array([n + c for n, c in zip(new, cached)] if seq_lens is None else seq_lens, dtype=np.int32)
        self.table, n_pages = scattered_table([n + c for n, c in zip(new, cached)], page, rng)
        if table is not None:
            self.table = table(self.table, n_pages)
        self.cu = None if one_each else np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.T = T = (len(new) if one_each else int(self.cu[-1])) + pad
        self.axis_pairs = axis_pairs
        rot = 2 * sum(axis_pairs) if axis_pairs else 0
        self.offset = d - rot if offset is None else offset
        self.rot = slice(self.offset, self.offset + rot) if rot else slice(0, 0)
        self.pos = rng.integers(0, 262144, (len(axis_pairs), T)).astype(np.int32) if own_positions and axis_pairs else None
        self.spec = P.rope_spec(THETA, rot, self.offset, axis_pairs) if axis_pairs else None
        if mla:
            up, pe = bits(rng, T, hk, self.offset + dv), bits(rng, T, rot)
            self.k, self.v = C.mla_rows(hw.bf16_bits_to_f64(up), hw.bf16_bits_to_f64(pe), self.offset)
            self.src = [self._rows(up, fused), self._rows(pe, fused)]
        else:
            kb, vb = bits(rng, T, hk, d), bits(rng, T, hk, dv)
            self.k, self.v = hw.bf16_bits_to_f64(kb), hw.bf16_bits_to_f64(vb)
            self.src = [self._rows(kb, fused), self._rows(vb, fused)]
        self.kp, self.check_k = guarded((n_pages, hk, page, d), torch.bfloat16)
        self.vp, self.check_v = guarded((n_pages, hk, page, dv), torch.bfloat16)
        self.kp.copy_(dev(bits(rng, n_pages, hk, page, d)))
        self.vp.copy_(dev(bits(rng, n_pages, hk, page, dv)))
        self.before = to_bits(self.kp), to_bits(self.vp)
        self.ld, self.td = i32(self.lens), i32(self.table)
        self.cache = P.paged_cache(self.kp, self.vp, self.td, self.ld)
        self.pd = None if self.pos is None else i32(self.pos)
        self.cd = None if self.cu is None else i32(self.cu)

    @staticmethod
    def _rows(b, fused):
        t = dev(b)
        if not fused:
            return t
        flat = t.reshape(t.shape[0], -1)
        wide = torch.full((t.shape[0], flat.shape[1] + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[:, 8:8 + flat.shape[1]] = flat
        return wide[:, 8:8 + flat.shape[1]].unflatten(1, t.shape[1:])

    def run(self, **kw):
        fn = self.P.hydra_mla_kv_append if self.mla else self.P.hydra_kv_append
        fn(*self.src, self.pd, self.cd, self.T, self.spec, self.cache, **kw)

    def verify(self):
        torch.cuda.synchronize()
        self.check_k(), self.check_v()
        rope = (THETA, self.offset, self.axis_pairs) if self.axis_pairs else None
        old = [hw.bf16_bits_to_f64(b) for b in self.before]
        ref_k, ref_v = C.kv_append(*old, self.table, self.lens, self.k, self.v, self.pos, self.cu, rope)
        got_k, got_v = f64(self.kp), f64(self.vp)
        assert np.array_equal(got_v, ref_v)
        stored = np.zeros(got_k.shape, dtype=bool)
        for t in range(self.T):
            where = C.place(self.table, self.lens, self.cu, got_k.shape[0], got_k.shape[2], t)
            if where is not None:
                stored[where[2], :, where[3], self.rot] = True
        assert np.array_equal(got_k[~stored], ref_k[~stored])
        r = ref_k[stored]
        over = np.abs(got_k[stored] - r) - (2.0 ** -8 * np.abs(r) * (1 + 2.0 ** -8) + 2.0 ** -21 * np.abs(self.k).max(initial=0.0))
        assert over.max(initial=0.0) <= 0.0, float(over.max())


def solve(*args, **kw):
    a = Append(*args, **kw)
    a.run()
    a.verify()
    return a


@pytest.mark.parametrize("mla", [False, True])
@pytest.mark.parametrize("page", [1, 5, 8, 16, 64])
@pytest.mark.parametrize("new,cached", [([1], [0]), ([7, 0, 33, 1], [0, 4, 15, 100]), ([130, 65], [63, 0])])
def test_prompts_and_continuations(mla, page, new, cached):
    solve(new, cached, 3, 192, 128, page, [8, 12, 12], mla=mla, seed=page)


@pytest.mark.parametrize("mla", [False, True])
@pytest.mark.parametrize("n", [1, 5, 300])
def test_one_token_of_every_sequence(mla, n):
    rng = np.random.default_rng(n)
    cached = rng.integers(0, 200, n).tolist()
    solve([1] * n, cached, 4, 192, 128, 16, [32], mla=mla, one_each=True, own_positions=False, seed=n)
    solve([1] * n, cached, 2, 192, 128, 16, [16, 16], mla=mla, one_each=True, seed=n)


@pytest.mark.parametrize("d,dv,axis_pairs,offset", [(128, 128, [64], 0), (128, 128, [16, 24, 24], 0), (64, 24, [3, 1], 16), (72, 40, [36], 0),
                                                    (8, 8, [4], 0), (1024, 1024, [128], 512), (192, 128, None, 0)])
def test_heads_of_other_sizes(d, dv, axis_pairs, offset):
    solve([40, 9], [3, 30], 2, d, dv, 16, axis_pairs, offset=offset, seed=d)
    solve([40, 9], [3, 30], 2, d, dv, 16, axis_pairs, offset=offset, seed=d, fused=True, pad=5)


def test_many_heads_share_a_token_and_many_tokens_a_block():
    solve([3], [10], 128, 192, 128, 16, [32], mla=True, seed=1)
    solve([5], [10], 128, 128, 128, 16, [64], seed=2)
    solve([1500, 700], [10, 0], 1, 128, 128, 16, [4, 28, 32], seed=3)
    solve([600] * 5, [1] * 5, 1, 16, 8, 8, [2, 2], seed=4)


@pytest.mark.parametrize("h", [3, 5, 33, 515])
def test_numbers_of_heads_that_do_not_halve(h):
    """A token's heads are shared by warps, the last of which has fewer of them."""
    solve([1, 2], [4, 0], h, 192, 128, 8, [16, 16], mla=True, seed=h)
    solve([1, 2], [4, 0], h, 128, 128, 8, [32, 32], seed=h)
    solve([1, 1], [7, 20], h, 256, 512, 8, [64], offset=64, one_each=True, seed=h)


def test_positions_of_the_cache_by_default_and_sequences_found_among_many():
    rng = np.random.default_rng(5)
    new = rng.integers(0, 4, 1500).tolist()
    solve(new, rng.integers(0, 40, 1500).tolist(), 1, 16, 8, 8, [8], own_positions=False, seed=5)
    solve([0] * 40 + [70] + [0] * 33 + [2], [0] * 75, 2, 32, 16, 8, [8], own_positions=False, seed=6)


@pytest.mark.parametrize("mla", [False, True])
def test_tokens_without_a_place_are_skipped(mla):
    def table(t, n):
        t[0, 1] = -1
        t[1, 0] = n
        t[2, 0] = 2 ** 31 - 1
        return t
    solve([40, 10, 3, 20], [0, 0, 0, 7], 2, 192, 128, 16, [32], mla=mla, table=table, pad=9, seed=7)
    # lengths smaller than the new tokens, behind the table's end, negative, empty rows of a padded batch
    solve([6, 6, 6, 6], [10, 10, 10, 10], 2, 192, 128, 16, [32], mla=mla, seq_lens=[4, 36, -3, 2 ** 31 - 1], own_positions=False, seed=8)
    solve([1, 1, 1], [5, 5, 5], 2, 192, 128, 16, [32], mla=mla, seq_lens=[0, 6, 0], one_each=True, own_positions=False, pad=4, seed=9)


def test_rows_are_those_of_the_assembly_bit_for_bit():
    import paper_2609_34318_b200 as P
    a = Append([300], [0], 4, 192, 128, 16, [32], mla=True, own_positions=False, seed=10)
    a.run()
    k = torch.empty(300, 4, 192, dtype=torch.bfloat16, device="cuda")
    v = torch.empty(300, 4, 128, dtype=torch.bfloat16, device="cuda")
    P.hydra_mla_kv_assemble(*a.src, i32(np.arange(300)), 300, 4, 128, 64, 128, THETA, k, v)
    at = torch.arange(300, device="cuda")
    pages = a.td[0].long()[at // 16]
    assert torch.equal(a.kp[pages, :, at % 16].view(torch.int16), k.view(torch.int16))
    assert torch.equal(a.vp[pages, :, at % 16].view(torch.int16), v.view(torch.int16))


def test_captured_step_by_step():
    """One captured append is replayed for every new token: lengths and inputs change between replays."""
    a = Append([1] * 3, [0, 20, 37], 2, 192, 128, 16, [32], mla=True, one_each=True, own_positions=False, seed=11)
    a.run()
    a.verify()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    a.ld += 1
    a.lens += 1                                     # within the pages that the table has: 20 + 2 <= 32, 37 + 2 <= 48
    a.before = to_bits(a.kp), to_bits(a.vp)
    graph.replay()
    a.verify()


def test_nothing_to_append_and_refusals():
    a = Append([4], [0], 2, 192, 128, 16, [32], seed=12)
    P, n0 = a.P, a.P.hydra_launch_count()
    P.hydra_kv_append(*a.src, a.pd, a.cd, 0, a.spec, a.cache)
    assert P.hydra_kv_append(*a.src, None, a.cd, 4, P.rope_spec(THETA, 64, 128, [16, 16]), a.cache, check=False) == P.HYDRA_ERR_INVALID_ARG
    assert P.hydra_kv_append(*a.src, a.pd, a.cd, 4, P.rope_spec(THETA, 60, 128), a.cache, check=False) == P.HYDRA_ERR_UNSUPPORTED
    with pytest.raises(P.HydraError):
        P.hydra_kv_append(*a.src, a.pd, a.cd, -1, a.spec, a.cache)
    assert P.hydra_launch_count() == n0
    torch.cuda.synchronize()
    assert np.array_equal(to_bits(a.kp), a.before[0])
