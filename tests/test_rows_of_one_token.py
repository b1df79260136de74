"""Rows of a single token: torch leaves any stride on a dimension of size one, so the distance between tokens is not read from it.
[heads, 1, d] transposed is such a tensor, contiguous, with d elements from a token to the next that does not exist."""
import numpy as np
import pytest
import torch

import paper_2609_34318_b200 as P
from paper_2609_34318_b200.binding import _rows
from paged_util import DV, THETA, bits, dev, i32


class OnDevice:
    """A CPU tensor that says it is a CUDA tensor; only its description is read."""

    def __init__(self, t):
        self.t = t
        self.is_cuda, self.shape = True, t.shape

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.mark.parametrize("t,row", [
    (torch.zeros(4, 1, 192).transpose(0, 1), 768), (torch.zeros(1, 4, 192), 768), (torch.zeros(4, 0, 192).transpose(0, 1), 768),
    (torch.zeros(3000).as_strided((1, 4, 192), (777, 192, 1)), 768), (torch.zeros(3000).as_strided((1, 64), (0, 1)), 64),
    (torch.zeros(4, 1, 1, 192).permute(2, 0, 1, 3), 768), (torch.zeros(1, 40, 192)[:, 8:12], 768)])
def test_the_distance_between_tokens_of_one_token_is_its_length(t, row):
    assert _rows(OnDevice(t), None) == (t.data_ptr(), row)
    assert _rows(OnDevice(t), 1000) == (t.data_ptr(), 1000)


def test_of_several_tokens_it_is_their_stride_and_rows_are_contiguous():
    wide = torch.zeros(3, 40, 192)
    assert _rows(OnDevice(wide[:, 8:12]), None) == (wide[:, 8:12].data_ptr(), 40 * 192)
    for bad in (torch.zeros(1, 192, 4).transpose(1, 2), torch.zeros(4, 3, 192).transpose(0, 1), torch.zeros(1, 4, 384)[..., ::2]):
        with pytest.raises(ValueError):
            _rows(OnDevice(bad), None)


def _odd(t):
    """The same one token [1, heads, d], contiguous, with d as its first stride."""
    u = torch.empty(t.shape[1], 1, t.shape[2], dtype=t.dtype, device=t.device).transpose(0, 1)
    u.copy_(t)
    assert u.is_contiguous() and u.stride(0) == t.shape[2] and torch.equal(u, t)
    return u


@pytest.mark.gpu
def test_all_entry_points_take_one_token_of_any_first_stride():
    rng = np.random.default_rng(1)
    h, hk, d, page = 4, 2, 192, 8
    q, k, v = (dev(bits(rng, 1, n, w)) for n, w in ((h, d), (hk, d), (hk, DV)))
    up, pe = dev(bits(rng, 1, hk, 128 + DV)), dev(bits(rng, 1, 64))
    spec, pos = P.rope_spec(THETA, 64, 128), i32([[9]])
    want, got = torch.empty_like(q), torch.empty(h, 1, d, dtype=q.dtype, device="cuda").transpose(0, 1)
    P.hydra_rope_axes(q, pos, 1, h, d, spec, False, want)
    P.hydra_rope_axes(_odd(q), pos, 1, h, d, spec, False, got)
    assert torch.equal(want, got)
    turned = torch.zeros(1, h + 3, d, dtype=q.dtype, device="cuda")[:, :h]      # in place, as one token of rows further apart
    turned.copy_(q)
    P.hydra_rope_axes(turned, pos, 1, h, d, spec, False, turned)
    assert torch.equal(want, turned)
    turned.copy_(q)
    P.hydra_rope_axes(turned, pos, 1, h, d, spec, False, turned.data_ptr(), y_stride=(h + 3) * d)
    assert torch.equal(want, turned)

    def cache():
        pages = [torch.zeros(3, hk, page, w, dtype=q.dtype, device="cuda") for w in (d, DV)]
        return pages, P.paged_cache(*pages, i32([[2, 0]]), i32([10]))
    (a, ca), (b, cb) = cache(), cache()
    P.hydra_kv_append(k, v, pos, None, 1, spec, ca)
    P.hydra_kv_append(_odd(k), _odd(v), pos, None, 1, spec, cb)
    assert all(torch.equal(x, y) and x.any() for x, y in zip(a, b))
    (c, cc), (e, ce) = cache(), cache()
    P.hydra_mla_kv_append(up, pe, pos, None, 1, spec, cc)
    P.hydra_mla_kv_append(_odd(up), pe.as_strided((1, 64), (0, 1)), pos, None, 1, spec, ce)
    assert all(torch.equal(x, y) and x.any() for x, y in zip(c, e))
    ws = torch.zeros(P.hydra_workspace_bytes_decode(h, hk), dtype=torch.uint8, device="cuda")
    outs = []
    for x in (q, _odd(q)):
        outs.append((torch.empty(1, h, DV, dtype=q.dtype, device="cuda"), torch.empty(h, 1, device="cuda")))
        P.hydra_attn_decode(x, ca, h, 0.07, *outs[-1], ws)
    assert all(torch.equal(x, y) for x, y in zip(*outs))


def test_in_place_strides_have_to_agree_from_two_tokens_on():
    buf = np.zeros(4096, dtype=np.uint8)
    at = (buf.ctypes.data + 63) // 64 * 64          # never read: refused, or no token
    call = lambda n: P.hydra_rope_axes(at, at, n, 2, 192, P.rope_spec(THETA, 64, 128), False, at, x_stride=384, y_stride=400, stream=0,
                                       check=False)
    assert call(2) == P.HYDRA_ERR_INVALID_ARG and call(0) == P.HYDRA_OK
