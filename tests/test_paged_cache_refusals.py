"""What the entry points of generation refuse, with the documented codes and before anything is launched. No kernel runs here:
host addresses stand for device memory, and what passes every check ends at the missing device (or is not called)."""
import numpy as np
import pytest

import paper_2609_34318_b200 as P

_BUF = np.zeros(4096 + 64, dtype=np.uint8)
A = (_BUF.ctypes.data + 63) // 64 * 64                      # an aligned address; never read
INVALID, UNSUPPORTED = P.HYDRA_ERR_INVALID_ARG, P.HYDRA_ERR_UNSUPPORTED


def spec(theta=1e4, dim=64, offset=128, pairs=(32,), n_axes=None):
    s = P.rope_spec(theta, dim, offset, pairs)
    if n_axes is not None:
        s.n_axes = n_axes
    return s


def cache(**change):
    d = dict(k=A, v=A, page_table=A, seq_lens=A, n_pages=10, page_size=16, n_kv_heads=2, d_qk=192, d_v=128, n_seqs=3, max_pages=4)
    d.update(change)
    c = P.hydra_paged_cache_t()
    for name, value in d.items():
        setattr(c, name, value)
    return c


def rope(x=A, positions=A, n=4, h=2, d=192, s=None, y=A + 16, xs=None, ys=None, inverse=False):
    return P.hydra_rope_axes(x, positions, n, h, d, s or spec(), inverse, y, x_stride=h * d if xs is None else xs,
                             y_stride=h * d if ys is None else ys, stream=0, check=False)


@pytest.mark.parametrize("change,status", [
    (dict(s=spec(theta=1.0)), INVALID), (dict(s=spec(theta=float("inf"))), INVALID), (dict(s=spec(theta=float("nan"))), INVALID),
    (dict(s=spec(pairs=(31,))), INVALID), (dict(s=spec(pairs=(40, -8))), INVALID), (dict(s=spec(n_axes=0)), INVALID),
    (dict(s=spec(n_axes=5)), INVALID), (dict(s=spec(offset=136)), INVALID), (dict(s=spec(offset=-8)), INVALID),
    (dict(s=spec(offset=2**31 - 8)), INVALID), (dict(s=spec(dim=63, pairs=(31,))), INVALID),
    (dict(s=spec(dim=60, pairs=(30,))), UNSUPPORTED), (dict(s=spec(offset=4)), UNSUPPORTED),
    (dict(s=spec(dim=264, offset=0, pairs=(132,)), d=512), UNSUPPORTED), (dict(d=1032), UNSUPPORTED),
    (dict(d=196, s=spec(dim=64, offset=0)), UNSUPPORTED), (dict(h=65537), UNSUPPORTED), (dict(h=0), INVALID), (dict(n=-1), INVALID),
    (dict(xs=383), INVALID), (dict(ys=376), INVALID), (dict(xs=388), UNSUPPORTED), (dict(ys=388), UNSUPPORTED),
    (dict(x=A, y=A, ys=400), INVALID), (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(positions=None), INVALID),
    (dict(x=A + 8), INVALID), (dict(y=A + 8), INVALID), (dict(positions=A + 2), INVALID), (dict(n=0, x=None), P.HYDRA_OK)])
def test_rope_axes(change, status):
    assert rope(**change) == status


def test_a_rope_of_too_many_axes_is_refused_in_the_binding():
    with pytest.raises(ValueError):
        P.rope_spec(1e4, 64, 0, [8, 8, 8, 4, 4])


def append(k=A, v=A, positions=A, cu=A, n=4, s=None, c=None, ks=None, vs=None, no_rope=False):
    c = c or cache()
    return P.hydra_kv_append(k, v, positions, cu, n, None if no_rope else s or spec(), c,
                             k_stride=c.n_kv_heads * c.d_qk if ks is None else ks,
                             v_stride=c.n_kv_heads * c.d_v if vs is None else vs, stream=0, check=False)


def mla(up=A, pe=A, positions=A, cu=A, n=4, s=None, c=None, us=2 * 256, ps=64):
    return P.hydra_mla_kv_append(up, pe, positions, cu, n, s or spec(), c or cache(), kv_up_stride=us, k_pe_stride=ps, stream=0,
                                 check=False)


BAD_CACHES = [(dict(n_pages=0), INVALID), (dict(page_size=0), INVALID), (dict(n_kv_heads=0), INVALID), (dict(d_qk=0), INVALID),
              (dict(n_seqs=-1), INVALID), (dict(max_pages=0), INVALID), (dict(k=None), INVALID), (dict(v=A + 8), INVALID),
              (dict(page_table=A + 2), INVALID), (dict(seq_lens=None), INVALID)]


@pytest.mark.parametrize("change,status", [
    (dict(c=cache(**ch)), st) for ch, st in BAD_CACHES] + [
    (dict(c=cache(d_qk=196), no_rope=True), UNSUPPORTED), (dict(c=cache(d_v=132)), UNSUPPORTED),
    (dict(c=cache(d_qk=1032), no_rope=True), UNSUPPORTED), (dict(ks=380), INVALID), (dict(vs=255), INVALID), (dict(ks=388), UNSUPPORTED),
    (dict(vs=260), UNSUPPORTED), (dict(n=-1), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=A + 8), INVALID),
    (dict(positions=None, s=spec(pairs=(16, 16))), INVALID), (dict(positions=A + 2), INVALID), (dict(cu=A + 2), INVALID),
    (dict(s=spec(pairs=(31,))), INVALID), (dict(s=spec(dim=60, pairs=(30,))), UNSUPPORTED),
    (dict(n=0, k=None), P.HYDRA_OK), (dict(c=cache(n_seqs=0, k=None)), P.HYDRA_OK)])
def test_kv_append(change, status):
    assert append(**change) == status


@pytest.mark.parametrize("change,status", [
    (dict(c=cache(**ch)), st) for ch, st in BAD_CACHES] + [
    (dict(s=spec(offset=64)), INVALID), (dict(us=511), INVALID), (dict(ps=63), INVALID), (dict(us=516), UNSUPPORTED), (dict(ps=65), UNSUPPORTED),
    (dict(up=None), INVALID), (dict(pe=None), INVALID), (dict(pe=A + 2), INVALID), (dict(up=A + 8), INVALID), (dict(n=0), P.HYDRA_OK)])
def test_mla_kv_append(change, status):
    assert mla(**change) == status


def test_the_mla_form_needs_its_rotation():
    assert P.hydra_mla_kv_append(A, A, A, A, 4, None, cache(), kv_up_stride=512, k_pe_stride=64, stream=0, check=False) == INVALID


def decode(q=A, c=None, h=4, scale=0.1, out=A, lse=A, ws=A, nbytes=1 << 30, qs=None):
    c = c or cache()
    return P.hydra_attn_decode(q, c, h, scale, out, lse, ws, workspace_bytes=nbytes, q_stride=h * c.d_qk if qs is None else qs,
                               stream=0, check=False)


@pytest.mark.parametrize("change,status", [
    (dict(c=cache(**ch)), st) for ch, st in BAD_CACHES] + [
    (dict(h=0), INVALID), (dict(h=3), INVALID), (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(qs=760), INVALID), (dict(qs=772), UNSUPPORTED), (dict(c=cache(d_qk=64)), UNSUPPORTED),
    (dict(c=cache(d_v=64)), UNSUPPORTED), (dict(c=cache(page_size=12)), UNSUPPORTED), (dict(c=cache(page_size=4)), UNSUPPORTED),
    (dict(c=cache(n_seqs=2**30)), UNSUPPORTED), (dict(c=cache(max_pages=2**27)), UNSUPPORTED),
    (dict(c=cache(n_seqs=2**13, max_pages=2**18)), UNSUPPORTED), (dict(q=None), INVALID), (dict(q=A + 8), INVALID), (dict(out=None), INVALID),
    (dict(lse=None), INVALID), (dict(out=A + 8), INVALID), (dict(ws=None), INVALID), (dict(ws=A + 8), INVALID),
    (dict(nbytes=P.hydra_workspace_bytes_decode(4, 2) - 1), P.HYDRA_ERR_WORKSPACE_TOO_SMALL)])
def test_attn_decode(change, status):
    assert decode(**change) == status


def test_workspace_of_a_decode():
    assert P.hydra_workspace_bytes_decode(4, 3) == 0 and P.hydra_workspace_bytes_decode(0, 1) == 0
    assert 0 < P.hydra_workspace_bytes_decode(16, 16) <= P.hydra_workspace_bytes_decode(16, 1) <= P.hydra_workspace_bytes_decode(32, 1)


def test_a_cache_is_described_by_its_tensors():
    import torch
    k, v = torch.zeros(5, 2, 8, 192, dtype=torch.bfloat16), torch.zeros(5, 2, 8, 128, dtype=torch.bfloat16)
    table, lens = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for bad in ((k, v[:4], table, lens), (k, v, table, lens[:2]), (k, v, table.long(), lens), (k.float(), v, table, lens),
                (k[0], v, table, lens), (k, v, table, lens)):           # (the last: not CUDA tensors)
        with pytest.raises(ValueError):
            P.paged_cache(*bad)
