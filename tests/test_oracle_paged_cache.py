"""Pins of oracle/paged_cache.py: rotary positions with several axes, the paged cache, attention of one new token."""
import numpy as np
import pytest

import hydra_workloads as hw
import oracle
from oracle import mla_ops, paged_cache as C


def test_one_axis_and_equal_positions_are_the_plain_rotation():
    rng = np.random.default_rng(1)
    x, pos = rng.standard_normal((5, 2, 24)), np.array([0, 1, 7, 4000, 262143])
    plain = mla_ops.rope(x, pos, 8, 16, 1e4)
    assert np.allclose(C.rope_axes(x, [pos], 8, [8], 1e4), plain, atol=1e-12, rtol=0)
    assert np.allclose(C.rope_axes(x, [pos, pos, pos], 8, [2, 0, 6], 1e4), plain, atol=1e-12, rtol=0)


def test_a_rotation_by_hand():
    x = np.array([1.0, 0.0, 0.0, 2.0]).reshape(1, 1, 4)
    y = C.rope_axes(x, [[3], [5]], 0, [1, 1], 100.0)            # pair 0: axis 0, rate 1; pair 1: axis 1, rate 1 / 10
    assert np.allclose(y.ravel(), [np.cos(3), np.sin(3), -2 * np.sin(0.5), 2 * np.cos(0.5)])


def test_the_inverse_undoes_the_rotation_and_is_its_adjoint():
    rng = np.random.default_rng(2)
    x, g = rng.standard_normal((6, 3, 16)), rng.standard_normal((6, 3, 16))
    pos = rng.integers(0, 1000, (3, 6))
    f = lambda z, inv: C.rope_axes(z, pos, 4, [1, 3, 2], 1e4, inv)
    assert np.allclose(f(f(x, False), True), x)
    assert np.isclose((f(x, False) * g).sum(), (x * f(g, True)).sum())
    eps = 1e-6                                                   # and the derivative: differences along a direction
    d = rng.standard_normal(x.shape)
    assert np.isclose(((f(x + eps * d, False) - f(x - eps * d, False)) * g).sum() / (2 * eps), (d * f(g, True)).sum(), rtol=1e-7)


def _cache(lengths, page, hk, d, dv, rng, spare=3):
    need = [-(-n // page) for n in lengths]
    table = np.full((len(lengths), max(need + [1]) + 1), -1, dtype=np.int32)
    ids = rng.permutation(sum(need) + spare)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    return rng.standard_normal((len(ids), hk, page, d)), rng.standard_normal((len(ids), hk, page, dv)), table


def test_a_cache_filled_token_by_token_is_the_cache_filled_at_once():
    rng = np.random.default_rng(3)
    lengths, page, hk, d, dv = [5, 0, 9, 1], 4, 2, 8, 6
    kp, vp, table = _cache(lengths, page, hk, d, dv, rng)
    T = sum(lengths)
    k, v = rng.standard_normal((T, hk, d)), rng.standard_normal((T, hk, dv))
    cu = np.concatenate([[0], np.cumsum(lengths)])
    rope = (1e4, 0, [4])
    once = C.kv_append(kp, vp, table, lengths, k, v, None, cu, rope)
    step_k, step_v = kp, vp
    for i in range(max(lengths)):
        lens = [i + 1 if i < n else 0 for n in lengths]         # a row of length 0 is skipped
        rows = [min(int(cu[b]) + i, T - 1) for b in range(len(lengths))]
        step_k, step_v = C.kv_append(step_k, step_v, table, lens, k[rows], v[rows], None, None, rope)
    assert np.array_equal(once[0], step_k) and np.array_equal(once[1], step_v)
    owned = set(table[table >= 0].tolist())
    for p in range(len(kp)):
        if p not in owned:
            assert np.array_equal(once[0][p], kp[p]) and np.array_equal(once[1][p], vp[p])


@pytest.mark.parametrize("h,hk", [(4, 4), (4, 2), (6, 1)])
def test_attention_over_the_cache_is_the_last_row_of_the_forward(h, hk):
    rng = np.random.default_rng(4)
    lengths, page = [1, 7, 8, 20], 8
    T = sum(lengths)
    cu = hw.cu_seqlens(lengths)
    bits = lambda *s: hw.f32_to_bf16_bits(rng.standard_normal(s).astype(np.float32))
    q, k, v = bits(T, h, 192), bits(T, hk, 192), bits(T, hk, 128)
    scale = np.float32(0.07)
    ref_o, ref_l = oracle.attn_fwd_gqa(q, k, v, cu, True, scale)
    kp, vp, table = _cache(lengths, page, hk, 192, 128, rng)
    kp, vp = C.kv_append(kp, vp, table, lengths, hw.bf16_bits_to_f64(k), hw.bf16_bits_to_f64(v), None, cu)
    last = cu[1:] - 1
    out, lse = C.decode(hw.bf16_bits_to_f64(q)[last], kp, vp, table, lengths, float(scale))
    assert np.allclose(out, ref_o[last], atol=1e-12) and np.allclose(lse, ref_l[:, last], atol=1e-12)


def test_missing_pages_are_keys_left_out_and_no_key_is_zero_and_minus_infinity():
    rng = np.random.default_rng(5)
    kp, vp, table = _cache([12, 12, 3], 4, 1, 8, 6, rng)
    q = rng.standard_normal((3, 2, 8))
    table[0, 1] = -1
    table[2, 0] = len(kp)
    out, lse = C.decode(q, kp, vp, table, [12, 0, 3], 0.3)
    keep = [table[0, 0], table[0, 2]]
    k, v = kp[keep][:, 0].reshape(-1, 8), vp[keep][:, 0].reshape(-1, 6)
    p = np.exp(0.3 * q[0] @ k.T)
    assert np.allclose(out[0], p @ v / p.sum(1, keepdims=True)) and np.allclose(lse[:, 0], np.log(p.sum(1)))
    assert (out[1:] == 0).all() and np.isneginf(lse[:, 1:]).all()


def test_mla_rows():
    up, pe = np.arange(2 * 3 * 5, dtype=float).reshape(2, 3, 5), np.array([[100.0, 101.0], [102.0, 103.0]])
    k, v = C.mla_rows(up, pe, 2)
    assert k.shape == (2, 3, 4) and (k[1, 2] == [up[1, 2, 0], up[1, 2, 1], 102, 103]).all() and (v[0, 1] == up[0, 1, 2:]).all()
