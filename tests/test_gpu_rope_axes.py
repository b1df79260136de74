"""hydra_rope_axes against its definition in 64 bits, element by element: half a bf16 step (2^-8 of the value) and, for what two
products that cancel leave of their inputs' scale, 2^-21 of it (each product and the cosine and sine are off by under 2^-23)."""
import numpy as np
import pytest
import torch

import hydra_workloads as hw
from oracle import paged_cache as C
from paged_util import THETA, bits, dev, f64, guarded, i32, to_bits

pytestmark = pytest.mark.gpu


def close(got, ref, scale):
    over = np.abs(got - ref) - (2.0 ** -8 * np.abs(ref) * (1 + 2.0 ** -8) + 2.0 ** -21 * scale)
    assert over.max(initial=0.0) <= 0.0, (float(over.max()), float(np.abs(got - ref).max()))


def solve(T, h, d, offset, axis_pairs, inverse=False, positions=None, seed=0, x_stride=None, y_stride=None, in_place=False):
    import paper_2609_34318_b200 as P
    rng = np.random.default_rng(seed)
    pos = rng.integers(0, 262144, (len(axis_pairs), T)).astype(np.int32) if positions is None else positions
    xb = bits(rng, T, h, d)
    x = hw.bf16_bits_to_f64(xb)
    xs, ys = x_stride or h * d, y_stride or h * d
    wide_x, check_x = guarded((T, xs), torch.bfloat16)
    wide_x[:, :h * d] = dev(xb).view(T, -1)
    wide_y, check_y = (wide_x, check_x) if in_place else guarded((T, ys), torch.bfloat16)
    view = lambda w: w[:, :h * d].unflatten(1, (h, d))
    spec = P.rope_spec(THETA, 2 * sum(axis_pairs), offset, axis_pairs)
    P.hydra_rope_axes(view(wide_x), i32(pos), T, h, d, spec, inverse, view(wide_y))
    torch.cuda.synchronize()
    check_x(), check_y()
    assert torch.isnan(wide_y[:, h * d:].float()).all()             # between the rows: untouched
    if not in_place:
        assert np.array_equal(to_bits(view(wide_x)), xb)
    got, ref = f64(view(wide_y)), C.rope_axes(x, pos, offset, axis_pairs, THETA, inverse)
    rot = slice(offset, offset + 2 * sum(axis_pairs))
    rest = np.ones(d, dtype=bool)
    rest[rot] = False
    assert np.array_equal(got[..., rest], x[..., rest])
    close(got[..., rot], ref[..., rot], np.abs(x).max())
    return to_bits(view(wide_y)), xb, pos


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("T,h,d,offset,axis_pairs", [
    (1, 1, 8, 0, [4]), (3, 2, 16, 8, [1, 3]), (37, 4, 192, 128, [8, 12, 12]), (700, 2, 128, 0, [16, 24, 24]), (65, 3, 72, 8, [5, 0, 7, 12]),
    (9, 130, 192, 128, [16, 16]), (5, 1, 264, 0, [60, 68]), (2, 16, 1024, 512, [128]), (1000, 1, 24, 16, [0, 0, 0, 4]), (7, 64, 128, 64, [10, 11, 11])])
def test_sections_offsets_and_sizes(T, h, d, offset, axis_pairs, in_place):
    solve(T, h, d, offset, axis_pairs, in_place=in_place, seed=T)


@pytest.mark.parametrize("T,h,d,axis_pairs", [(1, 33, 192, [8, 12, 12]), (3, 5, 1024, [40, 40]), (2, 131, 128, [16, 24, 24]), (1, 4101, 1024, [64])])
def test_numbers_of_heads_that_do_not_halve(T, h, d, axis_pairs):
    """A token's heads are shared by warps, the last of which has fewer of them."""
    solve(T, h, d, 0, axis_pairs, seed=h)
    solve(T, h, d, min(8, d - 2 * sum(axis_pairs)), axis_pairs, seed=h, in_place=True, inverse=True)


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("xs,ys", [(400, 384), (384, 392), (1000, 456)])
def test_rows_that_are_slices(xs, ys, inverse):
    solve(130, 2, 192, 128, [8, 12, 12], inverse=inverse, x_stride=xs, y_stride=ys, seed=xs)


@pytest.mark.parametrize("d,offset,pairs", [(192, 128, 32), (128, 0, 64), (40, 8, 8)])
def test_equal_positions_are_hydra_mla_rope_bit_for_bit(d, offset, pairs):
    import paper_2609_34318_b200 as P
    rng = np.random.default_rng(3)
    T, h = 513, 3
    pos = rng.integers(0, 262144, T).astype(np.int32)
    x = dev(bits(rng, T, h, d))
    for inverse in (False, True):
        plain = torch.empty_like(x)
        P.hydra_mla_rope(x, i32(pos), T, h, d, offset, 2 * pairs, THETA, inverse, plain)
        for axis_pairs in ([pairs], [pairs // 4, pairs // 2, pairs - pairs // 4 - pairs // 2]):
            y = torch.empty_like(x)
            P.hydra_rope_axes(x, i32(np.stack([pos] * len(axis_pairs))), T, h, d, P.rope_spec(THETA, 2 * pairs, offset, axis_pairs),
                              inverse, y)
            assert torch.equal(y.view(torch.int16), plain.view(torch.int16))


def test_negative_and_far_positions():
    pos = np.array([[-1, -4096, 2 ** 31 - 1, -2 ** 31], [0, 1, 2 ** 30, -7]], dtype=np.int32)
    solve(4, 2, 128, 0, [32, 32], positions=pos, seed=4)


def test_the_inverse_is_the_gradient():
    """<f(x + e d) - f(x - e d), g> / 2e against <d, f^-1(g)>, both sides from the kernel: bf16 rounds f and f^-1 only, the inputs are
    exact, so the two differ by half a step per term at most; linear, so e = 1/2 and no error of the difference."""
    import paper_2609_34318_b200 as P
    rng = np.random.default_rng(5)
    T, h, d = 64, 2, 128
    pos = i32(rng.integers(0, 5000, (3, T)))
    spec = P.rope_spec(THETA, d, 0, [16, 24, 24])
    whole = lambda: torch.from_numpy(rng.integers(-8, 9, (T, h, d)).astype(np.float32)).cuda().to(torch.bfloat16)
    x, dx, g = whole(), whole(), whole()
    f = lambda t, inv: (lambda y: (P.hydra_rope_axes(t, pos, T, h, d, spec, inv, y), y)[1])(torch.empty_like(t))
    up, down, back = f64(f(x + dx, False)), f64(f(x - dx, False)), f64(f(g, True))
    left, right = (up - down) * f64(g) / 2, f64(dx) * back
    slack = 2.0 ** -8 * ((np.abs(up) + np.abs(down)) / 2 * np.abs(f64(g))).sum() + 2.0 ** -8 * np.abs(right).sum() + 1e-3
    assert abs(left.sum() - right.sum()) <= slack


def test_no_tokens_and_refusals():
    import paper_2609_34318_b200 as P
    x = torch.zeros(4, 2, 192, dtype=torch.bfloat16, device="cuda")
    spec = P.rope_spec(THETA, 64, 128)
    n0 = P.hydra_launch_count()
    P.hydra_rope_axes(x, i32([[0]]), 0, 2, 192, spec, False, x)
    assert P.hydra_rope_axes(x, i32([[0]]), 4, 2, 192, P.rope_spec(THETA, 64, 132), False, x, check=False) == P.HYDRA_ERR_INVALID_ARG
    assert P.hydra_rope_axes(x, i32([[0]]), 4, 2, 192, P.rope_spec(THETA, 60, 128), False, x, check=False) == P.HYDRA_ERR_UNSUPPORTED
    with pytest.raises(ValueError):
        P.hydra_rope_axes(x.transpose(1, 2), i32([[0]]), 4, 2, 192, spec, False, x)
    assert P.hydra_launch_count() == n0


def test_captured_with_new_positions():
    import paper_2609_34318_b200 as P
    rng = np.random.default_rng(6)
    T, h, d, axis_pairs = 50, 4, 128, [16, 24, 24]
    xb = bits(rng, T, h, d)
    x, y, pos = dev(xb), torch.empty(T, h, d, dtype=torch.bfloat16, device="cuda"), i32(np.zeros((3, T)))
    spec = P.rope_spec(THETA, d, 0, axis_pairs)
    P.hydra_rope_axes(x, pos, T, h, d, spec, False, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.hydra_rope_axes(x, pos, T, h, d, spec, False, y)
    for _ in range(2):
        p = rng.integers(0, 9999, (3, T))
        pos.copy_(i32(p))
        graph.replay()
        close(f64(y), C.rope_axes(hw.bf16_bits_to_f64(xb), p, 0, axis_pairs, THETA), 5.0)
