"""Infinities in the low-rank adapters: where the formula's sum is an infinity the kernels' is the same one, not NaN."""
import numpy as np
import pytest

import oracle.adapter as A
from test_gpu_adapter import Case, backward, dr, forward  # noqa: F401  (dr: the fixture)

pytestmark = pytest.mark.gpu


def positive(M, K, N, R, adapters=3, kind="even"):
    """A case of positive numbers alone, none near zero: a sum with an infinity among its terms is that infinity."""
    c = Case(M, K, N, R, adapters, kind)
    for name in ("x", "w", "a", "b", "dy"):
        setattr(c, name, np.maximum(np.abs(getattr(c, name)), 2.0 ** -6))
    return c


def row_of(c, variant):
    """The last row of a variant's last request."""
    return [v for u, v, a in A.requests(c.row_start, c.ids, c.adapters) if a == variant][-1] - 1


def same_kind(got, want):
    assert np.array_equal(np.isnan(got), np.isnan(want)), "NaN"
    assert np.array_equal(np.isposinf(got), np.isposinf(want)) and np.array_equal(np.isneginf(got), np.isneginf(want))


def t32(c):
    t = A.forward(c.x, c.w, None, c.a, c.b, c.scale, c.row_start, c.ids, False)[1]
    return np.nan_to_num(t, nan=0.5, posinf=0.5, neginf=0.5).astype(np.float32).astype(np.float64)


def both(dr, c, f32, want=(0, 1, 2)):
    """Forward and backward against the formulas; want: which of dx, da, db."""
    with np.errstate(invalid="ignore", over="ignore"):
        y, t = A.forward(c.x, c.w, c.bias, c.a, c.b, c.scale, c.row_start, c.ids, False)
        gy, gt, inside = forward(dr, c, f32=f32)
        same_kind(gt[inside], t[inside])
        same_kind(gy[inside], y[inside])
        grads, tt = A.backward(c.dy, c.x, c.w, c.a, c.b, c.scale, c.row_start, c.ids, t32(c)), t32(c)
        got = backward(dr, c, tt)
        for i in want:
            same_kind(got[i][inside] if i == 0 else got[i], grads[i][inside] if i == 0 else grads[i])


# up to 128 rows, more of them, the tiles of the first product; ranks that are no multiple of 8
SHAPES = [(20, 72, 136, 1), (20, 72, 136, 5), (300, 72, 136, 3), (300, 64, 72, 12), (14300, 520, 72, 20), (14300, 520, 72, 130)]


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("M,K,N,R", SHAPES)
def test_an_infinity_in_a_row(dr, M, K, N, R, f32):
    c = positive(M, K, N, R)
    c.x[row_of(c, 1), 9] = np.inf
    both(dr, c, f32, want=(0,))
    c = positive(M, K, N, R)
    c.dy[row_of(c, 2), 11] = np.inf
    both(dr, c, f32, want=(0, 1))


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("M,K,N,R", SHAPES)
def test_an_infinite_scale(dr, M, K, N, R, f32):
    c = positive(M, K, N, R)
    c.scale[1] = np.inf
    both(dr, c, f32)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("M,K,N,R", SHAPES + [(19000, 1024, 1024, 16)])            # the last: pairs of CTAs, with one accumulator or two
def test_infinities_on_both_sides_of_a_product(dr, M, K, N, R, f32):
    """A row whose t (u) is infinite and an infinite entry of its own variant's second factor: their product is an infinity."""
    c = positive(M, K, N, R)
    c.x[row_of(c, 1), 9] = c.b[1, 70, R // 2] = np.inf
    c.dy[row_of(c, 1), 11] = c.a[1, R // 2, 5] = np.inf
    both(dr, c, f32, want=(0,))
    # the other sign: the shared part stays finite, t is infinite by its scale
    c = positive(M, K, N, R)
    c.scale[1] = np.inf
    c.b[1, 70] *= -1
    c.b[1, 70, R // 2] = -np.inf
    both(dr, c, f32, want=())
