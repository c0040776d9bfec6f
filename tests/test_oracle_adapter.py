"""Pins of the float64 forms of dropout and adapters: the generator's published answers, hand-worked cases, central differences."""
import numpy as np
import pytest

import oracle.adapter as A


@pytest.mark.parametrize("counter,key,want", [
    # known answers published with the generator
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator_known_answers(counter, key, want):
    got = A.philox4x32(np.array(counter, np.uint32), key)
    assert tuple(int(v) for v in got) == want


def test_mask_layout_and_share():
    # element e takes half-word e mod 8 of counter e / 8; a zero key and counter are the first published answer
    words = (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)
    halves = [h for w in words for h in (w & 0xFFFF, w >> 16)]
    for p in (0.1, 0.5, 0.9):
        assert A.keep_mask(1, 8, p, 0, 0)[0].tolist() == [h >= A.threshold(p) for h in halves]
    m = A.keep_mask(100, 1000, 0.3, 12345, 6)
    # 1e5 draws: the share is within five deviations, sqrt(0.21 / 1e5) each
    assert abs((~m).mean() - 0.3) < 5 * np.sqrt(0.21 / 1e5)
    assert np.array_equal(A.keep_mask(50, 1000, 0.3, 12345, 6, first=50000), m[50:])         # a tensor's rows do not depend on where they start
    assert (A.keep_mask(100, 1000, 0.3, 12345, 7) != m).any() and (A.keep_mask(100, 1000, 0.3, 12346, 6) != m).any()
    assert A.keep_mask(3, 5, 0.0, 1, 2).all() and not A.keep_mask(3, 5, 1.0, 1, 2).any()


def case(rng, M=11, K=6, N=5, R=3, adapters=3):
    x, w, bias = rng.normal(size=(M, K)), rng.normal(size=(N, K)), rng.normal(size=N)
    a, b, scale = rng.normal(size=(adapters, R, K)), rng.normal(size=(adapters, N, R)), rng.uniform(0.5, 2, adapters)
    return x, w, bias, a, b, scale, np.array([1, 3, 3, 6, 8, 10]), np.array([2, 0, 1, -1, 2])


def test_forward_is_a_layer_of_its_own_for_each_request():
    x, w, bias, a, b, scale, rs, ad = case(np.random.default_rng(0))
    y, t = A.forward(x, w, bias, a, b, scale, rs, ad, False)
    for m in range(11):
        s = {1: 2, 2: 2, 3: 1, 4: 1, 5: 1, 6: -1, 7: -1, 8: 2, 9: 2}.get(m)
        if s is None:
            assert np.isnan(y[m]).all() and np.isnan(t[m]).all()
            continue
        full = w if s < 0 else w + scale[s] * b[s] @ a[s]
        assert np.allclose(y[m], full @ x[m] + bias, rtol=1e-13)
    assert np.nanmin(A.forward(x, w, bias, a, b, scale, rs, ad, True)[0]) == 0


@pytest.mark.parametrize("p", [0.0, 0.4])
def test_gradients_against_differences(p):
    rng = np.random.default_rng(1)
    x, w, bias, a, b, scale, rs, ad = case(rng)
    f = A.factors(*x.shape, p, 9, 4)
    dy = rng.normal(size=(11, 5))
    inside = np.zeros((11, 1)) + [[float(1 <= m < 10)] for m in range(11)]

    def loss(x, a, b):
        return (np.nan_to_num(A.forward(x, w, bias, a, b, scale, rs, ad, False, f)[0]) * dy * inside).sum()

    t = A.forward(x, w, bias, a, b, scale, rs, ad, False, f)[1]
    dx, da, db = A.backward(dy, x, w, a, b, scale, rs, ad, t, f)
    for got, arg in ((np.nan_to_num(dx), 0), (da, 1), (db, 2)):
        args = [x, a, b]
        for i in np.ndindex(*args[arg].shape):
            h = np.zeros_like(args[arg])
            h[i] = 1e-5
            up, down = list(args), list(args)
            up[arg], down[arg] = args[arg] + h, args[arg] - h
            # the loss is linear in each argument alone: a central difference has no error but rounding (1e-16 * |loss| / 1e-5)
            assert abs((loss(*up) - loss(*down)) / 2e-5 - got[i]) < 1e-8
