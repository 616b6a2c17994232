"""The oracle of the microscaled formats and the scored routing against hand values and brute force (no GPU)."""
import math

import numpy as np
import pytest

from oracle import mx4


def test_hand_worked_block():
    x = np.zeros((1, 32))
    x[0, :8] = [7.9, -0.3, 0.25, 0.75, 2.5, 5.0, -6.5, 1.26]     # largest 7.9: exponent 2, scale 2^0
    codes, scale = mx4.quantize(x)
    assert scale.tolist() == [[127, 0, 0, 0]]
    assert mx4.dequantize(codes, scale)[0, :8].tolist() == [6.0, -0.5, 0.0, 1.0, 2.0, 4.0, -6.0, 1.5]
    assert codes[0, 0] == (7 | (9 << 4))


def test_every_code_round_trips_and_its_neighbourhood_rounds_to_it():
    for b in (1, 100, 127, 200, 252):
        for c in range(16):
            x = np.zeros((1, 32))
            x[0, 0] = 6.0 * math.ldexp(1, b - 127)
            x[0, 1] = mx4.VALUES[c & 7] * (-1 if c & 8 else 1) * math.ldexp(1, b - 127)
            codes, scale = mx4.quantize(x)
            assert scale[0, 0] == b and (codes[0, 0] >> 4) == c


def test_bounds_of_the_scale():
    x = np.zeros((4, 32))
    x[1, 3] = 2.0 ** -140
    x[2, 3] = np.inf
    x[3, 3] = np.nan
    codes, scale = mx4.quantize(x)
    assert scale[:, 0].tolist() == [0, 0, 255, 255]
    v = mx4.dequantize(codes, scale)
    assert (v[:2] == 0).all() and np.isnan(v[2:]).all()


@pytest.mark.parametrize("groups,keep,best", [(1, 1, 1), (4, 2, 1), (4, 3, 2)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_by_brute_force(groups, keep, best, score):
    rng = np.random.default_rng(5)
    x, bias = rng.normal(size=(20, 16)), rng.normal(size=16) * 0.1
    ids, w, _ = mx4.route_scored(x, 3, score, bias, groups, keep, best, True, 2.5)
    for t in range(20):
        s = [math.exp(v) / math.fsum(math.exp(u) for u in x[t]) if score == "softmax" else 1 / (1 + math.exp(-v)) for v in x[t]]
        key = [a + b for a, b in zip(s, bias)]
        size = 16 // groups
        value = [sum(sorted(key[g * size:(g + 1) * size])[::-1][:best]) for g in range(groups)]
        kept = sorted(range(groups), key=lambda g: (-value[g], g))[:keep]
        left = [e for e in range(16) if e // size in kept]
        want = sorted(left, key=lambda e: (-key[e], e))[:3]
        assert ids[t].tolist() == want
        total = sum(s[e] for e in want)
        assert np.allclose(w[t], [2.5 * s[e] / total for e in want], rtol=1e-12)


def test_product_and_combine_by_hand():
    x = np.array([[1.0, 2.0]])
    out, bound = mx4.product(x, [np.array([[3.0, -1.0]]), np.array([[0.0, 1.0]])], np.array([[1, 0, 2]], np.int32))
    assert out[0, :2, 0].tolist() == [2.0, 1.0] and np.isnan(out[0, 2, 0]) and bound[0, 1, 0] == 5.0
    out, _ = mx4.product(x, [(np.array([[1.0, 0.0]]), np.array([[0.0, 2.0]]))], np.array([[0]], np.int32))
    assert math.isclose(out[0, 0, 0], 4.0 / (1 + math.exp(-1)))
    y = mx4.combine(np.array([[[1.0], [2.0]]]), np.array([[0.5, 4.0]]), np.array([[0, 9]]), 3, np.array([[10.0]]))
    assert y.tolist() == [[10.5]]
