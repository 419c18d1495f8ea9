"""Pins of the MXFP4 and routing oracle: worked examples and properties that do not come from its code."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import formats as F
from oracle import mx


def one(values):
    x = np.zeros((1, 32))
    x[0, :len(values)] = values
    return mx.quantize(x)


def test_worked_examples():
    # amax 6: exponent 2, scale 1: the values themselves
    q = one([0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -6.0, -0.5, -0.0])
    assert q.scale[0, 0] == 127
    assert list(q.code[0, :10]) == [1, 2, 3, 4, 5, 6, 7, 15, 9, 8]
    # ties: 0.25 -> 0, 0.75 -> 1, 1.25 -> 1, 1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4
    q = one([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 4.0])
    assert list(q.code[0, :8]) == [0, 2, 2, 4, 4, 6, 6, 6]
    # amax 7.5 still has exponent 2: it saturates
    assert list(one([7.5, 7.0, 5.1]).code[0, :3]) == [7, 7, 7]
    # amax 8: exponent 3, scale 2
    q = one([8.0, 3.0, 0.5])
    assert q.scale[0, 0] == 128 and list(q.code[0, :3]) == [6, 3, 0]
    assert one([]).scale[0, 0] == 0                                  # zeros
    assert one([2.0 ** -133]).scale[0, 0] == 0 and one([2.0 ** -133]).code[0, 0] == 0
    assert one([2.0 ** -126]).scale[0, 0] == 0 and one([2.0 ** -126]).code[0, 0] == 4      # 2^-126 = 2 * 2^-127
    big = 2.0 ** 127 * (2 - 2.0 ** -7)
    assert one([big]).scale[0, 0] == 252 and one([big]).code[0, 0] == 7
    for bad in (np.inf, -np.inf, np.nan):
        q = one([bad, 1.0])
        assert q.scale[0, 0] == 255 and np.isnan(mx.dequantize(q)).all()


def test_against_rationals():
    rng = np.random.default_rng(5)
    values = [Fraction(0), Fraction(1, 2), Fraction(1), Fraction(3, 2), Fraction(2), Fraction(3), Fraction(4), Fraction(6)]
    for e in (-130, -20, 0, 90):
        bits = F.f64_to_bf16_bits_rne(np.ldexp(rng.standard_normal((1, 32)), e))
        x = F.bf16_bits_to_f64(bits)
        q = mx.quantize(x)
        exact = [abs(Fraction(float(v))) for v in x[0]]
        amax, s = max(exact), -127 + 2
        while Fraction(2) ** (s + 1) <= amax:
            s += 1
        scale = Fraction(2) ** (s - 2)
        assert q.scale[0, 0] == s - 2 + 127
        for v, code in zip(exact, q.code[0]):
            v = min(v / scale, Fraction(6))
            dist = [abs(v - w) for w in values]
            best = [i for i in range(8) if dist[i] == min(dist)]
            assert (code & 7) == (best[0] if len(best) == 1 else [i for i in best if i % 2 == 0][0])


def test_packing_round_trip():
    q = mx.quantize(np.random.default_rng(1).standard_normal((3, 96)))
    r = mx.unpacked(mx.packed_codes(q), q.scale)
    assert np.array_equal(r.code, q.code) and np.array_equal(mx.dequantize(r), mx.dequantize(q))


def test_route_by_hand():
    inf = np.inf
    r = mx.route([[1.0, 3.0, 3.0, 0.0], [-inf, -inf, -inf, -inf], [-inf, 2.0, -inf, np.nan], [0.0, 0.0, 0.0, 0.0]], 2, True)
    assert r.ids.tolist() == [[1, 2], [-1, -1], [1, -1], [0, 1]]
    assert np.allclose(r.weights, [[0.5, 0.5], [0, 0], [1, 0], [0.5, 0.5]])
    assert r.offsets.tolist() == [0, 1, 4, 5, 5]
    assert r.rows.tolist() == [3, 0, 2, 3, 0, -1, -1, -1]
    assert r.positions.tolist() == [[1, 4], [-1, -1], [2, -1], [0, 3]]
    over_all = mx.route([[np.log(1), np.log(2), np.log(5)]], 2, False)
    assert over_all.ids.tolist() == [[2, 1]] and np.allclose(over_all.weights, [[5 / 8, 2 / 8]])


def test_combine_by_hand():
    y = np.array([[1.0, 2.0], [10.0, 20.0], [np.nan, np.nan]])
    out, mag = mx.combine(y, np.array([[0, 1], [1, -1], [-1, 7]]), np.array([[0.5, -0.25], [2.0, 9.0], [1.0, 1.0]]), np.ones((3, 2)))
    assert out.tolist() == [[-1.0, -3.0], [21.0, 41.0], [1.0, 1.0]]
    assert mag.tolist() == [[4.0, 7.0], [21.0, 41.0], [1.0, 1.0]]


@pytest.mark.parametrize("renormalize", [True, False])
def test_route_places_every_row_once(renormalize):
    rng = np.random.default_rng(2)
    r = mx.route(rng.standard_normal((50, 7)).round(1), 3, renormalize)
    assert sorted(r.positions.reshape(-1).tolist()) == list(range(150))
    for e in range(7):
        got = r.rows[r.offsets[e]:r.offsets[e + 1]]
        assert got.tolist() == [t for t in range(50) if e in r.ids[t]]
