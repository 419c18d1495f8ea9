"""Pins of the cache's oracle: stored values against the quantizers', attention against small sums written out and against
properties of a softmax."""
import numpy as np
import pytest

from oracle import formats as F
from oracle import kv as OK
from oracle import quantize as Q


@pytest.mark.parametrize("fmt,group", [(F.FMT_NVFP4, 16), (F.FMT_INT4, 32), (F.FMT_INT4, 64), (OK.BF16, 0)])
def test_stored_values_are_those_of_rows_alone(fmt, group):
    rng = np.random.default_rng(5)
    x = F.bf16_bits_to_f64(F.f64_to_bf16_bits_rne(rng.standard_normal((3, 2, 64)) * 3))
    T = np.float32(np.abs(x).max() / 2688)
    whole = OK.stored(fmt, group, x, T)
    for i in range(3):
        for h in range(2):
            assert np.array_equal(whole[i, h], OK.stored(fmt, group, x[i, h], T))
    if fmt == OK.BF16:
        assert np.array_equal(whole, x)
    else:
        assert np.abs(whole - x).max() <= np.abs(x).max() / 7
    assert np.array_equal(F.bf16_bits_to_f64(OK.read_back(fmt, group, x, T)).shape, x.shape)


def test_int4_row_by_hand():
    x = np.zeros(32)
    x[:4] = [7.0, -3.5, 1.0, -0.25]                     # s = 1: ties go to the even code
    assert OK.stored(F.FMT_INT4, 32, x)[:4].tolist() == [7.0, -4.0, 1.0, 0.0]
    assert Q.quantize_int(x[None], 32, F.FMT_INT4).scale.tolist() == [[1.0]]


def test_attended_tokens():
    assert list(OK.attended(5)) == [0, 1, 2, 3, 4]
    assert list(OK.attended(5, 2)) == [3, 4] and list(OK.attended(1, 2)) == [0]
    assert list(OK.attended(0)) == [] and list(OK.attended(-3, 2)) == []


def test_attention_by_hand():
    q = np.array([[1.0, 0.0], [0.0, 2.0]])
    k = np.array([[[np.log(3.0), 0.0]], [[0.0, 0.0]]])
    v = np.array([[[4.0, 0.0]], [[0.0, -8.0]]])
    out, lse, mag, top = OK.attention(q, k, v, 1.0)
    assert np.allclose(out, [[3.0, -2.0], [2.0, -4.0]], rtol=1e-15)
    assert np.allclose(lse, [np.log(4.0), np.log(2.0)], rtol=1e-15)
    assert np.allclose(mag, [[3.0, 2.0], [2.0, 4.0]], rtol=1e-15)
    assert np.allclose(top, [np.log(3.0), 0.0], rtol=1e-15)


def test_attention_over_parts_joins_by_lse():
    rng = np.random.default_rng(6)
    q, k, v = rng.standard_normal((4, 8)), rng.standard_normal((9, 2, 8)), rng.standard_normal((9, 2, 8))
    out, lse, _, _ = OK.attention(q, k, v, 0.3)
    a, la, _, _ = OK.attention(q, k[:4], v[:4], 0.3)
    b, lb, _, _ = OK.attention(q, k[4:], v[4:], 0.3)
    w = np.exp(np.stack([la, lb]) - lse)
    assert np.allclose(w.sum(0), 1.0, rtol=1e-13)
    assert np.allclose(w[0][:, None] * a + w[1][:, None] * b, out, rtol=1e-12)


def test_nothing_attended():
    out, lse, _, _ = OK.attention(np.ones((2, 4)), np.zeros((0, 1, 4)), np.zeros((0, 1, 4)), 1.0)
    assert np.all(out == 0) and np.all(lse == -np.inf)
