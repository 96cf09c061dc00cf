"""Pins of oracle/w8_oracle.py: the e4m3 format against its definition, nearest codes by brute force, scales, and log probabilities by
hand-worked cases."""
import numpy as np
import pytest

from oracle import w8_oracle as Q


def test_codes_stand_for_what_the_format_says():
    v = Q.decode_e4m3(np.arange(256))
    assert v[0x7E] == 448 and v[0x38] == 1 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[0xB8] == -1
    assert np.isnan(v[0x7F]) and np.isnan(v[0xFF])
    assert np.all(np.diff(v[:127]) > 0)
    assert v[0x3C] == 1.5 and v[0x07] == 7 * 2.0 ** -9


def test_nearest_code_by_brute_force():
    rng = np.random.default_rng(0)
    levels = Q.decode_e4m3(np.arange(127))
    mids = (levels[1:] + levels[:-1]) / 2
    v = np.concatenate([levels, mids, np.nextafter(mids, 0), np.nextafter(mids, 999), np.exp(rng.uniform(-8, 6, 500)).clip(max=448)])
    for x, c in zip(v, Q.encode_e4m3(v)):
        d = np.abs(levels - x)
        best = np.flatnonzero(d == d.min())
        assert c in best and (len(best) == 1 or c % 2 == 0)
    assert np.array_equal(Q.encode_e4m3(-v), Q.encode_e4m3(v) | 128)


@pytest.mark.parametrize("most,e", [(448.0, 0), (448.5, 1), (896.0, 1), (1.0, -8), (0.875 * 2, -8), (1.76, -7), (0.0, -64), (2.0 ** -60, -64)])
def test_least_scale(most, e):
    assert Q.scale_exponent(most) == e


def test_quantize_shapes_padding_and_bad_blocks():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 136))
    x[1, 130] = np.nan
    codes, scales = Q.quantize_rows(x)
    assert codes.shape == (3, 144) and scales.shape == (3, 4)
    assert np.all(codes[:, 136:] == 0) and np.all(scales[:, 2:] == 127)
    assert np.all(codes[1, 128:136] == 0x7F) and scales[1, 1] == 127 and not np.any((codes[1, :128] & 127) == 127)
    v = Q.values(codes, scales, 1, 136)
    fine = np.isfinite(v)
    assert fine.sum() == 3 * 136 - 8
    assert np.all(np.abs(v - x)[fine] <= np.maximum(np.abs(x)[fine] * 2.0 ** -4, 2.0 ** -10 * np.abs(x[fine]).max()))
    W = rng.standard_normal((136, 264))
    codes, scales = Q.quantize_weight(W)
    assert codes.shape == (264, 144) and scales.shape == (3, 4)
    assert np.all(np.abs(Q.values(codes, scales, 128, 136) - W.T) <= np.maximum(np.abs(W.T) * 2.0 ** -4, 2.0 ** -10 * np.abs(W).max()))


def test_quantize_is_idempotent_and_exact_on_small_integers():
    rng = np.random.default_rng(2)
    x = rng.integers(-7, 8, (5, 256)).astype(float)
    codes, scales = Q.quantize_rows(x)
    assert np.array_equal(Q.values(codes, scales, 1, 256), x)
    again = Q.quantize_rows(Q.values(codes, scales, 1, 256))
    assert np.array_equal(again[0], codes) and np.array_equal(again[1], scales)


def test_product_is_the_sum_of_the_values_products():
    rng = np.random.default_rng(3)
    x, W = rng.standard_normal((2, 136)), rng.standard_normal((136, 8))
    xc, xs = Q.quantize_rows(x)
    wc, wsc = Q.quantize_weight(W)
    y, most = Q.product(wc, wsc, xc, xs, 136)
    a, b = Q.values(xc, xs, 1, 136), Q.values(wc, wsc, 128, 136)
    assert y[1, 3] == pytest.approx(sum(a[1, i] * b[3, i] for i in range(136)), rel=1e-13)
    assert most[1, 3] == pytest.approx(sum(abs(a[1, i] * b[3, i]) for i in range(136)), rel=1e-13)
    assert np.abs(y - x @ W).max() < 0.1 * np.abs(most).max()


def test_logprobs_by_hand():
    z = np.array([[0.0, np.log(3.0), -np.inf, 0.0]])
    logp, entropy, ids, top = Q.logprobs(z, np.array([[1, 2, -1, 4]]), 4)
    assert logp[0, 0] == pytest.approx(np.log(0.6)) and logp[0, 1] == -np.inf and logp[0, 2] == 0 and np.isnan(logp[0, 3])
    assert entropy[0] == pytest.approx(-(0.6 * np.log(0.6) + 0.4 * np.log(0.2)))
    assert ids[0].tolist() == [1, 0, 3, 2]
    assert top[0, :3] == pytest.approx(np.log([0.6, 0.2, 0.2])) and top[0, 3] == -np.inf


def test_logprobs_scale_sure_rows_and_undefined_rows():
    z = np.array([[0.0, np.log(3.0) / 2]])
    assert Q.logprobs(z, np.array([[1]]), 0, 2.0)[0][0, 0] == pytest.approx(np.log(0.75))
    z = np.array([[50.0, 0.0, 0.0]])
    assert Q.logprobs(z, np.array([[0]]), 0)[0][0, 0] == pytest.approx(-2 * np.exp(-50.0), rel=1e-12)
    z = np.array([[-np.inf, -np.inf, -np.inf], [0, np.nan, 1], [0, np.inf, 1]])
    logp, entropy, ids, top = Q.logprobs(z, np.array([[1], [0], [-1]]), 2)
    assert logp[0, 0] == -np.inf and entropy[0] == 0 and ids[0].tolist() == [0, 1]
    assert np.isnan(logp[1, 0]) and np.isnan(entropy[1]) and ids[1].tolist() == [-1, -1] and logp[2, 0] == 0 and np.isnan(top[2]).all()
