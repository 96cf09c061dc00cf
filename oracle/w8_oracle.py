"""Slow CPU fp64 statement of the operators on 8-bit floating-point weights: the format (e4m3 codes, a power-of-two scale for each
block of 128), the product over it, and log probabilities with entropy and top alternatives.  Test infrastructure only; shares no
code with the GPU path."""
from __future__ import annotations

import numpy as np

LEAST = -64                 # exponent of a scale


def decode_e4m3(codes) -> np.ndarray:
    """Values of e4m3 bytes: exponent bias 7, three bits of fraction, 0 = subnormal (multiples of 2^-9), 0x7F and 0xFF NaN."""
    c = np.asarray(codes, dtype=np.int64)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


_LEVELS = decode_e4m3(np.arange(127))


def encode_e4m3(v) -> np.ndarray:
    """Nearest code of finite |v| <= 448, ties to the even code: by search among all 127 magnitudes."""
    v = np.asarray(v, dtype=np.float64)
    a = np.abs(v)
    assert np.all(a <= 448.0)
    hi = np.searchsorted(_LEVELS, a)                      # first level >= a
    lo = np.maximum(hi - 1, 0)
    down, up = a - _LEVELS[lo], _LEVELS[hi] - a
    pick = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    pick = np.where(_LEVELS[hi] == a, hi, pick)
    return (pick + 128 * np.signbit(v)).astype(np.uint8)


def scale_exponent(most: float) -> int:
    """Least e >= LEAST with most <= 448 * 2^e."""
    e = LEAST
    while most > 448.0 * 2.0 ** e:
        e += 1
    return e


def _block(v):
    """Codes and scale byte of one block (any shape)."""
    if not np.all(np.isfinite(v)):
        return np.full(v.shape, 0x7F, np.uint8), 127
    e = scale_exponent(float(np.max(np.abs(v))))
    return encode_e4m3(v / 2.0 ** e), e + 127


def _pitches(d):
    return -(-d // 16) * 16, -(-(-(-d // 128)) // 4) * 4


def quantize(v, rows_of_block: int):
    """v [n, d] -> codes [n, d up to 16] (zeros behind d) and scale bytes [n / rows_of_block up, blocks up to 4] (127 behind the last)."""
    n, d = v.shape
    pitch, spitch = _pitches(d)
    codes = np.zeros((n, pitch), np.uint8)
    scales = np.full((-(-n // rows_of_block), spitch), 127, np.uint8)
    for i in range(scales.shape[0]):
        rows = slice(i * rows_of_block, min(n, (i + 1) * rows_of_block))
        for j in range(-(-d // 128)):
            cols = slice(j * 128, min(d, (j + 1) * 128))
            codes[rows, cols], scales[i, j] = _block(v[rows, cols])
    return codes, scales


def quantize_rows(x):
    return quantize(np.asarray(x, np.float64), 1)


def quantize_weight(W):
    """W [d_in, d_out]."""
    return quantize(np.ascontiguousarray(np.asarray(W, np.float64).T), 128)


def values(codes, scales, rows_of_block: int, d: int) -> np.ndarray:
    n = codes.shape[0]
    unit = 2.0 ** (scales.astype(np.float64) - 127.0)
    unit = np.repeat(np.repeat(unit, rows_of_block, 0)[:n], 128, 1)[:, :d]
    return decode_e4m3(codes[:, :d]) * unit


def normed(x, rms, eps: float):
    x = np.asarray(x, np.float64)
    v = x / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps)
    return v if rms is None else v * np.asarray(rms, np.float64)


def product(w_codes, w_scales, x_codes, x_scales, d_in: int):
    """(x W^T, sum of the products' magnitudes)."""
    w, x = values(w_codes, w_scales, 128, d_in), values(x_codes, x_scales, 1, d_in)
    return x @ w.T, np.abs(x) @ np.abs(w).T


def logprobs(logits, given, n_top: int, scale: float = 1.0):
    """logits [n, V] fp64 -> logp of given [n, g], entropy [n], top ids and log probabilities [n, n_top]."""
    n, V = logits.shape
    logp, entropy = np.zeros(given.shape), np.zeros(n)
    top_id, top_logp = np.zeros((n, n_top), np.int64), np.zeros((n, n_top))
    for r in range(n):
        z = scale * logits[r]
        if np.any(np.isnan(z)) or np.any(z == np.inf):
            p, entropy[r], top_id[r] = np.full(V, np.nan), np.nan, -1
        elif np.all(z == -np.inf):
            p, entropy[r] = np.full(V, -np.inf), 0.0
        else:
            m = z.max()
            first = int(np.argmax(z))
            e = np.exp(z - m)
            rest = np.delete(e, first).sum()                 # the largest apart: log1p keeps a sure row's bits
            p = z - m - np.log1p(rest)
            some = e > 0
            entropy[r] = -(np.exp(p[some]) * p[some]).sum()
        if not np.any(np.isnan(p)):
            top_id[r] = np.argsort(-(logits[r] + 0.0), kind="stable")[:n_top]
        top_logp[r] = p[top_id[r]] if n_top and top_id[r, 0] >= 0 else np.nan
        for i, t in enumerate(given[r]):
            logp[r, i] = 0.0 if t < 0 else np.nan if t >= V else p[t]
    return logp, entropy, top_id, top_logp
