"""Shared by the tests of the 4-bit key/value cache: an oracle cache with random contents and its twin on the GPU, and the
tolerance of an attention output."""
import numpy as np
import torch

from oracle import kv4_oracle as K
from oracle import larosa_oracle as O
from tests.gpu_util import to_bits, to_dev  # noqa: F401

HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def random_cache(rng, lengths, page_tokens, n_kv_heads, head_dim, dtype, n_layers=1, spare_slots=1, spare_pages=3, headroom=0,
                 wild=True, spread=2):
    """Sequences of the given lengths in random pages of random codes.  Scales within `spread` powers of two around 1; whatever lies
    past a sequence's end holds any byte (with wild), NaN scales among them.  headroom: tokens that the tables have room for
    beyond the longest sequence."""
    need = [K.pages_of(n, page_tokens) for n in lengths]
    max_pages = max(1, max(K.pages_of(n + headroom, page_tokens) for n in lengths))
    C = K.Cache(n_layers, sum(need) + spare_pages, page_tokens, len(lengths) + spare_slots, max_pages, n_kv_heads, head_dim, dtype)
    C.data[:] = rng.integers(0, 256, C.data.shape, dtype=np.uint8)
    codes = 32 * head_dim
    if not wild:
        C.data[..., codes:] = 127
    ids = rng.permutation(C.n_pages)
    slots = rng.permutation(C.n_slots)[:len(lengths)]
    at = 0
    for s, n, p in zip(slots, lengths, need):
        C.table[s, :p] = ids[at:at + p]
        C.refs[ids[at:at + p]] = 1
        C.length[s] = n
        at += p
        if n:
            t = np.arange(n)
            block, u, m = t % page_tokens // 32, t % 32 // 16, t % 16
            pages = C.table[s, t // page_tokens]
            for g in range(head_dim // 32):
                for off in (codes + u * (head_dim // 2) + 16 * g + m,
                            codes + head_dim + u * (head_dim // 2) + (m // 4 * (head_dim // 32) + g) * 4 + m % 4):
                    for layer in range(n_layers):
                        for h in range(n_kv_heads):
                            C.data[layer, pages, h, block, off] = 127 - 2 + rng.integers(-spread, spread + 1, n)
    return C, slots


def device_cache(C, device="cuda:0"):
    from paper_2507_01299_amd import api
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)       # noqa: E731
    return api.KvCache(C.n_layers, C.n_pages, C.page_tokens, C.n_slots, C.max_pages, C.n_kv_heads, C.head_dim, C.dtype,
                       data=dev(C.data.reshape(-1)), refs=dev(C.refs), table=dev(C.table), length=dev(C.length))


def same_state(cache, C, data=True):
    assert np.array_equal(cache.table.cpu().numpy(), C.table), "table"
    assert np.array_equal(cache.length.cpu().numpy(), C.length), "length"
    assert np.array_equal(cache.refs.cpu().numpy(), C.refs), "refs"
    if data:
        assert np.array_equal(cache.data.cpu().numpy().reshape(C.data.shape), C.data), "data"


def int32(values, device="cuda:0"):
    return None if values is None else torch.tensor([int(v) for v in values], dtype=torch.int32, device=device)


def rows_of(starts, n_seq, i, max_new):
    a, b = (i, i + 1) if starts is None else (starts[i], starts[i + 1])
    return a, b - a, range(a, min(b, a + max_new))


def attention_want(C, layer, slots, starts, q, n_heads, scale, window, max_new):
    """{row: (fp64 output [n_heads, D], tolerance [n_heads, D])}.

    A weight is rounded to 16 bits (u relative), the store rounds once (u of the output).  A logit of D products added in fp32 is
    off by at most D 2^-24 of the sum of their magnitudes, its scaling and the difference from the maximum by 3 2^-24 of its size; a
    weight by as much relative, plus 2^-22 for the exponential.  The sums over n tokens and their rescalings add 2 n 2^-24
    of the average of magnitudes.  Weights, numerator and denominator can each be off by these: twice.  A weight below
    2^-126, the smallest normal number of fp32 and bf16, may count as zero: n of them times the largest value."""
    D, u = C.head_dim, HALF_STEP[C.dtype]
    want = {}
    group = n_heads // C.n_kv_heads
    for i, slot in enumerate(slots):
        _, n_new, rows = rows_of(starts, len(slots), i, max_new)
        real = 0 <= slot < C.n_slots
        n = int(C.length[slot]) if real else 0
        for h in range(C.n_kv_heads):
            k, v, have = K.keys_values(C, layer, slot, n, h) if real else (np.zeros((0, D)),) * 2 + (np.zeros(0, bool),)
            for j, row in enumerate(rows):
                place = n - n_new + j
                t = np.arange(n)
                seen = have & (t <= place) & ((t > place - window) if window else True)
                for g in range(group):
                    hq = h * group + g
                    out, mag, size, spread = K.attention_row(q[row, hq], k, v, seen, scale)
                    logit = (D * size + 3 * (size + spread)) * 2.0 ** -24 + 2.0 ** -22
                    tol = u * np.abs(out) * 1.01 + mag * (u + 2 * (logit + 2 * (n + 8) * 2.0 ** -24))
                    tol = tol + n * 2.0 ** -126 * np.abs(np.nan_to_num(v)).max(initial=0.0)
                    o, e = want.setdefault(row, (np.zeros((n_heads, D)), np.zeros((n_heads, D))))
                    o[hq], e[hq] = out, tol + 2.0 ** -25 * (C.dtype == "f16")
    return want


def random_rows(rng, n_rows, width, dtype, size=1.0):
    return O.encode16(rng.standard_normal((n_rows, width)) * size, dtype)
