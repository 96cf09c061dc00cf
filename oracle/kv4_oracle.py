"""Slow CPU statement of the 4-bit key/value cache (test infrastructure only): the byte format token by token, rotary
positions and quantisation, attention in fp64, and the bookkeeping of pages as plain loops over plain lists.

A `Cache` mirrors the device state: data [layers, pages, heads, blocks, 34 D] bytes, table, length, refs.
"""
from __future__ import annotations

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
EXPONENTS = {"f16": (-23, 13), "bf16": (-100, 125)}
NAN_SCALE = 255


class Cache:
    def __init__(self, n_layers, n_pages, page_tokens, n_slots, max_pages, n_kv_heads, head_dim, dtype):
        self.n_layers, self.n_pages, self.page_tokens = n_layers, n_pages, page_tokens
        self.n_slots, self.max_pages, self.n_kv_heads, self.head_dim, self.dtype = n_slots, max_pages, n_kv_heads, head_dim, dtype
        self.data = np.zeros((n_layers, n_pages, n_kv_heads, page_tokens // 32, 34 * head_dim), np.uint8)
        self.refs = np.zeros(n_pages, np.int32)
        self.table = np.full((n_slots, max_pages), -1, np.int32)
        self.length = np.zeros(n_slots, np.int32)

    def block(self, layer, slot, t, head):
        """The bytes of the block that holds token t of a slot, or None."""
        p = t // self.page_tokens
        page = self.table[slot, p] if 0 <= p < self.max_pages else -1
        if not 0 <= page < self.n_pages:
            return None
        return self.data[layer, page, head, t % self.page_tokens // 32]


# ---- the format -----------------------------------------------------------------------------------------

def _lane_byte(D, half, lane, b):
    W = min(16, D // 8)
    return half * 8 * D + b // W * 64 * W + lane * W + b % W


def code_place(D, t, i, which):
    """(byte, high nibble?) of value i of token t of a block, K (0) or V (1)."""
    m = t % 16
    if which == 0:
        return _lane_byte(D, t // 16, i // (D // 4) * 16 + m, i % (D // 4) // 2), i % 2
    return 16 * D + _lane_byte(D, t // 16, m // 4 * 16 + i // (D // 16), m % 4 * (D // 32) + i % (D // 16) // 2), i % 2


def scale_place(D, t, g, which):
    m = t % 16
    if which == 0:
        return 32 * D + t // 16 * (D // 2) + 16 * g + m
    return 33 * D + t // 16 * (D // 2) + (m // 4 * (D // 32) + g) * 4 + m % 4


_PLACES: dict = {}


def _places(D, which):
    """Index arrays of a block: bytes and shifts [32, D], scale bytes [32, D / 32]."""
    if (D, which) not in _PLACES:
        at = np.array([[code_place(D, t, i, which) for i in range(D)] for t in range(32)])
        sc = np.array([[scale_place(D, t, g, which) for g in range(D // 32)] for t in range(32)])
        _PLACES[D, which] = at[..., 0], 4 * at[..., 1], sc
    return _PLACES[D, which]


def read_block(block, D, which):
    """The 32 tokens' values [32, D] that a block's bytes stand for."""
    at, shift, sc = _places(D, which)
    code = block[at] >> shift & 15
    scale = block[sc].astype(np.int64)
    unit = np.where(scale == NAN_SCALE, np.nan, 2.0 ** (scale - 127.0))
    v = np.where(code >= 8, -1.0, 1.0) * LEVELS[code & 7]
    with np.errstate(invalid="ignore"):
        return v * np.repeat(unit, 32, axis=1)


def write_token(block, D, t, which, codes, scales):
    at, shift, sc = _places(D, which)
    for i in range(D):
        b, s = at[t, i], shift[t, i]
        block[b] = block[b] & (0xF0 >> s) | codes[i] << s
    block[sc[t]] = scales


def quantise(x, dtype):
    """x [D] (fp64 or fp32, taken as exact) -> codes [D], scale bytes [D / 32]: nearest code, ties to the even one."""
    lowest, highest = EXPONENTS[dtype]
    codes, scales = np.zeros(len(x), np.uint8), np.zeros(len(x) // 32, np.uint8)
    for g in range(len(x) // 32):
        v = np.asarray(x[32 * g:32 * g + 32], np.float64)
        sign = np.signbit(v).astype(np.uint8) << 3
        if not np.isfinite(v).all():
            scales[g] = NAN_SCALE
            codes[32 * g:32 * g + 32] = sign
            continue
        top = np.abs(v).max()
        e = lowest
        if top > 0:
            e = int(np.frexp(top)[1]) - 1 - 2
            if top > 7 * 2.0 ** e:
                e += 1
            e = min(max(e, lowest), highest)
        away = np.abs(np.abs(v)[:, None] / 2.0 ** e - LEVELS[None, :])
        for k in range(32):
            best = [c for c in range(8) if away[k, c] == away[k].min()]
            codes[32 * g + k] = (best[0] if len(best) == 1 else next(c for c in best if c % 2 == 0)) | sign[k]
        scales[g] = e + 127
    return codes, scales


def stored(x, dtype):
    """The values that the format holds for x [D]."""
    codes, scales = quantise(x, dtype)
    unit = np.where(scales == NAN_SCALE, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    with np.errstate(invalid="ignore"):
        return np.where(codes >= 8, -1.0, 1.0) * LEVELS[codes & 7] * np.repeat(unit, 32)


# ---- rotary positions ------------------------------------------------------------------------------------

def rotate(x, table, positions, axis_pairs, interleaved, kind=np.float64):
    """One head x [D] turned by the table's rows: positions [n_axes].  kind float32: every product and sum rounded."""
    x = np.asarray(x, kind).copy()
    rot = table.shape[1]
    axis = np.repeat(np.arange(len(axis_pairs)), axis_pairs) if axis_pairs else np.zeros(rot // 2, int)
    y = x.copy()
    for j in range(rot // 2):
        p = positions[axis[j]]
        c, s = (kind(table[p, j]), kind(table[p, j + rot // 2])) if 0 <= p < table.shape[0] else (kind(np.nan),) * 2
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
        with np.errstate(invalid="ignore", over="ignore"):
            y[a] = x[a] * c - x[b] * s
            y[b] = x[b] * c + x[a] * s
    return y


# ---- attention -------------------------------------------------------------------------------------------

def keys_values(C: Cache, layer, slot, n, head):
    """Values of the first n tokens and whether each has a page."""
    D = C.head_dim
    k, v, have = np.zeros((n, D)), np.zeros((n, D)), np.zeros(n, bool)
    for t0 in range(0, n, 32):
        block = C.block(layer, slot, t0, head)
        if block is not None:
            m = min(32, n - t0)
            k[t0:t0 + m], v[t0:t0 + m], have[t0:t0 + m] = read_block(block, D, 0)[:m], read_block(block, D, 1)[:m], True
    return k, v, have


def attention_row(q, k, v, seen, scale):
    """One query q [D] over the seen tokens: output and what its tolerance needs, the same average of magnitudes."""
    if not seen.any():
        return np.zeros(len(q)), np.zeros(len(q)), 0.0, 0.0
    s = (k[seen] @ q) * scale
    size = float((np.abs(k[seen]) @ np.abs(q)).max() * abs(scale))
    with np.errstate(invalid="ignore"):
        w = np.exp(s - s.max())
        return w @ v[seen] / w.sum(), w @ np.abs(v[seen]) / w.sum(), size, float(np.abs(s - s.max()).max())


# ---- pages -----------------------------------------------------------------------------------------------

def pages_of(n, page_tokens):
    return -(-n // page_tokens)


def trim(C: Cache, slots, keep=None):
    for i, s in enumerate(slots):
        if not 0 <= s < C.n_slots:
            continue
        kept = min(int(C.length[s]), 0 if keep is None else max(0, int(keep[i])))
        for p in range(pages_of(kept, C.page_tokens), pages_of(int(C.length[s]), C.page_tokens)):
            if C.table[s, p] >= 0:
                C.refs[C.table[s, p]] -= 1
            C.table[s, p] = -1
        C.length[s] = kept


def fork(C: Cache, src, dst):
    """0, or -1 with nothing changed where the list is not in order."""
    if any(not 0 <= s < C.n_slots for s in list(src) + list(dst)) or len(set(dst)) != len(dst) or set(src) & set(dst):
        return -1
    if any(C.length[d] != 0 for d in dst):
        return -1
    for s, d in zip(src, dst):
        C.table[d], C.length[d] = C.table[s], C.length[s]
        for p in C.table[s]:
            if p >= 0:
                C.refs[p] += 1
    return 0


def grow(C: Cache, slots, counts):
    """0, the number of pages that are missing, or -1 where the list is not in order: then nothing is changed."""
    P = C.page_tokens
    if any(not 0 <= s < C.n_slots for s in slots) or len(set(slots)) != len(slots) or any(c < 0 for c in counts):
        return -1
    if any(pages_of(int(C.length[s]) + c, P) > C.max_pages for s, c in zip(slots, counts)):
        return -1
    shared = {}                       # page -> entries that would write into it
    for i, (s, c) in enumerate(zip(slots, counts)):
        n = int(C.length[s])
        if c > 0 and n % P and C.table[s, n // P] >= 0 and C.refs[C.table[s, n // P]] > 1:
            shared.setdefault(int(C.table[s, n // P]), []).append(i)
    copies = {i for page, entries in shared.items() for i in entries}
    for page, entries in shared.items():
        if len(entries) == C.refs[page]:
            copies.discard(entries[-1])       # the last of the list keeps it
    free = [p for p in range(C.n_pages) if C.refs[p] == 0]
    need = sum(pages_of(int(C.length[s]) + c, P) - pages_of(int(C.length[s]), P) + (i in copies) for i, (s, c) in enumerate(zip(slots, counts)))
    if need > len(free):
        return need - len(free)
    for i, (s, c) in enumerate(zip(slots, counts)):
        n = int(C.length[s])
        if i in copies:
            old, new = C.table[s, n // P], free.pop(0)
            C.data[:, new] = C.data[:, old]
            C.refs[old] -= 1
            C.refs[new] = 1
            C.table[s, n // P] = new
        for p in range(pages_of(n, P), pages_of(n + c, P)):
            C.table[s, p] = free.pop(0)
            C.refs[C.table[s, p]] = 1
        C.length[s] = n + c
    return 0


def compact(C: Cache):
    """Live pages to the lowest ids; returns their number."""
    live = [p for p in range(C.n_pages) if C.refs[p] > 0]
    n = len(live)
    to = {}
    holes = [p for p in range(n) if C.refs[p] == 0]
    for old, new in zip([p for p in live if p >= n], holes):
        C.data[:, new] = C.data[:, old]
        C.refs[new], C.refs[old] = C.refs[old], 0
        to[old] = new
    for s in range(C.n_slots):
        for p in range(C.max_pages):
            C.table[s, p] = to.get(int(C.table[s, p]), C.table[s, p])
    return n
