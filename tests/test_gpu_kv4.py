"""The 4-bit key/value cache on the GPU against its CPU statement: append (rotary positions, quantisation) bit for bit, attention
against fp64 softmax with a derived tolerance."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as K
from oracle import larosa_oracle as O
from tests import kv4_util as U

pytestmark = pytest.mark.gpu


def run_attention(C, slots, starts, q_bits, n_heads, window=0, scale=None, max_new=1, layer=0, ld_extra=0, max_len=0, n_rows=None):
    from paper_2507_01299_amd import api
    cache = U.device_cache(C)
    D, rows = C.head_dim, q_bits.shape[0]
    qd = torch.full((rows, n_heads * D + ld_extra), float("nan"), dtype=api.torch_dtype(C.dtype), device="cuda:0")
    qd[:, :n_heads * D] = U.to_dev(q_bits, C.dtype)
    out = torch.full((rows, n_heads * D + 2 * ld_extra), 77.0, dtype=api.torch_dtype(C.dtype), device="cuda:0")
    batch = api.KvBatch(U.int32(slots), rows if n_rows is None else n_rows, starts=U.int32(starts), max_new=max_new)
    ws = api.kv4_attention_workspace(cache, batch, n_heads, max_len)
    api.kv4_attention(cache, layer, batch, qd, n_heads, out, ws, scale=scale, window=window, max_len=max_len)
    torch.cuda.synchronize()
    got = O.decode16(U.to_bits(out[:, :n_heads * D].contiguous()), C.dtype).reshape(rows, n_heads, D)
    assert (out[:, n_heads * D:] == 77.0).all()
    return got, cache


def check_attention(C, slots, starts, q_bits, n_heads, window=0, scale=None, max_new=1, layer=0, **kw):
    scale = C.head_dim ** -0.5 if scale is None else scale
    got, _ = run_attention(C, slots, starts, q_bits, n_heads, window=window, scale=scale, max_new=max_new, layer=layer, **kw)
    q = O.decode16(q_bits, C.dtype).reshape(q_bits.shape[0], n_heads, C.head_dim)
    want = U.attention_want(C, layer, slots, starts, q, n_heads, scale, window, max_new)
    for row in range(q_bits.shape[0]):
        if row not in want:
            assert (got[row] == 77.0).all(), f"row {row} of no sequence was written"
            continue
        o, tol = want[row]
        assert np.array_equal(np.isnan(got[row]), np.isnan(o)), f"row {row}: NaN"
        ok = ~np.isnan(o)
        err = np.abs(got[row] - o)[ok]
        assert (err <= tol[ok]).all(), f"row {row}: error {err.max():.3e}, {(err / tol[ok]).max():.2f} of the tolerance"
    return got


CASES = [
    # dtype, head_dim, heads, kv heads, page tokens, lengths
    ("f16", 128, 4, 4, 32, [1, 2, 15, 16, 17, 31, 32, 33]),
    ("bf16", 128, 8, 2, 64, [63, 64, 65, 127, 128, 129]),
    ("f16", 64, 6, 2, 32, [5, 100, 257]),
    ("bf16", 64, 16, 1, 128, [300, 1]),
    ("f16", 256, 4, 1, 64, [90, 33]),
    ("bf16", 256, 3, 3, 256, [257, 40]),
    ("bf16", 128, 34, 2, 32, [200, 64]),          # 17 rows: a second tile of one row
    ("f16", 128, 2, 1, 32, [3000, 1100, 5]),
    ("bf16", 128, 1, 1, 128, [5001]),
]


@pytest.mark.parametrize("dtype,D,heads,kv,P,lengths", CASES)
def test_attention_one_token(gpu_device, dtype, D, heads, kv, P, lengths):
    rng = np.random.default_rng(len(lengths) * D + heads)
    C, slots = U.random_cache(rng, lengths, P, kv, D, dtype)
    check_attention(C, slots, None, U.random_rows(rng, len(lengths), heads * D, dtype), heads)


@pytest.mark.parametrize("dtype,D,heads,kv,P,window", [("f16", 128, 8, 2, 32, 0), ("bf16", 64, 4, 4, 64, 40), ("bf16", 128, 10, 2, 32, 1),
                                                       ("f16", 256, 4, 2, 32, 64), ("f16", 128, 32, 1, 64, 33)])
def test_attention_several_new_tokens(gpu_device, dtype, D, heads, kv, P, window):
    rng = np.random.default_rng(D + heads + window)
    lengths, news = [70, 9, 33, 400, 20], [5, 9, 1, 7, 3]
    C, slots = U.random_cache(rng, lengths, P, kv, D, dtype, n_layers=2)
    starts = np.concatenate([[0], np.cumsum(news)])
    q = U.random_rows(rng, int(starts[-1]) + 2, heads * D, dtype)      # two rows behind the last sequence
    check_attention(C, slots, starts, q, heads, window=window, max_new=9, layer=1, ld_extra=8)


WIDE = 256000         # tokens that the page tables have room for: enough work by the plan for tiles of 32 rows and 250 splits


@pytest.mark.parametrize("dtype,D,heads,kv,window", [("f16", 128, 12, 4, 0), ("bf16", 64, 32, 2, 0), ("bf16", 128, 8, 2, 37),
                                                     ("f16", 64, 20, 4, 300)])
def test_attention_tiles_of_32_rows(gpu_device, dtype, D, heads, kv, window):
    rng = np.random.default_rng(D + heads + window)
    lengths, news = [170, 9, 1100, 40, 0], [41, 9, 33, 17, 6]
    C, slots = U.random_cache(rng, lengths, 256, kv, D, dtype, headroom=WIDE)
    starts = np.concatenate([[0], np.cumsum(news)])
    q = U.random_rows(rng, int(starts[-1]) + 1, heads * D, dtype)
    wide = check_attention(C, slots, starts, q, heads, window=window, max_new=41)
    C.block(0, slots[0], 160, 0)[K.scale_place(D, 160 % 32, 1, 1)] = K.NAN_SCALE         # tokens 160 (V) and 165 (K) of the first
    C.block(0, slots[0], 165, 0)[K.scale_place(D, 165 % 32, 0, 0)] = K.NAN_SCALE
    got = check_attention(C, slots, starts, q, heads, window=window, max_new=41)
    assert np.array_equal(got[41:], wide[41:]) and np.array_equal(got[:31], wide[:31]) and np.isnan(got[31:41]).any((1, 2)).all()


def test_attention_past_4_gib(gpu_device):
    """Pages whose bytes lie past 32-bit offsets: the same output and the same stored bytes as low ones."""
    from paper_2507_01299_amd import api
    rng = np.random.default_rng(17)
    C, slots = U.random_cache(rng, [500, 300], 256, 8, 128, "bf16")
    q = U.random_rows(rng, 2, (16 + 16) * 128, "bf16")
    page = C.data[0, 0].nbytes
    n_pages = (5 << 30) // page
    far = np.where(C.table >= 0, n_pages - 1 - C.table, -1)
    big = api.KvCache(1, n_pages, 256, C.n_slots, C.max_pages, 8, 128, "bf16")
    big.table.copy_(torch.from_numpy(far))
    big.length.copy_(torch.from_numpy(C.length))
    pages = big.data[:n_pages * page].view(n_pages, page)
    ids = C.table[C.table >= 0]
    for p in ids:
        pages[n_pages - 1 - int(p)] = torch.from_numpy(C.data[0, p].reshape(-1)).to("cuda:0")
    small = U.device_cache(C)
    outs = []
    for cache in (small, big):
        batch = api.KvBatch(U.int32(slots), 2)
        qkv = U.to_dev(q, "bf16")
        turned, out = torch.zeros_like(qkv), torch.zeros(2, 16 * 128, dtype=qkv.dtype, device="cuda:0")
        api.kv4_append(cache, 0, batch, qkv, 16, out=turned)
        api.kv4_attention(cache, 0, batch, turned, 16, out, api.kv4_attention_workspace(cache, batch, 16))
        torch.cuda.synchronize()
        outs.append((turned.view(torch.int16), out.view(torch.int16)))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    low = small.data.view(-1, page)
    for p in ids:
        assert torch.equal(low[int(p)], pages[n_pages - 1 - int(p)])
    # and copied from there
    api.kv4_copy_pages(big, U.int32([n_pages - 1 - int(ids[0])]), U.int32([n_pages - 1 - C.n_pages]))
    torch.cuda.synchronize()
    assert torch.equal(pages[n_pages - 1 - C.n_pages], low[int(ids[0])])


def test_attention_prompt(gpu_device):
    """A whole prompt's rows against its own keys: row 0 sees one token."""
    rng = np.random.default_rng(11)
    C, slots = U.random_cache(rng, [150], 32, 1, 128, "bf16")
    check_attention(C, slots, [0, 150], U.random_rows(rng, 150, 2 * 128, "bf16"), 2, max_new=150)


def test_attention_rows_that_see_nothing(gpu_device):
    """Empty sequences, padding, more new tokens than tokens, missing pages, more rows than a batch allows."""
    rng = np.random.default_rng(12)
    D, heads = 128, 4
    C, slots = U.random_cache(rng, [0, 40, 70, 100, 64, 33], 32, 2, D, "f16", headroom=32)
    slots = slots.tolist()
    C.table[slots[2], 0] = -1                     # a dropped page: seen as if masked
    C.table[slots[3], :] = C.n_pages + 5          # ids outside the pool
    C.table[slots[5], 1] = -7
    slots[1] = -1
    starts = [0, 1, 2, 4, 6, 11, 75, 75]
    slots.append(C.n_slots)
    q = U.random_rows(rng, 80, heads * D, "f16")
    got = check_attention(C, slots, starts, q, heads, max_new=70)
    assert not got[0].any() and not got[1].any() and not got[4:6].any()
    assert not got[11:42].any() and got[42].any()      # 64 new rows of a sequence of 33
    check_attention(C, slots, starts, q, heads, max_new=3)
    # rows outside the buffer are not touched whatever `starts` says
    got, _ = run_attention(C, slots[:2], [0, 1, 2], q[:4], heads, max_new=2, n_rows=1)
    assert not got[0].any() and (got[1:] == 77.0).all()
    got, _ = run_attention(C, slots[4:6], [-2, 1, 900], q[:4], heads, max_new=900)
    assert (got[0] != 77.0).any()


def test_attention_window_with_dropped_pages(gpu_device):
    """A sliding window never looks at the pages it has left behind."""
    rng = np.random.default_rng(13)
    C, slots = U.random_cache(rng, [500], 32, 2, 64, "bf16")
    q = U.random_rows(rng, 1, 4 * 64, "bf16")
    want = check_attention(C, slots, None, q, 4, window=100)
    C.table[slots[0], :12] = -1                   # tokens 0 .. 383; the window starts at 400
    assert np.array_equal(check_attention(C, slots, None, q, 4, window=100), want)


@pytest.mark.parametrize("dtype,D", [("f16", 128), ("bf16", 64), ("bf16", 256)])
def test_attention_nan_reaches_the_rows_that_see_it_and_no_other(gpu_device, dtype, D):
    rng = np.random.default_rng(14)
    heads = 2
    C, slots = U.random_cache(rng, [45, 45, 45], 32, 1, D, dtype)
    for i, which in ((0, 0), (1, 1)):             # token 43 of sequences 0 (K) and 1 (V): the last group is NaN
        C.block(0, slots[i], 43, 0)[K.scale_place(D, 43 % 32, D // 32 - 1, which)] = K.NAN_SCALE
    q = U.random_rows(rng, 9, heads * D, dtype)
    got = check_attention(C, slots, [0, 3, 6, 9], q, heads, max_new=3)
    assert not np.isnan(got[0]).any() and np.isnan(got[1:3]).all()
    assert not np.isnan(got[3]).any() and np.isnan(got[4:6, :, -32:]).all() and not np.isnan(got[4:6, :, :-32]).any()
    assert not np.isnan(got[6:]).any()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attention_scales_from_smallest_to_largest(gpu_device, dtype):
    """Values of the smallest to the largest powers of two: the codes' conversion and the sums keep them (below what 40 of them
    add up to in fp32)."""
    rng = np.random.default_rng(15)
    lowest, highest = K.EXPONENTS[dtype]
    for e in (lowest, lowest + 5, 0, highest - 12, min(highest, 115)):
        C, slots = U.random_cache(rng, [40], 32, 1, 128, dtype, spread=0)
        blocks = C.data[:, C.table[slots[0]], :, :, 33 * 128:]
        blocks[blocks == 125] = e + 127
        C.data[:, C.table[slots[0]], :, :, 33 * 128:] = blocks
        print(dtype, "2 **", e, flush=True)
        check_attention(C, slots, None, U.random_rows(rng, 1, 2 * 128, dtype), 2)


def test_attention_extreme_logits(gpu_device):
    """One key far above the others, all equal, and differences that underflow."""
    rng = np.random.default_rng(16)
    C, slots = U.random_cache(rng, [700, 700], 64, 1, 64, "bf16")
    q = U.random_rows(rng, 2, 64, "bf16", size=30.0)
    check_attention(C, slots, None, q, 1, scale=1.0)
    check_attention(C, slots, None, q, 1, scale=0.0)
    check_attention(C, slots, None, q, 1, scale=-1.0)


def chosen_tokens(rng, dtype, keys, values, page=64):
    """One sequence whose keys are keys[t] in their first value and zero elsewhere, whose values are values[t]: a logit is
    then the query's first value times keys[t] times the scale."""
    n, D = values.shape
    C, slots = U.random_cache(rng, [n], page, 1, D, dtype)
    quantised = {}
    for t in range(n):
        block = C.block(0, slots[0], t, 0)
        k = np.zeros(D)
        k[0] = keys[t]
        for which, x in ((0, k), (1, values[t])):
            if x.tobytes() not in quantised:
                quantised[x.tobytes()] = K.quantise(x, dtype)
            codes, scales = quantised[x.tobytes()]
            at, _, sc = K._places(D, which)           # two neighbouring values to a byte
            block[at[t % 32, ::2]] = codes[::2] | codes[1::2] << 4
            block[sc[t % 32]] = scales
    return C, slots


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,gap", [(700, 8.1), (700, 11.2), (700, 13.3), (700, 14.2), (3000, 12.4), (3000, 14.0), (3000, 14.5)])
def test_attention_many_small_weights_behind_a_large_one(gpu_device, dtype, n, gap):
    """The first token's logit lies `gap` above all others' (weights down to 2^-20.9 of its own), and its value is zero: the output
    is made of the small weights alone, each of which keeps its half step (the tolerance knows no floor of the weights)."""
    rng = np.random.default_rng(18)
    D = 64
    keys, values = np.zeros(n), np.tile(rng.choice(K.LEVELS[1:], D) * 64.0, (n, 1))
    keys[0], values[0] = 4.0, 0.0
    C, slots = chosen_tokens(rng, dtype, keys, values)
    q = rng.standard_normal((1, 2 * D))
    q[0, 0] = q[0, D] = 1.0
    got = check_attention(C, slots, None, O.encode16(q, dtype), 2, scale=gap / 4)
    assert got.any()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n", [700, 4000])
def test_attention_weights_that_round_alike(gpu_device, dtype, n):
    """The first 128 tokens' logits are zero (every wave's reference), all others' weights just below the middle between two
    neighbouring 16-bit numbers, and all values equal: their average is that value again, to the bit."""
    rng = np.random.default_rng(19)
    D = 64
    step = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -10
    keys = np.where(np.arange(n) < 128, 0.0, 1.0)
    values = np.tile(rng.choice(K.LEVELS[1:], D), (n, 1))
    C, slots = chosen_tokens(rng, dtype, keys, values)
    q = np.zeros((1, D))
    q[0, 0] = 1.0
    for octaves in (0, 2):
        scale = np.log(2.0 ** octaves * (1 + 0.495 * step))
        got = check_attention(C, slots, None, O.encode16(q, dtype), 1, scale=scale)
        assert np.array_equal(got[0, 0], values[0])


def test_attention_extreme_logits_f16(gpu_device):
    """As for bf16: differences that underflow, the whole range of f16's weights."""
    rng = np.random.default_rng(26)
    C, slots = U.random_cache(rng, [700, 700], 64, 1, 64, "f16")
    q = U.random_rows(rng, 2, 64, "f16", size=30.0)
    for scale in (1.0, 0.0, -1.0):
        check_attention(C, slots, None, q, 1, scale=scale)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("scale", [1.0, 30.0, 700.0, 2.0e4, 1.0e6])
def test_attention_logits_beyond_what_fp32_tells_apart(gpu_device, dtype, scale):
    """Logits up to 10^11, where fp32's neighbours lie further apart than any weight reaches: the keys that lead share the output, and no
    weight leaves its type's range."""
    rng = np.random.default_rng(29)
    n, D = 700, 64
    keys = rng.choice([0.5, 1.0, 2.0, 3.0], n)
    leads = [5, 40, 41, 300, 699]
    keys[leads] = 4.0
    values = rng.choice(K.LEVELS[1:], (n, D))
    C, slots = chosen_tokens(rng, dtype, keys, values)
    for q0 in (1000.0, 1001.0, 30016.0, 60000.0):
        q = np.zeros((1, D))
        q[0, 0] = q0
        got, _ = run_attention(C, slots, None, O.encode16(q, dtype), 1, scale=scale)
        # (q0 scale is at least 1000 between the leading keys and the next: weights of zero)
        k, v, have = K.keys_values(C, 0, slots[0], n, 0)
        want = v[leads].mean(0)
        assert have.all() and (np.abs(got[0, 0] - want) <= U.HALF_STEP[dtype] * np.abs(want) * 1.01).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attention_infinite_queries(gpu_device, dtype):
    """Logits of -infinity alone: zeros, whole and split; +infinity among them: NaN; a finite query beside them stays finite."""
    rng = np.random.default_rng(30)
    for n in (20, 1500):
        keys, values = np.ones(n), rng.choice(K.LEVELS[1:], (n, 64))
        C, slots = chosen_tokens(rng, dtype, keys, values)
        q = np.zeros((1, 3, 64))
        q[0, :, 0] = -np.inf, np.inf, 0.5
        got, _ = run_attention(C, slots, None, O.encode16(q.reshape(1, -1), dtype), 3)
        assert not got[0, 0].any() and np.isnan(got[0, 1]).all() and np.isfinite(got[0, 2]).all()
        keys[3:] = -1.0                               # logits of +infinity behind the first three's -infinity, and the reverse
        C, slots = chosen_tokens(rng, dtype, keys, values)
        got, _ = run_attention(C, slots, None, O.encode16(q.reshape(1, -1), dtype), 3)
        assert np.isnan(got[0, :2]).all() and np.isfinite(got[0, 2]).all()


# ---- every way in which a call is divided: tiles of 16 and 32 rows, alone and several, whole and split, with and without a window ----

def plan_of(C, slots, starts, n_rows, n_heads, max_new=1, window=0, max_len=0):
    from paper_2507_01299_amd import api
    batch = api.KvBatch(U.int32(slots), n_rows, starts=U.int32(starts), max_new=max_new)
    return api.kv4_attention_plan(U.device_cache(C), batch, n_heads, window, max_len)


def real_splits(C, slots, plan, window=0):
    """Workgroups that the longest sequence's last tile is divided among (at least: a window may begin inside a block)."""
    longest = max(int(C.length[s]) for s in slots)
    return min(plan["splits"], -(-(-(-(min(longest, window) if window else longest) // 32)) // plan["chunk"]))


@pytest.mark.parametrize("dtype,D,heads,kv,news,window,row_tiles", [
    ("bf16", 128, 16, 4, [7, 1, 5, 7, 2, 7, 3, 7], 0, 1),             # 28 rows: one tile, 28 rows of sums
    ("f16", 64, 4, 4, [17, 16, 3, 17, 9, 17, 1, 17], 0, 1),           # 17: one row in the tile's second half
    ("f16", 128, 8, 4, [16, 16, 15, 16, 1, 16, 8, 16], 0, 1),         # 32: a full tile
    ("bf16", 64, 24, 4, [7, 6, 7, 5, 1, 7, 7, 3], 0, 2),              # 42: two tiles
    ("f16", 128, 16, 4, [9, 9, 1, 9, 4, 9, 9, 9], 0, 2),              # 36
])
def test_attention_split_tiles_of_32_rows(gpu_device, dtype, D, heads, kv, news, window, row_tiles):
    rng = np.random.default_rng(D + heads + len(news))
    lengths = [3000, 2047, 40, 1025, 9, 2600, 700, 1500]
    lengths = [max(n, k) for n, k in zip(lengths, news)]
    C, slots = U.random_cache(rng, lengths, 256, kv, D, dtype, headroom=33000)
    starts = np.concatenate([[0], np.cumsum(news)])
    plan = plan_of(C, slots, starts, int(starts[-1]), heads, max(news), max_len=33000)
    assert (plan["tile_rows"], plan["row_tiles"]) == (32, row_tiles) and real_splits(C, slots, plan) >= 2, plan
    q = U.random_rows(rng, int(starts[-1]), heads * D, dtype)
    check_attention(C, slots, starts, q, heads, max_new=max(news), max_len=33000)


@pytest.mark.parametrize("dtype,heads,kv,new,row_tiles", [("bf16", 64, 16, 5, 1), ("f16", 32, 8, 9, 2)])
def test_attention_split_tiles_of_32_rows_with_a_window(gpu_device, dtype, heads, kv, new, row_tiles):
    rng = np.random.default_rng(heads + new)
    lengths = [2500, 2100, 2040] + rng.integers(new, 300, 29).tolist()
    C, slots = U.random_cache(rng, lengths, 256, kv, 64, dtype)
    starts = np.arange(33) * new
    plan = plan_of(C, slots, starts, 32 * new, heads, new, window=2000)
    assert (plan["tile_rows"], plan["row_tiles"]) == (32, row_tiles) and real_splits(C, slots, plan, 2000) >= 2, plan
    check_attention(C, slots, starts, U.random_rows(rng, 32 * new, heads * 64, dtype), heads, window=2000, max_new=new)


@pytest.mark.parametrize("dtype,D,heads,n,least", [("bf16", 64, 3, 66001, 200), ("f16", 128, 1, 66001, 200), ("f16", 256, 5, 25000, 90)])
def test_attention_many_splits(gpu_device, dtype, D, heads, n, least):
    """One sequence among up to 256 workgroups: the joining launch takes its sums in several rounds."""
    rng = np.random.default_rng(D)
    C, slots = U.random_cache(rng, [n], 256, 1, D, dtype)
    plan = plan_of(C, slots, None, 1, heads)
    assert real_splits(C, slots, plan) >= least, plan
    check_attention(C, slots, None, U.random_rows(rng, 1, heads * D, dtype), heads)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 12, 2 ** 30])
def test_attention_largest_windows_with_rows_before_the_first_token(gpu_device, window):
    """More new rows than tokens: the first ones see nothing, the others in the same tile everything, however large the window."""
    rng = np.random.default_rng(28)
    C, slots = U.random_cache(rng, [10, 0, 40, 700], 32, 1, 64, "f16")
    q = U.random_rows(rng, 14 + 5 + 60 + 3, 2 * 64, "f16")
    starts = [0, 14, 19, 79, 82]
    got = check_attention(C, slots, starts, q, 2, window=window, max_new=60)
    assert not got[:4].any() and got[4:14].any((1, 2)).all()
    assert np.array_equal(got, check_attention(C, slots, starts, q, 2, max_new=60))


@pytest.mark.parametrize("window", [0, 700])
@pytest.mark.parametrize("max_len", [1, 700, 800, 1500, 100000])
def test_attention_longer_and_shorter_than_announced(gpu_device, window, max_len):
    """max_len only divides the work: the last workgroup of a tile takes what is left, those past the end nothing."""
    rng = np.random.default_rng(27)
    C, slots = U.random_cache(rng, [3000, 801, 5, 0], 64, 2, 64, "f16")
    check_attention(C, slots, None, U.random_rows(rng, 4, 6 * 64, "f16"), 6, window=window, max_len=max_len)


@pytest.mark.parametrize("dtype,D,heads,kv,n,new,window,tile_rows", [
    ("bf16", 128, 8, 2, 2300, 1400, 0, 16), ("f16", 64, 6, 2, 2999, 1100, 0, 16), ("bf16", 64, 8, 2, 2500, 2500, 900, 32),
    ("bf16", 128, 8, 2, 2300, 1900, 0, 32), ("f16", 64, 6, 2, 2999, 1900, 0, 32), ("f16", 256, 2, 1, 700, 450, 0, 16)])
def test_attention_long_prompts(gpu_device, dtype, D, heads, kv, n, new, window, tile_rows):
    """Prompts, the longer ones in tiles of 32 rows by their own length, against fp64 in whole matrices."""
    rng = np.random.default_rng(D + n)
    C, slots = U.random_cache(rng, [n], 64, kv, D, dtype)
    q_bits = U.random_rows(rng, new, heads * D, dtype)
    assert plan_of(C, slots, [0, new], new, heads, new, window)["tile_rows"] == tile_rows
    got, _ = run_attention(C, slots, [0, new], q_bits, heads, window=window, scale=D ** -0.5, max_new=new)
    q, group = O.decode16(q_bits, dtype).reshape(new, heads, D), heads // kv
    place, t = np.arange(n - new, n)[:, None], np.arange(n)[None, :]
    seen = (t <= place) & ((t > place - window) if window else True)
    for h in range(heads):
        k, v, have = K.keys_values(C, 0, slots[0], n, h // group)
        assert have.all()
        s = np.where(seen, q[:, h] @ k.T * D ** -0.5, -np.inf)
        size = np.where(seen, np.abs(q[:, h]) @ np.abs(k).T * D ** -0.5, 0).max(1, keepdims=True)
        top = s.max(1, keepdims=True)
        spread = np.where(seen, top - s, 0).max(1, keepdims=True)
        w = np.exp(s - top)
        w /= w.sum(1, keepdims=True)
        out, mag = w @ v, w @ np.abs(v)
        # the terms of attention_want: a weight's and the store's half step, the logit's and the sums' fp32
        u = U.HALF_STEP[dtype]
        logit = (D * size + 3 * (size + spread)) * 2.0 ** -24 + 2.0 ** -22
        tol = u * np.abs(out) * 1.01 + mag * (u + 2 * (logit + 2 * (n + 8) * 2.0 ** -24)) + 2.0 ** -25
        err = np.abs(got[:, h] - out)
        assert (err <= tol).all(), f"head {h}: {(err / tol).max():.2f} of the tolerance"


# ---- append ---------------------------------------------------------------------------------------------------

def make_table(rng, n, rot):
    a = rng.uniform(-np.pi, np.pi, (n, rot // 2))
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def check_append(rng, C, slots, starts, n_heads, qkv_bits, rot=0, axis_pairs=None, positions=None, interleaved=False, n_pos=512,
                 max_new=1, in_place=False, layer=0, ld_extra=0):
    from paper_2507_01299_amd import api
    D, H, dt = C.head_dim, C.n_kv_heads, C.dtype
    heads = n_heads + 2 * H
    rows = qkv_bits.shape[0]
    cache = U.device_cache(C)
    qkv = torch.zeros(rows, heads * D + ld_extra, dtype=api.torch_dtype(dt), device="cuda:0")
    qkv[:, :heads * D] = U.to_dev(qkv_bits, dt)
    out = qkv if in_place else torch.full((rows, heads * D + ld_extra), 77.0, dtype=api.torch_dtype(dt), device="cuda:0")
    table = make_table(rng, n_pos, rot) if rot else None
    rotary = api.Rotary(torch.from_numpy(table).to("cuda:0"), axis_pairs=axis_pairs, interleaved=interleaved,
                        positions=None if positions is None else torch.from_numpy(positions).to("cuda:0")) if rot else None
    batch = api.KvBatch(U.int32(slots), rows, starts=U.int32(starts), max_new=max_new)
    api.kv4_append(cache, layer, batch, qkv, n_heads, out=out, rotary=rotary)
    torch.cuda.synchronize()
    got = U.to_bits(out[:, :heads * D].contiguous()).reshape(rows, heads, D)
    if ld_extra:
        assert (out[:, heads * D:] == (0.0 if in_place else 77.0)).all()
    x = O.decode16(qkv_bits, dt).reshape(rows, heads, D)
    done = set()
    for i, slot in enumerate(slots):
        _, n_new, mine = U.rows_of(starts, len(slots), i, max_new)
        if not 0 <= slot < C.n_slots:
            continue
        for j, row in enumerate(mine):
            done.add(row)
            place = int(C.length[slot]) - n_new + j
            for h in range(heads):
                y32, y64 = x[row, h].astype(np.float32), x[row, h]
                if rot and h < n_heads + H:
                    pos = [place] if positions is None else positions[:, row]
                    y32 = K.rotate(x[row, h], table, pos, axis_pairs, interleaved, np.float32)
                    y64 = K.rotate(x[row, h], table, pos, axis_pairs, interleaved)
                if h < n_heads:
                    a, b = O.decode16(got[row, h], dt), y64
                    assert np.array_equal(np.isnan(a), np.isnan(b))
                    size = 2 * np.abs(np.where(np.isfinite(x[row, h]), x[row, h], 0.0)).max()
                    ok = np.isfinite(a) & np.isfinite(b)
                    # one store, two products and a sum in fp32; f16 subnormals are 2^-24 apart
                    assert (np.abs(a - b)[ok] <= (U.HALF_STEP[dt] * np.abs(b) * 1.01 + 4 * 2.0 ** -24 * size + 2.0 ** -25)[ok]).all()
                    ok = ~np.isnan(b)
                    assert np.array_equal(got[row, h][ok], O.encode16(y32.astype(np.float64), dt)[ok])
                else:
                    which, kv = divmod(h - n_heads, H)
                    codes, scales = K.quantise(y32, dt)
                    want = O.encode16(K.stored(y32, dt), dt)
                    a, b = O.decode16(got[row, h], dt), O.decode16(want, dt)
                    assert np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(a[~np.isnan(a)], b[~np.isnan(b)])
                    block = C.block(layer, slot, place, kv) if place >= 0 else None
                    if block is not None:
                        K.write_token(block, D, place % 32, which, codes, scales)
    for row in set(range(rows)) - done:
        assert np.array_equal(got[row].reshape(-1), qkv_bits[row] if in_place else O.encode16(np.full(heads * D, 77.0), dt))
    U.same_state(cache, C)                        # every byte: what was to be written, and nothing else


@pytest.mark.parametrize("dtype,D,heads,kv,P,rot,interleaved", [
    ("f16", 128, 4, 2, 32, 128, False), ("bf16", 128, 2, 1, 64, 64, False), ("bf16", 64, 4, 4, 32, 64, True),
    ("f16", 256, 2, 1, 128, 256, False), ("bf16", 256, 1, 1, 32, 16, True), ("f16", 64, 3, 1, 32, 0, False)])
def test_append_one_token(gpu_device, dtype, D, heads, kv, P, rot, interleaved):
    rng = np.random.default_rng(D + rot + heads)
    C, slots = U.random_cache(rng, [1, 16, 17, 32, 33, 90], P, kv, D, dtype)
    check_append(rng, C, slots, None, heads, U.random_rows(rng, 6, (heads + 2 * kv) * D, dtype), rot=rot, interleaved=interleaved)


@pytest.mark.parametrize("in_place", [False, True])
def test_append_prompts_with_three_axes(gpu_device, in_place):
    rng = np.random.default_rng(21)
    heads, kv, D = 4, 2, 128
    C, slots = U.random_cache(rng, [70, 5, 40], 32, kv, D, "bf16", n_layers=2)
    starts = [0, 60, 65, 70]
    positions = rng.integers(0, 512, (3, 72)).astype(np.int32)
    check_append(rng, C, slots, starts, heads, U.random_rows(rng, 72, (heads + 2 * kv) * D, "bf16"), rot=128, axis_pairs=(16, 24, 24),
                 positions=positions, max_new=60, layer=1, in_place=in_place, ld_extra=16)


def test_append_special_values_and_bad_places(gpu_device):
    """Zeros, infinities, NaN, the largest and smallest numbers; padding, missing pages, places below zero, positions outside the table."""
    for dtype in ("f16", "bf16"):
        rng = np.random.default_rng(22)
        heads, kv, D = 2, 1, 64
        C, slots = U.random_cache(rng, [3, 40, 64, 20, 2], 32, kv, D, dtype, headroom=32)
        slots = slots.tolist()
        C.table[slots[1], 1] = -1
        C.table[slots[2], 1] = C.n_pages
        slots[3] = -5
        starts = [0, 3, 5, 7, 9, 14]
        bits = U.random_rows(rng, 15, (heads + 2 * kv) * D, dtype).reshape(15, -1, 32)
        special = O.encode16(np.array([0.0, -0.0, np.inf, -np.inf, np.nan, 65504.0, -65504.0, 2.0 ** -24, 6e-5, 1.0]), dtype)
        bits[0, :, 3] = special[2]
        bits[1, :, 7] = special[4]
        bits[2] = 0
        bits[9, :, :] = special[7]
        bits[10, :, 5] = special[5]
        bits[11, :, 5] = special[6]
        bits[12, :, :] = special[[0, 1, 7, 8] * 8]
        if dtype == "bf16":
            bits[13, :, 1] = O.encode16(np.array([3.3e38]), dtype)
            bits[5, :, :] = O.encode16(np.array([1e-38]), dtype)
        positions = rng.integers(0, 100, (1, 15)).astype(np.int32)
        positions[0, [3, 4]] = -1, 100
        check_append(rng, C, slots, starts, heads, bits.reshape(15, -1), rot=64, positions=positions, n_pos=100, max_new=5)


def test_append_ties(gpu_device):
    """Halves between all neighbouring codes, at several scales and both signs."""
    for dtype in ("f16", "bf16"):
        rng = np.random.default_rng(23)
        x = np.tile([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 0.5, 1.5, 3.0, 4.0, 2.0, 1.0, 0.0], (4, 2 * 16))
        x *= np.array([1.0, -1.0, 2.0 ** -9, -2.0 ** 5])[:, None]
        C, slots = U.random_cache(rng, [1, 2, 3, 4], 32, 2, 64, dtype)
        bits = np.concatenate([O.encode16(x[:, :4 * 64], dtype), U.random_rows(rng, 4, 2 * 64, dtype)], 1)
        check_append(rng, C, slots, None, 2, np.ascontiguousarray(np.roll(bits, 128, axis=1)))
