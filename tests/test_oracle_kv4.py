"""Pins of the CPU statement of the 4-bit key/value cache (no GPU): the format against hand-worked values and brute force, rotary
positions against complex numbers, attention against a separately written softmax, page bookkeeping by its invariants."""
import numpy as np
import pytest

from oracle import kv4_oracle as K


@pytest.mark.parametrize("D", [64, 128, 256])
def test_every_code_and_scale_has_a_byte_of_its_own(D):
    nibbles, scales = set(), set()
    for t in range(32):
        for which in (0, 1):
            nibbles |= {K.code_place(D, t, i, which) for i in range(D)}
            scales |= {K.scale_place(D, t, g, which) for g in range(D // 32)}
    assert len(nibbles) == 2 * 32 * D and {b for b, _ in nibbles} == set(range(32 * D))
    assert scales == set(range(32 * D, 34 * D))


def test_layout_by_hand():
    # D = 128: the first 16-byte piece of a tile is values 0..31 of its first token, the 17th values 32..63
    assert K.code_place(128, 0, 0, 0) == (0, 0) and K.code_place(128, 0, 1, 0) == (0, 1) and K.code_place(128, 0, 31, 0) == (15, 1)
    assert K.code_place(128, 1, 0, 0) == (16, 0) and K.code_place(128, 0, 32, 0) == (256, 0) and K.code_place(128, 16, 0, 0) == (1024, 0)
    # V: 16 bytes are values 0..7 of tokens 0..3
    assert K.code_place(128, 0, 0, 1) == (2048, 0) and K.code_place(128, 1, 2, 1) == (2053, 0) and K.code_place(128, 4, 0, 1) == (2304, 0)
    assert K.scale_place(128, 5, 2, 0) == 4096 + 37 and K.scale_place(128, 21, 2, 1) == 4224 + 64 + (4 + 2) * 4 + 1


def test_write_and_read_agree():
    rng = np.random.default_rng(3)
    for D in (64, 128, 256):
        block = rng.integers(0, 256, 34 * D).astype(np.uint8)
        x = rng.standard_normal((32, 2, D))
        for t in rng.permutation(32):
            for which in (0, 1):
                K.write_token(block, D, t, which, *K.quantise(x[t, which], "f16"))
        for which in (0, 1):
            got = K.read_block(block, D, which)
            for t in range(32):
                assert np.array_equal(got[t], K.stored(x[t, which], "f16"))


def test_quantise_hand_values():
    x = np.zeros(32)
    x[:9] = [6.0, 5.0, 5.1, 2.5, 0.25, 0.75, -0.3, 7.0, 1.25]
    assert K.stored(x, "f16")[:9].tolist() == [6.0, 4.0, 6.0, 2.0, 0.0, 1.0, -0.5, 6.0, 1.0]     # ties: 5, 2.5, 0.25, 0.75, 1.25
    x[0] = 7.1                                               # past 7: the scale doubles
    assert K.quantise(x, "f16")[1][0] == 128 and K.stored(x, "f16")[0] == 8.0
    assert K.quantise(np.zeros(32), "f16")[1][0] == 127 - 23
    x[3] = np.inf
    assert np.isnan(K.stored(x, "bf16")).all()


def test_quantise_is_within_half_a_step_of_the_nearest():
    rng = np.random.default_rng(4)
    for _ in range(50):
        x = rng.standard_normal(32) * 2.0 ** rng.integers(-8, 8)
        s = K.stored(x, "bf16")
        unit = 2.0 ** (K.quantise(x, "bf16")[1][0] - 127.0)
        grid = np.concatenate([-K.LEVELS, K.LEVELS]) * unit
        assert np.array_equal(np.abs(x - s), np.abs(x[:, None] - grid[None]).min(1))
        assert np.abs(x - s).max() <= unit                   # the widest step is 2: half of it


def test_rotation_is_a_complex_product_and_keeps_lengths():
    rng = np.random.default_rng(5)
    D, rot = 64, 32
    angle = rng.uniform(-3, 3, (9, rot // 2))
    table = np.concatenate([np.cos(angle), np.sin(angle)], 1)
    x = rng.standard_normal(D)
    y = K.rotate(x, table, [4], None, False)
    z = (x[:16] + 1j * x[16:32]) * np.exp(1j * angle[4])
    assert np.allclose(y[:16], z.real) and np.allclose(y[16:32], z.imag) and np.array_equal(y[32:], x[32:])
    y = K.rotate(x, table, [4], None, True)
    z = (x[0:32:2] + 1j * x[1:32:2]) * np.exp(1j * angle[4])
    assert np.allclose(y[0:32:2], z.real) and np.allclose(y[1:32:2], z.imag)
    y = K.rotate(x, table, [1, 7], [6, 10], False)
    z = (x[:16] + 1j * x[16:32]) * np.exp(1j * np.concatenate([angle[1, :6], angle[7, 6:]]))
    assert np.allclose(y[:16], z.real) and np.allclose(y[16:32], z.imag)
    assert np.isnan(K.rotate(x, table, [9], None, False)[:32]).all()


def test_attention_row_against_a_direct_softmax():
    rng = np.random.default_rng(6)
    k, v, q = rng.standard_normal((20, 64)), rng.standard_normal((20, 64)), rng.standard_normal(64)
    seen = np.arange(20) % 3 != 0
    w = np.array([np.exp(np.dot(q, k[t]) / 8) if seen[t] else 0.0 for t in range(20)])
    want = sum(w[t] * v[t] for t in range(20)) / w.sum()
    assert np.allclose(K.attention_row(q, k, v, seen, 1 / 8)[0], want)
    assert not K.attention_row(q, k, v, np.zeros(20, bool), 1 / 8)[0].any()


def consistent(C):
    named = np.zeros(C.n_pages, int)
    for s in range(C.n_slots):
        n = K.pages_of(int(C.length[s]), C.page_tokens)
        assert (C.table[s, :n] >= 0).all() and (C.table[s, n:] == -1).all()
        for p in C.table[s, :n]:
            named[p] += 1
    assert np.array_equal(named, C.refs)


def contents(C, slot):
    return [C.data[0, C.table[slot, p]].copy() for p in range(K.pages_of(int(C.length[slot]), C.page_tokens))]


def test_pages_random_walk_keeps_invariants_and_contents():
    rng = np.random.default_rng(7)
    C = K.Cache(1, 24, 32, 6, 5, 1, 64, "f16")
    C.data[:] = rng.integers(0, 256, C.data.shape)
    for step in range(300):
        before = {s: contents(C, s) for s in range(6)}
        lengths = C.length.copy()
        op = rng.integers(4)
        touched = []
        if op == 0:
            touched = [int(s) for s in rng.permutation(6)[:2]]
            keep = rng.integers(0, 100, 2)
            K.trim(C, touched, keep)
            for s, k in zip(touched, keep):
                assert C.length[s] == min(lengths[s], k)
        elif op == 1:
            src, dst = rng.permutation(6)[:2]
            status = K.fork(C, [src], [dst])
            assert status == (0 if lengths[dst] == 0 else -1)
            if status == 0:
                assert all(np.array_equal(a, b) for a, b in zip(contents(C, dst), before[src]))
                touched = [dst]
        elif op == 2:
            touched = [int(s) for s in rng.permutation(6)[:3]]
            counts = [int(c) for c in rng.integers(0, 40, 3)]
            if K.grow(C, touched, counts) != 0:
                assert np.array_equal(C.length, lengths)
            for s in touched:                                # what was there stays; the page being written is its own
                assert all(np.array_equal(a, b) for a, b in zip(before[s], contents(C, s)))
                if C.length[s] > lengths[s] and lengths[s] % 32:
                    assert C.refs[C.table[s, lengths[s] // 32]] == 1
        else:
            n = K.compact(C)
            assert (C.refs[:n] > 0).all() and (C.refs[n:] == 0).all()
        consistent(C)
        for s in set(range(6)) - set(touched):
            assert all(np.array_equal(a, b) for a, b in zip(before[s], contents(C, s))) and C.length[s] == lengths[s]


def test_grow_last_holder_keeps_the_page_and_refusals_change_nothing():
    C = K.Cache(1, 6, 32, 4, 3, 1, 64, "f16")
    assert K.grow(C, [0], [40]) == 0 and C.table[0].tolist() == [0, 1, -1]
    assert K.fork(C, [0, 0], [1, 2]) == 0 and C.refs.tolist()[:2] == [3, 3]
    assert K.grow(C, [2, 0, 1], [1, 1, 1]) == 0              # two copies, slot 1 keeps page 1
    assert [C.table[s, 1] for s in (2, 0, 1)] == [2, 3, 1] and C.refs.tolist() == [3, 1, 1, 1, 0, 0]
    state = C.table.copy(), C.refs.copy(), C.length.copy()
    assert K.grow(C, [0, 1, 2], [30, 30, 30]) == 1           # three pages wanted, two are free
    assert K.grow(C, [0, 0], [1, 1]) == K.grow(C, [4], [1]) == K.grow(C, [0], [-1]) == K.grow(C, [0], [100]) == -1
    assert K.fork(C, [0], [1]) == K.fork(C, [0, 1], [3, 3]) == -1
    assert all(np.array_equal(a, b) for a, b in zip(state, (C.table, C.refs, C.length)))
