"""Host-side checks of the 4-bit key/value cache's entry points that need no GPU: sizes, and refusals before a device is touched."""
import ctypes
import os

import pytest

FAKE, OTHER, ODD = 0x1000, 0x2000, 0x1004        # never dereferenced: checks fail first
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    from paper_2507_01299_amd import api, build
    if not os.path.exists(api.LIB_PATH):
        build.build_library()
    return api.lib()


def cache(**kw):
    from paper_2507_01299_amd import api
    d = dict(n_layers=2, n_pages=10, page_tokens=64, n_slots=4, max_pages=8, n_kv_heads=2, head_dim=128, dtype=1, data=FAKE, refs=FAKE,
             table=FAKE, length=FAKE)
    d.update(kw)
    return api._KvCache(**d)


def batch(**kw):
    from paper_2507_01299_amd import api
    d = dict(slots=FAKE, starts=None, n_seq=3, n_rows=3, max_new=1)
    d.update(kw)
    return api._KvBatch(**d)


def rotary(axis_pairs=(), **kw):
    from paper_2507_01299_amd import api
    d = dict(table=FAKE, n_positions=100, rot_dim=128, interleaved=0, positions=None, n_axes=1)
    d.update(kw)
    r = api._Rotary(**d)
    for i, n in enumerate(axis_pairs):
        r.axis_pairs[i] = n
    return r


BAD_CACHES = [dict(n_layers=0), dict(n_pages=0), dict(n_slots=0), dict(max_pages=0), dict(n_kv_heads=0), dict(page_tokens=16),
              dict(page_tokens=48), dict(page_tokens=512), dict(dtype=2), dict(dtype=-1)]
UNSUPPORTED_CACHES = [dict(head_dim=32), dict(head_dim=96), dict(head_dim=512), dict(max_pages=1 << 25), dict(n_pages=1 << 29),
                      dict(n_slots=(1 << 18) + 1), dict(n_slots=1 << 18, max_pages=1 << 14), dict(n_layers=1 << 16), dict(n_kv_heads=5000)]
BAD_POINTERS = [dict(data=None), dict(refs=None), dict(table=None), dict(length=None), dict(data=0x1008), dict(table=0x1002)]


def test_sizes(lib):
    ref = ctypes.byref
    assert lib.larosa_kv4_page_bytes(64, 8, 128) == 8 * 64 * 136
    assert lib.larosa_kv4_page_bytes(32, 1, 64) == 32 * 68 and lib.larosa_kv4_page_bytes(33, 1, 64) == 0
    assert lib.larosa_kv4_data_bytes(ref(cache())) == 2 * 10 * 2 * 64 * 136
    assert lib.larosa_kv4_data_bytes(ref(cache(n_layers=80, n_pages=1 << 20, n_kv_heads=8))) == 80 * (1 << 20) * 8 * 64 * 136
    for bad in BAD_CACHES + UNSUPPORTED_CACHES:
        assert lib.larosa_kv4_data_bytes(ref(cache(**bad))) == 0
    n = lib.larosa_kv4_attention_workspace_bytes(ref(cache(data=None)), ref(batch()), 8, 0)
    assert n > 0
    assert lib.larosa_kv4_attention_workspace_bytes(ref(cache()), ref(batch(n_seq=0)), 8, 0) == 0
    assert lib.larosa_kv4_attention_workspace_bytes(ref(cache()), ref(batch()), 7, 0) == 0
    assert lib.larosa_kv4_attention_workspace_bytes(ref(cache()), ref(batch()), 8, -1) == 0


def test_every_call_checks_the_cache(lib):
    from paper_2507_01299_amd import api
    ref = ctypes.byref
    calls = [lambda c: lib.larosa_kv4_clear(ref(c), None),
             lambda c: lib.larosa_kv4_grow(ref(c), FAKE, None, 2, FAKE, FAKE, BIG, None),
             lambda c: lib.larosa_kv4_fork(ref(c), FAKE, OTHER, 2, FAKE, None),
             lambda c: lib.larosa_kv4_trim(ref(c), FAKE, None, 2, None),
             lambda c: lib.larosa_kv4_compact(ref(c), None, FAKE, BIG, None),
             lambda c: lib.larosa_kv4_copy_pages(ref(c), FAKE, OTHER, 2, None),
             lambda c: lib.larosa_kv4_append(ref(c), 0, ref(batch()), FAKE, 1536, 8, None, None, 0, None),
             lambda c: lib.larosa_kv4_attention(ref(c), 0, ref(batch()), FAKE, 1024, 8, 1.0, 0, 0, OTHER, 1024, FAKE, BIG, None)]
    for call in calls:
        for bad in BAD_CACHES + BAD_POINTERS:
            assert call(cache(**bad)) == api.EINVAL, bad
        for bad in UNSUPPORTED_CACHES:
            assert call(cache(**bad)) == api.EUNSUPPORTED, bad
    assert lib.larosa_kv4_clear(None, None) == api.EINVAL


BAD_BATCHES = [dict(slots=None), dict(n_seq=0), dict(n_rows=0), dict(max_new=0), dict(max_new=2), dict(n_rows=2), dict(slots=0x1001),
               dict(starts=0x1002)]


def test_append_refuses(lib):
    from paper_2507_01299_amd import api
    ref = ctypes.byref

    def call(b=None, layer=0, qkv=FAKE, ld=1536, heads=8, r=None, out=OTHER, ld_out=1536):
        return lib.larosa_kv4_append(ref(cache()), layer, ref(b or batch()), qkv, ld, heads, ref(r) if r else None, out, ld_out, None)

    for bad in BAD_BATCHES:
        assert call(batch(**bad)) == api.EINVAL, bad
    assert call(batch(starts=FAKE, max_new=(1 << 18) + 1)) == api.EUNSUPPORTED
    assert call(batch(n_seq=70000, n_rows=70000)) == api.EUNSUPPORTED
    for bad in (dict(layer=-1), dict(layer=2), dict(qkv=None), dict(qkv=ODD), dict(out=ODD), dict(ld=1528), dict(ld=1540), dict(ld_out=1528),
                dict(ld_out=1537), dict(heads=0), dict(heads=7), dict(out=FAKE, ld_out=1544), dict(out=None, r=rotary()),
                dict(r=rotary(table=None)), dict(r=rotary(table=0x1008)), dict(r=rotary(n_positions=0)), dict(r=rotary(rot_dim=24)), dict(r=rotary(rot_dim=256)),
                dict(r=rotary(rot_dim=0)), dict(r=rotary(n_axes=0)), dict(r=rotary(n_axes=5)), dict(r=rotary((32, 32), n_axes=2)),
                dict(r=rotary((32, 31), n_axes=2, positions=FAKE)), dict(r=rotary((-1, 65), n_axes=2, positions=FAKE)),
                dict(r=rotary(positions=0x1002))):
        assert call(**bad) == api.EINVAL, bad


def test_attention_refuses(lib):
    from paper_2507_01299_amd import api
    ref = ctypes.byref

    def call(b=None, layer=0, q=FAKE, ld=1024, heads=8, scale=1.0, window=0, max_len=0, out=OTHER, ld_out=1024, ws=FAKE, nbytes=BIG):
        return lib.larosa_kv4_attention(ref(cache()), layer, ref(b or batch()), q, ld, heads, scale, window, max_len, out, ld_out, ws, nbytes,
                                        None)

    for bad in BAD_BATCHES:
        assert call(batch(**bad)) == api.EINVAL, bad
    for bad in (dict(layer=-1), dict(layer=2), dict(q=None), dict(q=ODD), dict(out=None), dict(out=ODD), dict(out=FAKE), dict(ld=1016),
                dict(ld=1025), dict(ld_out=1016), dict(ld_out=1028), dict(heads=0), dict(heads=9), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(window=-1), dict(max_len=-1)):
        assert call(**bad) == api.EINVAL, bad
    need = lib.larosa_kv4_attention_workspace_bytes(ref(cache()), ref(batch()), 8, 0)
    for bad in (dict(ws=None), dict(ws=0x1010), dict(nbytes=need - 1)):
        assert call(**bad) == api.EWORKSPACE, bad


def test_page_calls_refuse(lib):
    from paper_2507_01299_amd import api
    c = ctypes.byref(cache())
    need = lib.larosa_kv4_pages_workspace_bytes(c)
    assert need > 1 << 20 and lib.larosa_kv4_pages_workspace_bytes(ctypes.byref(cache(page_tokens=7))) == 0
    for slots, counts, n, status in ((None, None, 2, FAKE), (0x1001, None, 2, FAKE), (FAKE, 0x1002, 2, FAKE), (FAKE, None, 0, FAKE),
                                     (FAKE, None, 5, FAKE), (FAKE, None, 2, None), (FAKE, None, 2, 0x1001)):
        assert lib.larosa_kv4_grow(c, slots, counts, n, status, FAKE, BIG, None) == api.EINVAL
    for ws, n in ((None, BIG), (0x1010, BIG), (FAKE, need - 1)):
        assert lib.larosa_kv4_grow(c, FAKE, None, 2, FAKE, ws, n, None) == api.EWORKSPACE
        assert lib.larosa_kv4_compact(c, None, ws, n, None) == api.EWORKSPACE
    for src, dst, n, status in ((None, FAKE, 1, FAKE), (FAKE, None, 1, FAKE), (FAKE, OTHER, 0, FAKE), (FAKE, OTHER, 5, FAKE),
                                (FAKE, OTHER, 1, None), (0x1001, OTHER, 1, FAKE)):
        assert lib.larosa_kv4_fork(c, src, dst, n, status, None) == api.EINVAL
    for slots, keep, n in ((None, None, 1), (FAKE, 0x1001, 1), (FAKE, None, 0)):
        assert lib.larosa_kv4_trim(c, slots, keep, n, None) == api.EINVAL
    assert lib.larosa_kv4_trim(c, FAKE, None, 1 << 21, None) == api.EUNSUPPORTED
    assert lib.larosa_kv4_compact(c, 0x1002, FAKE, BIG, None) == api.EINVAL
    for src, dst, n in ((None, FAKE, 1), (FAKE, None, 1), (FAKE, OTHER, 0), (FAKE, OTHER, 11), (FAKE, 0x2001, 1)):
        assert lib.larosa_kv4_copy_pages(c, src, dst, n, None) == api.EINVAL


def test_layer_with_cache_refuses(lib):
    from paper_2507_01299_amd import api
    ref = ctypes.byref
    layer = lambda **kw: api._Layer(**dict(dict(d=256, d_q=512, d_kv=256, d_ff=704, head_dim=128, K1=100, K2=100, K3=100, K4=300, Wqkv=FAKE,  # noqa: E731
                                                Wo=FAKE, Wgu=FAKE, Wdown=FAKE, rms_eps=-1.0, dtype=1), **kw))
    L, C, b = layer(), cache(), batch()
    need = lib.larosa_layer_kv4_workspace_bytes(ref(L), ref(C), ref(b), 0)
    assert need > lib.larosa_layer_workspace_bytes(ref(L), 3)

    def call(L=L, C=C, b=b, layer=0, r=None, scale=1.0, window=0, max_len=0, x=FAKE, x_out=OTHER, ws=FAKE, n=BIG):
        return lib.larosa_layer_forward_kv4(ref(L), ref(C), layer, ref(b), ref(r) if r else None, scale, window, max_len, x, x_out, None, ws, n,
                                            None)

    for bad in (dict(L=layer(head_dim=64)), dict(L=layer(dtype=0)), dict(L=layer(d_kv=128)), dict(L=layer(d_q=576)), dict(L=layer(K1=0)),
                dict(L=layer(Wo=None)), dict(C=cache(data=None)), dict(C=cache(page_tokens=5)), dict(b=batch(n_seq=0)), dict(layer=2),
                dict(layer=-1), dict(scale=float("inf")), dict(window=-1), dict(max_len=-1), dict(x=None), dict(x=ODD), dict(x_out=None),
                dict(x_out=FAKE), dict(x_out=ODD), dict(r=rotary(rot_dim=8))):
        assert call(**bad) == api.EINVAL, bad
    for bad in (dict(ws=None), dict(ws=0x1010), dict(n=need - 1)):
        assert call(**bad) == api.EWORKSPACE, bad
    assert call(L=layer(attn_mode=1)) == api.EUNSUPPORTED


def test_layer_with_cache_refuses_rows_before_anything_is_enqueued(lib):
    """More rows than the layer's projections have counters for (4096, one for each 32 rows and 128 columns), and more attention
    tiles than a launch has workgroups: refused by the size query and by the call, which with these addresses could enqueue nothing."""
    from paper_2507_01299_amd import api
    ref = ctypes.byref
    big = dict(d=4096, d_q=4096, d_kv=1024, d_ff=14336, head_dim=128, K1=2000, K2=2000, K3=2000, K4=7000, Wqkv=FAKE, Wo=FAKE, Wgu=FAKE,
               Wdown=FAKE, rms_eps=1e-5, dtype=1)
    small = dict(big, d=256, d_q=512, d_kv=256, d_ff=704, K1=100, K2=100, K3=100, K4=300)
    C8, C2 = cache(n_kv_heads=8), cache()

    def both(L, C, n):
        L, b = api._Layer(**L), batch(starts=FAKE, n_seq=1, n_rows=n, max_new=n)
        size = lib.larosa_layer_kv4_workspace_bytes(ref(L), ref(C), ref(b), 0)
        rc = [lib.larosa_layer_forward_kv4(ref(L), ref(C), 0, ref(b), None, 1.0, 0, 0, FAKE, OTHER, None, FAKE, BIG, None)] if not size else []
        if rc:                        # and the layer's own calls that reach the projection at fault
            rc += [lib.larosa_layer_forward(ref(L), FAKE, OTHER, n, None, FAKE, BIG, None),
                   lib.larosa_layer_after_attention(ref(L), FAKE, FAKE, OTHER, n, None, FAKE, BIG, None)]
        return size, rc

    # gate|up: 224 strips of 128 columns, 18 groups of 32 rows; with a shortcut adapter 256 strips, 16 groups; a rotation behind a
    # learned scale: 32 strips, 128 groups of 4 rows
    for L, C, most in ((big, C8, 576), (dict(big, shortcut_mlp=FAKE), C8, 512), (small, C2, 32 * (4096 // 11)),
                       (dict(big, Q_mlp=FAKE, rms_mlp=FAKE), C8, 512)):
        assert both(L, C, most)[0] > 0 and both(L, C, 1)[0] > 0
        for n in (most + 1, most + 40, 16384):
            assert both(L, C, n) == (0, [api.EUNSUPPORTED] * 3), n
    assert both(small, C2, 65536) == (0, [api.EINVAL] * 3)
    # tiles of 16 rows times key/value heads: below 2^24
    wide, C1 = dict(small, d_q=16384, d_kv=64, head_dim=64), cache(n_kv_heads=1, head_dim=64)
    b = lambda most: batch(starts=FAKE, n_seq=1, n_rows=8, max_new=most)                  # noqa: E731
    assert lib.larosa_layer_kv4_workspace_bytes(ref(api._Layer(**wide)), ref(C1), ref(b(1 << 18)), 0) > 0
    wide["d_q"] = 32768
    assert lib.larosa_kv4_attention_workspace_bytes(ref(C1), ref(b(1 << 18)), 1024, 0) == 0
    assert lib.larosa_kv4_attention(ref(C1), 0, ref(b(1 << 18)), FAKE, 65536, 1024, 1.0, 0, 0, OTHER, 65536, FAKE, BIG, None) == api.EUNSUPPORTED


def test_binding_refuses():
    import torch
    from paper_2507_01299_amd import api
    with pytest.raises(api.LarosaError):
        api.KvCache(1, 4, 48, 1, 1, 1, 64, "f16", device="cpu")
    z = torch.zeros(4, dtype=torch.int32)
    for kw in (dict(refs=z), dict(refs=z, table=z[:1], length=z), dict(refs=z, table=z[:2], length=z[:1].float())):
        with pytest.raises(ValueError):
            api.KvCache(1, 4, 32, 1, 2, 1, 64, "f16", device="cpu", **kw)
    with pytest.raises(ValueError):
        api.Rotary(torch.zeros(8, 64), positions=torch.zeros(2, 8, dtype=torch.int32), axis_pairs=(8, 8, 16))
    for bad in (lambda: api.Rotary(torch.zeros(8, 64, dtype=torch.float64)), lambda: api.Rotary(torch.zeros(64, 8).T),
                lambda: api.Rotary(torch.zeros(8, 64), positions=torch.zeros(1, 8)), lambda: api.KvBatch(z.long(), 4),
                lambda: api.KvBatch(z, 4, starts=z)):
        with pytest.raises(ValueError):
            bad()
    # shapes that the C call cannot see
    c = api.KvCache(1, 4, 32, 1, 4, 1, 64, "f16", data=torch.zeros(4 * 32 * 68, dtype=torch.uint8), refs=z, table=z, length=z[:1])
    b = api.KvBatch(z[:3], 3)
    few, enough, turned = torch.zeros(2, 256), torch.zeros(3, 256), torch.zeros(256, 3).T
    rot = api.Rotary(torch.zeros(8, 64), positions=torch.zeros(1, 2, dtype=torch.int32))
    for call in (lambda: api.kv4_append(c, 0, b, few, 2), lambda: api.kv4_append(c, 0, b, turned, 2), lambda: api.kv4_append(c, 0, b, enough, 2, out=few),
                 lambda: api.kv4_append(c, 0, b, enough, 2, out=enough, rotary=rot), lambda: api.kv4_attention(c, 0, b, few, 2, enough, None),
                 lambda: api.kv4_attention(c, 0, b, enough, 2, turned, None), lambda: api.layer_forward_kv4(None, c, 0, b, few, enough, None)):
        with pytest.raises(ValueError):
            call()


def cpu_cache(api):
    import torch
    z = torch.zeros(4, dtype=torch.int32)
    return api.KvCache(1, 4, 32, 4, 1, 1, 64, "f16", data=torch.zeros(4 * 32 * 68, dtype=torch.uint8), refs=z, table=z.clone(), length=z.clone())


def test_binding_refuses_lists_that_the_device_would_misread(lib):
    """64-bit, floating or strided lists, partners of another length, a status that is no int32."""
    import torch
    from paper_2507_01299_amd import api
    c = cpu_cache(api)
    ws = type("Ws", (), dict(ptr=FAKE, nbytes=BIG))
    good, status = torch.tensor([0, 1], dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    lists = [good.long(), good.short(), good.float(), torch.zeros(4, dtype=torch.int32)[::2]]
    partners = lists + [good[:1], torch.zeros(3, dtype=torch.int32)]
    calls = []
    for bad in lists:
        calls += [lambda t=bad: api.kv4_trim(c, t), lambda t=bad: api.kv4_grow(c, t, status, ws), lambda t=bad: api.kv4_fork(c, t, good, status),
                  lambda t=bad: api.kv4_copy_pages(c, t, good), lambda t=bad: api.KvBatch(t, 2)]
    for bad in partners:
        calls += [lambda t=bad: api.kv4_trim(c, good, t), lambda t=bad: api.kv4_grow(c, good, status, ws, t),
                  lambda t=bad: api.kv4_fork(c, good, t, status), lambda t=bad: api.kv4_copy_pages(c, good, t)]
    for bad in (torch.zeros(4, dtype=torch.int32)[::2], torch.zeros(4, dtype=torch.int32), torch.zeros(3)):
        calls.append(lambda t=bad: api.KvBatch(good, 2, starts=t))
    for bad in (status.long(), status[:0], status.float()):
        calls += [lambda t=bad: api.kv4_grow(c, good, t, ws), lambda t=bad: api.kv4_fork(c, good, good, t), lambda t=bad: api.kv4_compact(c, t, ws)]
    for call in calls:
        with pytest.raises(ValueError):
            call()
    api.KvBatch(good, 2, starts=torch.zeros(3, dtype=torch.int32))


def test_binding_refuses_rows_of_another_type(lib):
    """Rows of another 16-bit type than the cache's, or of 32 bits; a layer's rows that are not dense."""
    import torch
    from paper_2507_01299_amd import api
    c = cpu_cache(api)
    b = api.KvBatch(torch.tensor([0, 1, 2], dtype=torch.int32), 3)
    good = torch.zeros(3, 256, dtype=torch.float16)
    layer = type("L", (), dict(c=api._Layer(d=256)))
    for bad in (good.bfloat16(), good.float(), good.view(torch.int16)):
        for call in (lambda: api.kv4_append(c, 0, b, bad, 2), lambda: api.kv4_append(c, 0, b, good, 2, out=bad),
                     lambda: api.kv4_attention(c, 0, b, bad, 2, good, None), lambda: api.kv4_attention(c, 0, b, good, 2, bad, None),
                     lambda: api.layer_forward_kv4(layer, c, 0, b, bad, good, None), lambda: api.layer_forward_kv4(layer, c, 0, b, good, bad, None)):
            with pytest.raises(ValueError):
                call()
    for bad in (torch.zeros(3, 512, dtype=torch.float16)[:, :256], torch.zeros(3, 264, dtype=torch.float16), good.T.contiguous().T):
        for call in (lambda: api.layer_forward_kv4(layer, c, 0, b, bad, good, None), lambda: api.layer_forward_kv4(layer, c, 0, b, good, bad, None)):
            with pytest.raises(ValueError):
                call()


def plan_of(lib, C, b, heads, window=0, max_len=0):
    plan = (ctypes.c_int * 5)()
    assert lib.larosa_kv4_attention_plan(ctypes.byref(C), ctypes.byref(b), heads, window, max_len, plan) == 0
    return dict(zip(("tile_rows", "row_tiles", "chunk", "splits", "sums"), plan))


def test_sums_of_splits_start_at_16_bytes(lib):
    """Each split's sums are moved 16 bytes at a time: whole pieces for any number of rows, and the workspace holds all of them."""
    from paper_2507_01299_amd import api
    ref = ctypes.byref
    for D in (64, 128, 256):
        for kv, group, new in ((1, 1, 1), (4, 7, 1), (2, 1, 3), (1, 3, 5), (8, 4, 1), (1, 5, 3), (2, 3, 9), (1, 1, 31), (1, 4, 100)):
            for seqs, most in ((1, 2000), (3, 900), (40, 300)):
                C = cache(n_kv_heads=kv, head_dim=D, max_pages=most, n_pages=1 << 20, n_slots=64)
                b = batch(starts=FAKE, n_seq=seqs, n_rows=seqs * new, max_new=new)
                p = plan_of(lib, C, b, kv * group)
                rows = min(new * group, p["tile_rows"])
                assert p["row_tiles"] == -(-new * group // p["tile_rows"])
                assert p["sums"] % 4 == 0 and rows * (D + 2) <= p["sums"] < rows * (D + 2) + 4
                left = p["row_tiles"] * kv * seqs * p["splits"] * p["sums"] * 4 if p["splits"] > 1 else 0
                assert lib.larosa_kv4_attention_workspace_bytes(ref(C), ref(b), kv * group, 0) >= (1 << 20) + left
    bad = (ctypes.c_int * 5)()
    for args in ((None, ref(batch()), 8, 0, 0, bad), (ref(cache()), ref(batch(n_seq=0)), 8, 0, 0, bad), (ref(cache()), ref(batch()), 7, 0, 0, bad),
                 (ref(cache()), ref(batch()), 8, -1, 0, bad), (ref(cache()), ref(batch()), 8, 0, -1, bad), (ref(cache()), ref(batch()), 8, 0, 0, None)):
        assert lib.larosa_kv4_attention_plan(*args) == api.EINVAL


def test_binding_refuses_a_cache_of_another_than_the_current_device(lib, monkeypatch):
    import torch
    from paper_2507_01299_amd import api
    c = cpu_cache(api)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: c.device + 1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    ws = type("Ws", (), dict(ptr=FAKE, nbytes=BIG))
    one, status = torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    b, rows, q = api.KvBatch(one, 1), torch.zeros(1, 192, dtype=torch.float16), torch.zeros(1, 64, dtype=torch.float16)
    layer = type("L", (), dict(c=api._Layer(d=64)))
    for call in (lambda: api.kv4_clear(c), lambda: api.kv4_trim(c, one), lambda: api.kv4_grow(c, one, status, ws),
                 lambda: api.kv4_fork(c, one, one + 1, status), lambda: api.kv4_compact(c, None, ws), lambda: api.kv4_copy_pages(c, one, one + 1),
                 lambda: api.kv4_append(c, 0, b, rows, 1), lambda: api.kv4_attention(c, 0, b, rows, 1, q, ws),
                 lambda: api.layer_forward_kv4(layer, c, 0, b, q, q.clone(), ws)):
        with pytest.raises(ValueError, match="current"):
            call()


def test_data_of_2_to_the_43_bytes_is_refused(lib):
    """Bytes are counted in 64 bits and pieces of pages in 32: a product of sizes that are fine one by one may pass both."""
    from paper_2507_01299_amd import api
    ref = ctypes.byref
    page = lib.larosa_kv4_page_bytes(64, 2, 128)
    most = ((1 << 43) - 1) // page
    for layers in (1, 2, 1000, 65535):
        n = min(most // layers, 1 << 28)
        assert lib.larosa_kv4_data_bytes(ref(cache(n_layers=layers, n_pages=n))) == layers * n * page
    for sizes in (dict(n_layers=2, n_pages=1 << 28), dict(n_layers=1000, n_pages=most // 1000 + 1),
                  dict(n_layers=65535, n_pages=1 << 28, n_kv_heads=4096, head_dim=256, page_tokens=256),
                  # 2^64 + 2^54 bytes and the like: what is left of them in 64 bits would look modest
                  dict(n_layers=4096, n_pages=(1 << 28) - 1, n_kv_heads=4096, head_dim=256, page_tokens=256),
                  dict(n_layers=61681, n_pages=17 * (1 << 22), n_kv_heads=1 << 12, head_dim=256, page_tokens=32)):
        C = cache(**sizes)
        assert lib.larosa_kv4_data_bytes(ref(C)) == 0, sizes
        assert lib.larosa_kv4_clear(ref(C), None) == api.EUNSUPPORTED
        assert lib.larosa_kv4_pages_workspace_bytes(ref(C)) == 0
        assert lib.larosa_kv4_copy_pages(ref(C), FAKE, OTHER, 1, None) == api.EUNSUPPORTED
