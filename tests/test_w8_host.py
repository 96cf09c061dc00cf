"""Host-side checks of the entry points on 8-bit weights and of the log probabilities that need no GPU: sizes, and refusals before a device
is touched."""
import os

import pytest
import torch

P, ODD = 0x10000, 0x10004           # never dereferenced: checks fail first
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    from paper_2507_01299_amd import api, build
    if not os.path.exists(api.LIB_PATH):
        build.build_library()
    return api.lib()


def call(fn, defaults, **kw):
    unknown = set(kw) - set(defaults)
    assert not unknown, unknown
    return fn(*{**defaults, **kw}.values())


WEIGHT = dict(W=P, d_in=256, d_out=512, t=1, codes=P, scales=P, stream=None)
ROWS = dict(x=P, ld_x=256, n_rows=5, d=256, rms=None, rms_eps=-1.0, t=1, codes=P, scales=P, stream=None)
PRODUCT = dict(wc=P, ws=P, xc=P, xs=P, y=P, ld_y=512, n_rows=5, d_in=256, d_out=512, t=1, work=P, bytes=1 << 40, stream=None)
DENSE = dict(wc=P, ws=P, x=P, ld_x=256, rms=None, rms_eps=-1.0, y=P, ld_y=512, n_rows=5, d_in=256, d_out=512, t=1, work=P,
             bytes=1 << 40, stream=None)
LOGPROBS = dict(logits=P, ld=1000, n_rows=5, n_vocab=1000, t=1, scale=1.0, given=P, n_given=2, logp=P, entropy=P, n_top=3, top_id=P,
                top_logp=P, work=P, bytes=1 << 40, stream=None)
SCORE = dict(wc=P, ws=P, x=P, ld_x=256, rms=None, rms_eps=-1.0, n_rows=5, d_in=256, n_vocab=1001, t=1, scale=1.0, given=P, n_given=2,
             logp=P, entropy=P, n_top=3, top_id=P, top_logp=P, work=P, bytes=1 << 40, stream=None)


@pytest.mark.parametrize("kw", [dict(W=None), dict(W=ODD), dict(codes=None), dict(codes=ODD), dict(scales=None), dict(scales=P + 2),
                                dict(d_in=0), dict(d_in=12), dict(d_out=0), dict(d_out=-8), dict(d_out=12), dict(t=2), dict(t=7)])
def test_weight_refusals(lib, kw):
    assert call(lib.larosa_quantize_w8, WEIGHT, **kw) == EINVAL


def test_weight_beyond_the_kernels(lib):
    assert call(lib.larosa_quantize_w8, WEIGHT, d_in=(1 << 20) + 8) == EUNSUPPORTED
    assert call(lib.larosa_quantize_w8, WEIGHT, d_out=1 << 21) == EUNSUPPORTED


@pytest.mark.parametrize("kw", [dict(x=None), dict(x=ODD), dict(ld_x=248), dict(ld_x=260), dict(n_rows=0), dict(d=0), dict(d=20), dict(rms=ODD),
                                dict(rms_eps=float("nan")), dict(t=2), dict(codes=ODD), dict(scales=None)])
def test_rows_refusals(lib, kw):
    assert call(lib.larosa_quantize_rows8, ROWS, **kw) == EINVAL


def test_rows_beyond_the_kernels(lib):
    assert call(lib.larosa_quantize_rows8, ROWS, n_rows=(1 << 24) + 1) == EUNSUPPORTED
    assert call(lib.larosa_quantize_rows8, ROWS, d=(1 << 20) + 8, ld_x=(1 << 20) + 8) == EUNSUPPORTED


@pytest.mark.parametrize("kw", [dict(wc=None), dict(wc=ODD), dict(ws=None), dict(xc=ODD), dict(xs=P + 1), dict(y=None), dict(y=ODD), dict(ld_y=504),
                                dict(ld_y=516), dict(n_rows=0), dict(d_in=4), dict(d_out=12, ld_y=512), dict(d_out=0), dict(t=2)])
def test_product_refusals(lib, kw):
    assert call(lib.larosa_product8, PRODUCT, **kw) == EINVAL


@pytest.mark.parametrize("kw", [dict(x=None), dict(x=ODD), dict(ld_x=128), dict(rms=ODD), dict(rms_eps=float("nan")), dict(y=ODD), dict(ld_y=505),
                                dict(n_rows=-1), dict(d_in=9), dict(d_out=20), dict(t=2), dict(wc=ODD)])
def test_dense_refusals(lib, kw):
    assert call(lib.larosa_dense_w8, DENSE, **kw) == EINVAL


@pytest.mark.parametrize("kw", [dict(logits=None), dict(logits=P + 1), dict(logits=P + 2, t=2), dict(ld=999), dict(n_rows=0), dict(n_vocab=0), dict(t=3),
                                dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(given=None),
                                dict(logp=None), dict(n_given=-1), dict(n_top=-1), dict(top_id=None), dict(n_top=1001), dict(entropy=P + 2),
                                dict(top_logp=P + 1)])
def test_logprobs_refusals(lib, kw):
    assert call(lib.larosa_logprobs, LOGPROBS, **kw) == EINVAL


def test_logprobs_beyond_the_kernels(lib):
    assert call(lib.larosa_logprobs, LOGPROBS, n_top=65) == EUNSUPPORTED
    assert call(lib.larosa_logprobs, LOGPROBS, n_rows=(1 << 24) + 1) == EUNSUPPORTED
    assert call(lib.larosa_logprobs, LOGPROBS, n_vocab=(1 << 28) + 1, ld=(1 << 28) + 1) == EUNSUPPORTED


@pytest.mark.parametrize("kw", [dict(x=ODD), dict(ld_x=252), dict(rms_eps=float("nan")), dict(n_vocab=0), dict(scale=0.0), dict(given=None), dict(t=2),
                                dict(n_top=-2), dict(ws=P + 2), dict(top_id=None)])
def test_score_refusals(lib, kw):
    assert call(lib.larosa_score_w8, SCORE, **kw) == EINVAL


@pytest.mark.parametrize("name,defaults,sizes", [
    ("product8", PRODUCT, (5, 256, 512)), ("product8", dict(PRODUCT, n_rows=100), (100, 256, 512)), ("dense_w8", DENSE, (5, 256, 512)),
    ("logprobs", LOGPROBS, (5, 1000, 3, 1)), ("score_w8", SCORE, (5, 256, 1001, 3))])
def test_workspaces(lib, name, defaults, sizes):
    need = getattr(lib, f"larosa_{name}_workspace_bytes")(*sizes)
    assert need >= 1 << 20
    fn = getattr(lib, f"larosa_{name}")
    assert call(fn, defaults, bytes=need - 1) == EWORKSPACE
    assert call(fn, defaults, work=None) == EWORKSPACE
    assert call(fn, defaults, work=P + 16) == EWORKSPACE


def test_workspace_of_refused_sizes_is_zero(lib):
    for sizes in ((0, 256, 512), (5, 12, 512), (5, 256, 0), (5, (1 << 20) + 8, 512), (1 << 24, 256, 1 << 20)):
        assert lib.larosa_product8_workspace_bytes(*sizes) == 0
        assert lib.larosa_dense_w8_workspace_bytes(*sizes) == 0
        assert lib.larosa_score_w8_workspace_bytes(*sizes, 0) == 0
    for sizes in ((0, 10, 0, 1), (1, 0, 0, 1), (1, 10, 11, 1), (1, 100, 65, 1), (1, 10, -1, 1), (1, 10, 0, 9)):
        assert lib.larosa_logprobs_workspace_bytes(*sizes) == 0


def test_a_score_needs_room_for_its_last_part_too(lib):
    """Parts of the rows are divided by themselves: the query covers every part of every number of rows."""
    for rows in (1, 16, 17, 255, 256, 257, 511, 700):
        whole = lib.larosa_score_w8_workspace_bytes(rows, 4096, 128256, 20)
        assert whole >= (1 << 20) + rows * (4096 + 32)


@pytest.mark.parametrize("whole,tail,d,V,top,parts,slices", [
    (1024, 17, 128, 32000, 20, False, True),         # of the logits of 17 rows each goes in slices, of 1024 none
    (4096, 17, 8192, 8000, 0, True, False)])         # of the products of 17 rows the sums go in parts, of 4096 none
def test_room_for_the_last_part_of_a_score(lib, whole, tail, d, V, top, parts, slices):
    """Worked out by hand: counters, the whole part's rows and logits, and what only the last part asks for.  A workspace that lacks the latter is
    refused."""
    partial = lib.larosa_product8_workspace_bytes(tail, d, V) - (1 << 20)
    probs = lib.larosa_logprobs_workspace_bytes(tail, V, top, 2) - (1 << 20)
    assert (partial > 0, probs > 0) == (parts, slices)
    need = (1 << 20) + whole * d + whole * -(-d // 512) * 4 + partial + whole * V * 4 + probs
    assert lib.larosa_score_w8_workspace_bytes(whole + tail, d, V, top) >= need
    sizes = dict(ld_x=d, n_rows=whole + tail, d_in=d, n_vocab=V, n_top=top)
    assert call(lib.larosa_score_w8, SCORE, bytes=need - 1, **sizes) == EWORKSPACE


def test_a_workspace_serves_smaller_numbers_of_rows(lib):
    """Fewer rows go in more slices and parts; the query covers them, so one workspace for the largest batch does."""
    for name, sizes, rows in (("logprobs", (128256, 20, 1), (1, 7, 64, 127, 128, 200, 511, 512, 600, 2048, 300000)),
                              ("logprobs", (50257, 0, 2), (1, 2, 3, 5, 77, 127, 128, 129, 513)),
                              ("product8", (11008, 4096), (1, 16, 17, 40, 100, 200, 333, 700, 1024, 4096, 32768, 1 << 17)),
                              ("dense_w8", (8192, 264), (1, 17, 64, 65, 300, 2000, 40000)),
                              ("score_w8", (8192, 32000, 20), (1, 5, 17, 100, 600, 1024, 1041, 2048, 5000))):
        query = getattr(lib, f"larosa_{name}_workspace_bytes")
        answers = [query(n, *sizes) for n in rows]
        assert answers == sorted(answers), (name, sizes, answers)
        assert answers[0] >= 1 << 20


def test_binding_refuses_what_would_be_misread():
    from paper_2507_01299_amd import api
    codes, scales = torch.empty(256, 128, dtype=torch.float8_e4m3fn), torch.empty(2, 4, dtype=torch.uint8)
    assert api._held8(codes, scales, 128, 128, -1) == (codes.data_ptr(), scales.data_ptr())
    for c, s, d in ((codes.float(), scales, 128), (codes, scales.int(), 128), (codes, scales, 256), (codes[:, ::2], scales, 64),
                    (codes[:200], torch.empty(1, 4, dtype=torch.uint8), 128)):
        with pytest.raises(ValueError):
            api._held8(c, s, d, 128, -1)
    with pytest.raises(ValueError):
        api._held8(codes, scales, 128, 128, 0)
    x = torch.empty(4, 64, dtype=torch.float16)
    assert api._matrix16(x, api.F16) == 64 and api._matrix16(x[:, :16], api.F16) == 64 and api._matrix16(x[:1, :16], api.F16) == 64
    for bad in (x.float(), x.t(), x.reshape(-1), x[:, ::2]):
        with pytest.raises(ValueError):
            api._matrix16(bad, api.F16)
    with pytest.raises(ValueError):
        api._norm8(torch.empty(8, dtype=torch.bfloat16), 16, api.BF16)
    given, logp = torch.empty(4, 2, dtype=torch.int32), torch.empty(4, 2)
    assert api._outputs8(4, given, logp, None, None, None) == (2, 0)
    for args in ((given.long(), logp, None, None, None), (given, logp.half(), None, None, None), (given, logp[:3], None, None, None),
                 (given, logp, torch.empty(3), None, None), (given, logp, None, torch.empty(4, 3), None),
                 (given, logp, None, torch.empty(4, 3, dtype=torch.int32), torch.empty(4, 2)), (given, None, None, None, None)):
        with pytest.raises(ValueError):
            api._outputs8(4, *args)


def test_tiles_that_there_are(lib):
    """Each tile's workspace query answers, also where sums go in parts; others are refused."""
    for bad in (-1, 6):
        assert lib.larosa_set_tuning(11, bad) == EINVAL
    try:
        for tile in range(6):
            assert lib.larosa_set_tuning(11, tile) == 0
            for n, d_in, d_out in ((17, 8, 8), (40, 4096, 264), (333, 11008, 4096), (1 << 14, 4096, 1 << 20)):
                assert lib.larosa_product8_workspace_bytes(n, d_in, d_out) > 0
    finally:
        lib.larosa_set_tuning(11, 0)


def test_scales_whose_exponent_would_overflow_are_refused(lib):
    """scale / ln 2 leaves fp32 from 2.4e38 on, and infinity times the difference of two equal logits is NaN."""
    for scale in (3e38, 2.4e38, 1.0000001 * 2.0 ** 126):
        assert call(lib.larosa_logprobs, LOGPROBS, scale=scale) == EUNSUPPORTED
        assert call(lib.larosa_score_w8, SCORE, scale=scale) == EUNSUPPORTED
    assert call(lib.larosa_logprobs, LOGPROBS, scale=2.0 ** 126, work=None) == EWORKSPACE


def test_a_tile_that_would_be_too_many_is_refused(lib):
    """2^23 tiles of 128 x 128 are 2^24 of 128 x 64: with that tile asked for there is no plan, neither for the query nor for the call."""
    sizes = dict(n_rows=1 << 17, d_in=256, d_out=1 << 20, ld_y=1 << 20)
    try:
        for tile in (0, 1, 2, 3, 4):
            assert lib.larosa_set_tuning(11, tile) == 0
            assert lib.larosa_product8_workspace_bytes(1 << 17, 256, 1 << 20) > 0
        assert lib.larosa_set_tuning(11, 5) == 0
        assert lib.larosa_product8_workspace_bytes(1 << 17, 256, 1 << 20) == 0
        assert lib.larosa_dense_w8_workspace_bytes(1 << 17, 256, 1 << 20) == 0
        assert call(lib.larosa_product8, PRODUCT, **sizes) == EUNSUPPORTED
        assert call(lib.larosa_dense_w8, DENSE, **sizes) == EUNSUPPORTED
        assert lib.larosa_product8_workspace_bytes(1 << 16, 256, 1 << 20) > 0
        assert lib.larosa_product8_workspace_bytes(16, 256, 1 << 20) > 0
    finally:
        lib.larosa_set_tuning(11, 0)


def test_log_probabilities_take_the_same_room_for_every_type(lib):
    for n, V, top in ((1, 32000, 5), (77, 50257, 8), (300, 128256, 0), (5, 300000, 64)):
        assert len({lib.larosa_logprobs_workspace_bytes(n, V, top, t) for t in (0, 1, 2)}) == 1


def strided(shape, stride, dtype=torch.float16):
    """A matrix that takes no memory."""
    return torch.empty_strided(shape, stride, dtype=dtype, device="meta")


@pytest.mark.parametrize("shape,stride", [((2, 8), ((1 << 32) + 8, 1)), ((3, 64), ((1 << 31) + 64, 1)), (((1 << 32) + 5, 8), (8, 1)),
                                          ((1, (1 << 32) + 64), ((1 << 32) + 64, 1)), ((1 << 31, 8), (8, 1))])
def test_sizes_beyond_32_bits_are_refused(shape, stride):
    """In an int argument 2^32 + 8 arrives as 8: rows of a wide tensor, such as the last token's logits of a long batch, would be read from
    other places."""
    from paper_2507_01299_amd import api
    with pytest.raises(ValueError):
        api._matrix16(strided(shape, stride), api.F16)
    with pytest.raises(ValueError):
        api._logits(strided(shape, stride, torch.float32))


def test_one_row_of_a_matrix_of_any_distance():
    """What a single row's tensor says of the distance to the next one counts for nothing."""
    from paper_2507_01299_amd import api
    for ld in (1, 64, 1001, 1 << 21, (1 << 31) + 4, (1 << 32) + 64):
        one = api._matrix16(strided((1, 64), (ld, 1)), api.F16)
        assert one % 8 == 0 and 64 <= one < 1 << 21
        assert api._logits(strided((1, 65), (ld, 1), torch.bfloat16)) == (65, api.BF16)
    assert api._matrix16(strided((2, 64), ((1 << 31) - 8, 1)), api.F16) == (1 << 31) - 8
    assert api._logits(strided((2, 1), (7, 5))) == (7, api.F16)
    for bad in (strided((2, 64), (64, 2)), strided((2, 64, 1), (64, 1, 1)), strided((2, 64), (64, 1), torch.float64)):
        with pytest.raises(ValueError):
            api._logits(bad)


@pytest.mark.parametrize("eps", [None, -1.0, -1e-5, float("nan")])
def test_a_norms_scale_without_a_norm_is_refused(monkeypatch, eps):
    """rms given and rms_eps left at "no norm": the scale would be dropped in silence."""
    from paper_2507_01299_amd import api

    class Library:
        def __getattr__(self, name):
            def called(*args):
                raise AssertionError(f"{name} was called")
            return called
    monkeypatch.setattr(api, "_device_stream", lambda *tensors: (-1, None))
    monkeypatch.setattr(api, "lib", Library)
    x, rms, y = torch.empty(2, 128, dtype=torch.float16), torch.empty(128, dtype=torch.float16), torch.empty(2, 256, dtype=torch.float16)
    codes, scales = torch.empty(256, 128, dtype=torch.float8_e4m3fn), torch.empty(2, 4, dtype=torch.uint8)

    class Work:
        buf, ptr, nbytes = None, 0, 0
    kw = dict(rms=rms) if eps is None else dict(rms=rms, rms_eps=eps)
    for call in (lambda: api.quantize_rows8(x, "f16", **kw), lambda: api.dense_w8(codes, scales, x, y, "f16", Work, **kw),
                 lambda: api.score_w8(codes, scales, x, torch.empty(2, 1, dtype=torch.int32), torch.empty(2, 1), "f16", Work, **kw)):
        with pytest.raises(ValueError):
            call()
