"""GPU parity, through the C ABI, of log probabilities, entropy and top alternatives, and of the whole way from hidden rows to them."""
import numpy as np
import pytest
import torch

from oracle import w8_oracle as Q

pytestmark = pytest.mark.gpu
TYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
# A lane adds at most 128 exponentials one by one, the rest in a tree: the sum is off by at most 150 roundings (2^-24) of itself, and as
# much again from the exponentials (an ulp of exp2; an exponent u is rounded by |u| 2^-23, and |u| 2^u < 0.54).
SUM = 3e-5
REL = 2.0 ** -22            # difference to the largest logit, its product with the scale, the last subtraction


@pytest.fixture(scope="module")
def api(gpu_device):
    from paper_2507_01299_amd import api as A
    A.lib()
    return A


def run(api, logits, given, n_top, scale=1.0, entropy=True):
    n, V = logits.shape
    dev = lambda *s, t=torch.float32: torch.full(s, -55, dtype=t, device="cuda")     # noqa: E731
    g = torch.as_tensor(given, dtype=torch.int32).cuda()
    logp, ent = dev(n, g.shape[1]), dev(n) if entropy else None
    ids, tops = (dev(n, n_top, t=torch.int32), dev(n, n_top)) if n_top else (None, None)
    ws = api.logprobs_workspace(n, V, n_top, logits.dtype)
    api.logprobs(logits, g, logp, ws, entropy=ent, top_id=ids, top_logp=tops, scale=scale)
    assert int(ws.buf[ws.ptr - ws.buf.data_ptr():][:1 << 20].count_nonzero()) == 0
    out = [t.double().cpu().numpy() if t is not None else None for t in (logp, ent)]
    return out + [ids.cpu().numpy() if n_top else np.zeros((n, 0)), tops.double().cpu().numpy() if n_top else np.zeros((n, 0))]


def near(got, want, rel=REL):
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
    fine = np.isfinite(want)
    assert np.all(got[np.isinf(want)] == want[np.isinf(want)])
    off = np.abs(got - want)[fine]
    assert np.all(off <= SUM + rel * np.abs(want[fine])), off.max()


def check(api, logits, given, n_top, scale=1.0):
    got = run(api, logits, given, n_top, scale)
    want = Q.logprobs(logits.double().cpu().numpy(), np.asarray(given), n_top, scale)
    # the difference of two logits is rounded against the largest of them
    with np.errstate(invalid="ignore"):
        near(got[0], want[0])
        near(got[1], want[1], rel=SUM)
        near(got[3], want[3])
    assert np.array_equal(got[2], want[2])
    return got, want


def draw(n, V, seed, dtype, masked=0.0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(n, V, generator=g) * 3
    z += torch.where(torch.rand(n, V, generator=g) < 3 / V, 9.0, 0.0)
    if masked:
        z.masked_fill_(torch.rand(n, V, generator=g) < masked, -float("inf"))
    given = torch.randint(V, (n, 3), generator=g)
    given[0, 0] = -1
    return z.to(TYPE[dtype]).cuda(), given


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("n,V,top", [(1, 1, 1), (2, 2, 2), (3, 7, 3), (1, 8, 8), (5, 9, 4), (2, 63, 63), (3, 64, 64), (2, 65, 64), (1, 2047, 5), (1, 2048, 64),
                                     (4, 2049, 1), (1, 5000, 20), (3, 16383, 7), (2, 16385, 33), (1, 32000, 5), (600, 333, 2), (513, 4099, 9)])
def test_against_the_oracle(api, dtype, n, V, top):
    print(f"logprobs {dtype} {n}x{V} top {top}", flush=True)
    check(api, *draw(n, V, n * 31 + V, dtype), top)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("V,masked", [(32767, 0.0), (32769, 0.5), (50257, 0.4), (70001, 0.999), (131073, 0.0), (200003, 0.2)])
def test_long_rows(api, dtype, V, masked):
    print(f"logprobs {dtype} 3x{V}", flush=True)
    check(api, *draw(3, V, V, dtype, masked), 20)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_many_rows_of_several_slices(api, dtype):
    """Rows enough that a slice is as long as it gets, and each row has several."""
    z, given = draw(180, 66000, 4, dtype)
    check(api, z, given, 12)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("V,ld,first", [(1000, 1001, 0), (1000, 1003, 5), (33001, 33003, 1), (777, 777, 3), (6, 7, 2)])
def test_rows_at_any_alignment(api, dtype, V, ld, first):
    n = 9
    whole = torch.full((n * ld + first,), float("nan"), dtype=TYPE[dtype], device="cuda")      # what lies between the rows counts for nothing
    rows = whole[first:].view(n, ld)[:, :V]
    z, given = draw(n, V, ld, dtype)
    rows.copy_(z)
    check(api, rows, given, min(V, 6))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("V", [300, 9000, 40000])
def test_ties_and_orders(api, dtype, V):
    """All equal, two values only, rising, falling, -0 beside 0: the order of the logits changes nothing, ties go to the lower id."""
    z = torch.zeros(6, V)
    z[1] = torch.randint(0, 2, (V,), generator=torch.Generator().manual_seed(1)).float()
    z[2] = torch.arange(V) / 256.0
    z[3] = -torch.arange(V) / 256.0
    z[4, ::2] = -0.0
    z[5] = -3.0
    z[5, -7:] = 2.0
    check(api, z.to(TYPE[dtype]).cuda(), torch.tensor([[0, V - 1, V // 2]] * 6), 64)


@pytest.mark.parametrize("V", [50, 3000, 33000])
def test_masks_that_leave_little_or_nothing(api, V):
    inf = float("inf")
    z = torch.randn(8, V, generator=torch.Generator().manual_seed(V)) * 2
    z[0] = -inf
    z[1] = -inf
    z[1, V - 1] = -4.0
    z[2, : V // 2] = -inf
    z[3, 1:] = torch.finfo(torch.bfloat16).min               # a mask by the type's lowest value
    z[4, 17] = float("nan")
    z[5, V - 3] = inf
    z[6] = torch.finfo(torch.bfloat16).min                   # nothing but it: all alike
    z[7] = -inf
    z[7, 5:9] = 1.0
    given = torch.tensor([[0, V - 1, 6, -1, V]] * 8)
    for dtype in ("bf16", "f32"):
        check(api, z.to(TYPE[dtype]).cuda(), given, 6)


def test_sure_rows_keep_their_bits(api):
    """Where one token holds nearly all of the probability, its log probability is minus the sum of the others, to that sum's own precision."""
    V = 40000
    z = torch.zeros(5, V)
    for r, m in enumerate((20.0, 25.0, 30.0, 40.0, 60.0)):
        z[r, 1000 * r + 3] = m
    given = torch.tensor([[1000 * r + 3, 0] for r in range(5)])
    for dtype in ("f32", "bf16"):
        got, want = check(api, z.to(TYPE[dtype]).cuda(), given, 1)
        assert np.all(np.abs(got[0][:, 0] - want[0][:, 0]) <= SUM * np.abs(want[0][:, 0]))
        assert np.all(np.abs(got[1] - want[1]) <= 2 * SUM * want[1])


@pytest.mark.parametrize("scale", [0.25, 1 / 0.7, 8.0])
def test_scale(api, scale):
    s = float(np.float32(scale))
    for dtype in ("f16", "f32"):
        z, given = draw(5, 20011, 3, dtype, 0.1)
        check(api, z, given, 9, s)


@pytest.mark.parametrize("scale", [2.0 ** 126, 1e30, 2.0 ** -126, 1e-42])
@pytest.mark.parametrize("V", [50, 33000])
def test_extreme_scales(api, V, scale):
    """Next to the largest scale only the largest logit's equals count, next to 0 all logits count alike."""
    s = float(np.float32(scale))
    z = -torch.randint(0, 3, (4, V), generator=torch.Generator().manual_seed(V)).float()
    z[1, ::3] = -float("inf")
    z[2, 7] = 1.0
    z[3] = -float("inf")
    for dtype in ("bf16", "f32"):
        check(api, z.to(TYPE[dtype]).cuda(), torch.tensor([[0, 1, 7, V - 1]] * 4), 6, s)


def test_what_is_not_asked_for(api):
    z, given = draw(4, 5000, 8, "bf16")
    assert run(api, z, given[:, :0], 0)[0].shape == (4, 0)
    full = run(api, z, given, 3)
    assert np.array_equal(run(api, z, given, 0, entropy=False)[0], full[0])
    ids = torch.zeros(4, 3, dtype=torch.int32, device="cuda")
    api.logprobs(z, None, None, api.logprobs_workspace(4, 5000, 3), top_id=ids)
    assert np.array_equal(ids.cpu().numpy(), full[2])
    many = torch.randint(-2, 5003, (4, 300), generator=torch.Generator().manual_seed(1))
    check(api, z, many, 0)


def test_rows_by_the_launch(api):
    """More rows than one launch has counters for."""
    n, V = (1 << 18) + 77, 24
    z = torch.randn(n, V, device="cuda", generator=torch.Generator("cuda").manual_seed(2)).bfloat16()
    given = torch.randint(V, (n, 1), device="cuda", generator=torch.Generator("cuda").manual_seed(3)).int()
    logp, ids = torch.empty(n, 1, device="cuda"), torch.empty(n, 2, dtype=torch.int32, device="cuda")
    api.logprobs(z, given, logp, api.logprobs_workspace(n, V, 2), top_id=ids)
    p = z.double().log_softmax(-1)
    assert float((logp.double() - p.gather(1, given.long())).abs().max()) < SUM
    assert torch.equal(ids.long(), z.float().sort(dim=-1, descending=True, stable=True).indices[:, :2])


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("top", [1, 20, 64])
def test_alike_logits_of_many_rows(api, dtype, top):
    """Rows enough that none is cut, with more groups of 128 logits at the border than a wave has lanes: all alike, two values, a few above many."""
    n, V = 130, 20011
    z = torch.zeros(n, V)
    z[1::3] = torch.randint(0, 2, (len(z[1::3]), V), generator=torch.Generator().manual_seed(top)).float()
    z[2::3, ::999] = 1.0
    z[2::3, 5] = -float("inf")
    given = torch.arange(2 * n).view(n, 2)
    check(api, z.to(TYPE[dtype]).cuda(), given, top)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("n,V,top", [(520, 140003, 64), (520, 270001, 9), (3, 300007, 64), (2, 1 << 20, 5)])
def test_vocabularies_beyond_a_slice(api, dtype, n, V, top):
    """Rows that are not cut though long (more groups than are read at once), and rows that have to be: more than 262137 tokens.  Few values, so that
    equal ones lie everywhere.  Against 64 bits on the GPU.  A lane adds at most V / (256 slices) exponentials, in runs of 32: within SUM."""
    print(f"logprobs {dtype} {n}x{V} top {top}", flush=True)
    g = torch.Generator("cuda").manual_seed(V)
    z = (torch.randint(-40, 9, (n, V), generator=g, device="cuda") / 4).to(TYPE[dtype])
    z[0] = 1.0
    given = torch.randint(V, (n, 2), generator=g, device="cuda").int()
    logp, entropy = torch.empty(n, 2, device="cuda"), torch.empty(n, device="cuda")
    ids, tops = torch.empty(n, top, dtype=torch.int32, device="cuda"), torch.empty(n, top, device="cuda")
    ws = Guarded(api, api.lib().larosa_logprobs_workspace_bytes(n, V, top, api.F32))
    api.logprobs(z, given, logp, ws, entropy=entropy, top_id=ids, top_logp=tops)
    assert ws.whole()
    for r in range(0, n, 130):
        p = z[r:r + 130].double().log_softmax(-1)
        best = z[r:r + 130].float().sort(dim=-1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(ids[r:r + 130].long(), best)
        for got, want in ((logp, p.gather(1, given[r:r + 130].long())), (tops, p.gather(1, best))):
            assert bool(((got[r:r + 130].double() - want).abs() <= SUM + REL * want.abs()).all())
        want = -(p.exp() * p).sum(-1)
        assert bool(((entropy[r:r + 130].double() - want).abs() <= SUM + SUM * want).all())


def test_two_streams_and_replays(api):
    z, given = draw(6, 60000, 12, "f16")
    given = given.int().cuda()
    other = torch.cuda.Stream()
    jobs = []
    for i in range(2):
        jobs.append(dict(logp=torch.empty(6, 3, device="cuda"), entropy=torch.empty(6, device="cuda"), top_id=torch.empty(6, 20, dtype=torch.int32, device="cuda"),
                         top_logp=torch.empty(6, 20, device="cuda"), ws=api.logprobs_workspace(6, 60000, 20, "f16")))
    torch.cuda.synchronize()
    for _ in range(5):
        api.logprobs(z, given, **jobs[0])
        with torch.cuda.stream(other):
            api.logprobs(z, given, **jobs[1])
    torch.cuda.synchronize()
    for k in ("logp", "entropy", "top_id", "top_logp"):
        assert torch.equal(jobs[0][k], jobs[1][k])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.logprobs(z, given, **jobs[0])
    for i in range(4):
        z.copy_(draw(6, 60000, 100 + i, "f16")[0])
        graph.replay()
        api.logprobs(z, given, **jobs[1])
        torch.cuda.synchronize()
        for k in ("logp", "entropy", "top_id", "top_logp"):
            assert torch.equal(jobs[0][k], jobs[1][k])


class Guarded:
    """A workspace of just the bytes that a query asks for, with a pattern behind them."""

    def __init__(self, api, need):
        self.nbytes = need
        self.buf = torch.full((need + 256 + 65536,), 0xA5, dtype=torch.uint8, device="cuda")
        self.ptr = self.buf.data_ptr() + (-self.buf.data_ptr()) % 256
        assert api.lib().larosa_workspace_init(self.ptr, need, torch.cuda.current_stream().cuda_stream) == 0

    def whole(self):
        behind = self.buf[self.ptr - self.buf.data_ptr() + self.nbytes:]
        return bool((behind == 0xA5).all())


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_one_workspace_for_every_batch(api, dtype):
    """Sized for the most rows, used for fewer, which go in more slices."""
    V, top = 50257, 20
    z, given = draw(600, V, 5, dtype)
    ws = Guarded(api, api.lib().larosa_logprobs_workspace_bytes(600, V, top, api.F32 if dtype == "f32" else api.F16))
    for n in (600, 1, 7, 127, 128, 200, 511):
        ids, tops = torch.empty(n, top, dtype=torch.int32, device="cuda"), torch.empty(n, top, device="cuda")
        logp, entropy = torch.empty(n, 3, device="cuda"), torch.empty(n, device="cuda")
        api.logprobs(z[:n], given[:n].int().cuda(), logp, ws, entropy=entropy, top_id=ids, top_logp=tops)
        want = run(api, z[:n], given[:n], top)
        for got, w in zip((logp, entropy, ids, tops), want):
            assert np.array_equal(got.double().cpu().numpy(), w)
        assert ws.whole()


# ---- from hidden rows to log probabilities ---------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,d,V,top", [(1, 128, 1000, 5), (3, 520, 2011, 0), (16, 256, 4099, 9), (40, 264, 3001, 4), (150, 136, 5003, 3), (700, 256, 64007, 2)])
def test_score(api, dtype, n, d, V, top):
    """Logits are off by the product's bound b (2^-10 of the sum of magnitudes where the 8-bit instruction adds them, see test_gpu_w8.CUT), so log probabilities
    are within 2 b, the entropy within 2 b (1 + ln V), and a top token's logit is within 2 b of the one that belongs there."""
    print(f"score {dtype} {n}x{d}x{V}", flush=True)
    g = torch.Generator().manual_seed(V)
    x = torch.randn(n, d, generator=g).to(TYPE[dtype])
    wide = torch.randn(d, V + (-V % 8), generator=g) * 0.3
    wc, ws = Q.quantize_weight(wide.to(TYPE[dtype]).double().numpy()[:, :V])
    given = torch.randint(V, (n, 2), generator=g).int()
    given[-1, 1] = -1
    logp, entropy = torch.full((n, 2), 9.0, device="cuda"), torch.empty(n, device="cuda")
    ids, tops = (torch.empty(n, top, dtype=torch.int32, device="cuda"), torch.empty(n, top, device="cuda")) if top else (None, None)
    work = api.score_w8_workspace(n, d, V, top)
    head = torch.from_numpy(wc).view(torch.float8_e4m3fn).cuda(), torch.from_numpy(ws).cuda()
    api.score_w8(*head, x.cuda(), given.cuda(), logp, dtype, work, entropy=entropy, top_id=ids, top_logp=tops, scale=0.5)
    z, most = Q.product(wc, ws, *Q.quantize_rows(x.double().numpy()), d)
    want = Q.logprobs(z, given.numpy(), top, 0.5)
    b = 0.5 * most.max() * ((d + 8) * 2.0 ** -24 + (0 if n <= 16 else 2.0 ** -10)) + SUM
    assert np.all(np.abs(logp.double().cpu().numpy() - want[0]) <= 2 * b + REL * np.abs(want[0]))
    assert np.all(np.abs(entropy.double().cpu().numpy() - want[1]) <= 2 * b * (1 + np.log(V)))
    if top:
        got = ids.cpu().numpy()
        assert all(len(set(r)) == top for r in got.tolist())
        assert np.all(np.abs(np.take_along_axis(z, got, 1) - np.take_along_axis(z, want[2], 1)) * 0.5 <= 2 * b)
        assert np.all(np.abs(tops.double().cpu().numpy() - want[3]) <= 4 * b + REL * np.abs(want[3]))


@pytest.mark.parametrize("tile", range(6))
@pytest.mark.parametrize("n,d,V", [(17, 128, 1), (40, 264, 127), (33, 4104, 129), (150, 136, 5003), (300, 128, 100003), (1100, 64, 32001)])
def test_score_without_alternatives(api, tile, n, d, V):
    """With and without alternatives, whatever the tile and the number of given tokens: the same products, so the same logits.  A row of NaN stays alone; ids
    that are padding, beyond the vocabulary, the same twice."""
    print(f"score without alternatives {tile} {n}x{d}x{V}", flush=True)
    g = torch.Generator().manual_seed(n + V)
    x = torch.randn(n, d, generator=g).bfloat16().cuda()
    x[n // 2, d - 1] = float("nan")
    head = api.quantize_rows8((torch.randn(V, d, generator=g) * 0.5).bfloat16().cuda(), "bf16")[0], torch.full((-(-V // 128), -(-d // 512) * 4), 127, dtype=torch.uint8, device="cuda")
    given = torch.randint(V, (n, 5), generator=g).int()
    given[:, 1] = V - 1
    given[3] = torch.tensor([-1, V, 0, 0, V // 2])
    given[4, 2] = -2 ** 31
    given[4, 3] = 2 ** 31 - 1
    try:
        api.set_tuning(11, tile)
        work = api.score_w8_workspace(n, d, V, 1)
        kept = [torch.full((n, 5), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")]
        api.score_w8(*head, x, given.cuda(), kept[0], "bf16", work, entropy=kept[1], top_id=torch.empty(n, 1, dtype=torch.int32, device="cuda"), scale=0.7)
        work = api.score_w8_workspace(n, d, V)
        for few in (4, 1, 0, 5):
            logp, entropy = torch.full((n, few), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
            api.score_w8(*head, x, given[:, :few].contiguous().cuda(), logp, "bf16", work, entropy=entropy, scale=0.7)
            for got, want in ((logp, kept[0][:, :few]), (entropy, kept[1])):
                assert torch.equal(got.isnan(), want.isnan())
                got, want = got.double().nan_to_num(nan=0.0), want.double().nan_to_num(nan=0.0)
                assert bool(((got - want).abs() <= 2 * (SUM + REL * want.abs())).all())
            if few:
                api.score_w8(*head, x, given[:, :few].contiguous().cuda(), logp, "bf16", work, scale=0.7)       # (no entropy)
                assert torch.equal(logp.isnan(), kept[0][:, :few].isnan())
    finally:
        api.set_tuning(11, 0)


def head_of(api, W, dtype):
    """W [d, V], any V, as a head: columns of zeros up to the next multiple of 8, codes cut again."""
    V = W.shape[1]
    codes, scales = api.quantize_w8(torch.nn.functional.pad(W, (0, -V % 8)).to(TYPE[dtype]).cuda(), dtype)
    return codes[:V], scales


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,d,V", [(3, 136, 1001), (20, 264, 4099), (2, 128, 32001), (5, 64, 50257)])
def test_head_of_any_vocabulary(api, dtype, n, d, V):
    """A head that this library made, of a vocabulary that is no multiple of 8: the codes of the weight itself, and log probabilities over its tokens
    alone.  Sums of integers up to 2, so that logits are exact."""
    g = torch.Generator().manual_seed(V)
    x, W = torch.randint(-2, 3, (n, d), generator=g).float(), torch.randint(-2, 3, (d, V), generator=g).float()
    head = head_of(api, W, dtype)
    codes, scales = Q.quantize_weight(W.double().numpy())
    assert np.array_equal(head[0].view(torch.uint8).cpu().numpy(), codes) and np.array_equal(head[1].cpu().numpy(), scales)
    given = torch.randint(V, (n, 3), generator=g)
    given[0] = torch.tensor([V - 1, V, -1])
    logp, entropy = torch.empty(n, 3, device="cuda"), torch.empty(n, device="cuda")
    ids, tops = torch.empty(n, 9, dtype=torch.int32, device="cuda"), torch.empty(n, 9, device="cuda")
    api.score_w8(*head, x.to(TYPE[dtype]).cuda(), given.int().cuda(), logp, dtype, api.score_w8_workspace(n, d, V, 9), entropy=entropy, top_id=ids,
                 top_logp=tops, scale=0.125)
    want = Q.logprobs((x @ W).double().numpy(), given.numpy(), 9, 0.125)
    near(logp.double().cpu().numpy(), want[0])
    near(entropy.double().cpu().numpy(), want[1], rel=SUM)
    assert np.array_equal(ids.cpu().numpy(), want[2])
    near(tops.double().cpu().numpy(), want[3])


@pytest.mark.parametrize("tile", range(6))
@pytest.mark.parametrize("n,d,V", [(17, 128, 1), (33, 4104, 129), (40, 8200, 1003), (150, 136, 5003), (300, 520, 2011), (600, 2056, 777)])
def test_score_of_exact_logits(api, tile, n, d, V):
    """32-bit logits of every tile, with the sums in one piece and in parts, against the oracle: integers up to 2, differently scaled in each row and each
    block of the head, so that every logit is exact and only the softmax's own roundings are left."""
    print(f"exact score {tile} {n}x{d}x{V}", flush=True)
    g = torch.Generator().manual_seed(n + d + V)
    x = torch.randint(-2, 3, (n, d), generator=g).float() * 2.0 ** torch.randint(-2, 2, (n, 1), generator=g)
    W = torch.randint(-2, 3, (d, V), generator=g).float()
    for o in range(0, V, 128):
        W[:, o:o + 128] *= 2.0 ** ((o // 128) % 3 - 1)
    top, scale = min(V, 7), 2.0 ** -6
    given = torch.randint(V, (n, 2), generator=g)
    given[-1] = torch.tensor([V - 1, -1])
    logp, entropy = torch.full((n, 2), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    ids, tops = torch.empty(n, top, dtype=torch.int32, device="cuda"), torch.empty(n, top, device="cuda")
    head = head_of(api, W, "f16")
    try:
        api.set_tuning(11, tile)
        api.score_w8(*head, x.half().cuda(), given.int().cuda(), logp, "f16", api.score_w8_workspace(n, d, V, top), entropy=entropy, top_id=ids,
                     top_logp=tops, scale=scale)
    finally:
        api.set_tuning(11, 0)
    want = Q.logprobs(x.double().numpy() @ W.double().numpy(), given.numpy(), top, scale)
    near(logp.double().cpu().numpy(), want[0])
    near(entropy.double().cpu().numpy(), want[1], rel=SUM)
    assert np.array_equal(ids.cpu().numpy(), want[2])
    near(tops.double().cpu().numpy(), want[3])


def test_score_over_the_largest_vocabulary(api):
    """2^21 - 16 tokens: 16 rows at once, then the other four.  Small integers, so that logits are exact."""
    n, d, V, top = 20, 16, (1 << 21) - 16, 9
    g = torch.Generator("cuda").manual_seed(4)
    x = torch.randint(-2, 3, (n, d), generator=g, device="cuda").bfloat16()
    W = torch.randint(-2, 3, (d, V), generator=g, device="cuda").bfloat16()
    given = torch.randint(V, (n, 2), generator=g, device="cuda").int()
    logp, entropy = torch.empty(n, 2, device="cuda"), torch.empty(n, device="cuda")
    ids, tops = torch.empty(n, top, dtype=torch.int32, device="cuda"), torch.empty(n, top, device="cuda")
    ws = Guarded(api, api.lib().larosa_score_w8_workspace_bytes(n, d, V, top))
    api.score_w8(*api.quantize_w8(W, "bf16"), x, given, logp, "bf16", ws, entropy=entropy, top_id=ids, top_logp=tops, scale=0.5)
    assert ws.whole()
    z = x.float() @ W.float()
    p = (0.5 * z.double()).log_softmax(-1)
    best = z.sort(dim=-1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(ids.long(), best)
    for got, want in ((logp, p.gather(1, given.long())), (tops, p.gather(1, best))):
        assert bool(((got.double() - want).abs() <= SUM + REL * want.abs()).all())
    want = -(p.exp() * p).sum(-1)
    assert bool(((entropy.double() - want).abs() <= SUM + SUM * want).all())


@pytest.mark.parametrize("top", [0, 20])
@pytest.mark.parametrize("d,V,rows", [(128, 32000, (1041, 1024, 17, 1, 100)), (4104, 1003, (700, 40, 257, 3))])
def test_scores_stay_within_their_workspace(api, d, V, rows, top):
    """Parts of the rows, the last one divided by itself (1041 rows: 1024 and 17, which go in slices), and smaller batches in the workspace of
    the largest: nothing behind it is written, and every batch has the bits that it has in a workspace of its own."""
    g = torch.Generator().manual_seed(V)
    head = api.quantize_w8((torch.randn(d, V + (-V % 8), generator=g) * 0.2).half().cuda(), "f16")
    head = head[0][:V], head[1]
    x = torch.randn(rows[0], d, generator=g).half().cuda()
    given = torch.randint(V, (rows[0], 2), generator=g).int().cuda()
    ws = Guarded(api, api.lib().larosa_score_w8_workspace_bytes(rows[0], d, V, top))
    for n in rows:
        out = []
        for work in (ws, Guarded(api, api.lib().larosa_score_w8_workspace_bytes(n, d, V, top))):
            kw = dict(entropy=torch.full((n,), 7.0, device="cuda"))
            if top:
                kw.update(top_id=torch.empty(n, top, dtype=torch.int32, device="cuda"), top_logp=torch.empty(n, top, device="cuda"))
            logp = torch.full((n, 2), 7.0, device="cuda")
            api.score_w8(*head, x[:n], given[:n], logp, "f16", work, **kw)
            assert work.whole()
            out.append(dict(kw, logp=logp))
        assert all(torch.equal(out[0][k], out[1][k]) for k in out[0])


def test_score_is_its_parts_behind_a_norm(api):
    """The whole call against its parts as a program would run them one by one, up to the parts' rounding of logits to 16 bits."""
    n, d, V = 20, 512, 2048
    x, rms = torch.randn(n, d).bfloat16().cuda(), (1 + 0.2 * torch.randn(d)).bfloat16().cuda()
    head = api.quantize_w8((torch.randn(d, V) * 0.1).bfloat16().cuda(), "bf16")
    given = torch.randint(V, (n, 1)).int().cuda()
    logp, parts = torch.empty(n, 1, device="cuda"), torch.empty(n, 1, device="cuda")
    api.score_w8(*head, x, given, logp, "bf16", api.score_w8_workspace(n, d, V), rms=rms, rms_eps=1e-5)
    logits = torch.empty(n, V, dtype=torch.bfloat16, device="cuda")
    api.dense_w8(*head, x, logits, "bf16", api.dense_w8_workspace(n, d, V), rms=rms, rms_eps=1e-5)
    api.logprobs(logits, given, parts, api.logprobs_workspace(n, V))
    assert float((logp - parts).abs().max()) <= 2 * 2.0 ** -8 * float(logits.float().abs().max()) + SUM


def test_score_captured_and_replayed(api):
    n, d, V = 40, 256, 30011
    head = api.quantize_rows8((torch.randn(V, d) * 0.1).bfloat16().cuda(), "bf16")[0], torch.full((-(-V // 128), 4), 122, dtype=torch.uint8, device="cuda")
    x, given = torch.randn(n, d).bfloat16().cuda(), torch.randint(V, (n, 1)).int().cuda()
    out = [dict(logp=torch.empty(n, 1, device="cuda"), entropy=torch.empty(n, device="cuda"), top_id=torch.empty(n, 4, dtype=torch.int32, device="cuda"),
                ws=api.score_w8_workspace(n, d, V, 4)) for _ in range(2)]

    def score(o):
        api.score_w8(*head, x, given, o["logp"], "bf16", o["ws"], entropy=o["entropy"], top_id=o["top_id"], rms_eps=1e-5)

    score(out[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        score(out[0])
    for _ in range(4):
        x.copy_(torch.randn(n, d).bfloat16())
        graph.replay()
        score(out[1])
        torch.cuda.synchronize()
        for k in ("logp", "entropy", "top_id"):
            assert torch.equal(out[0][k], out[1][k])
