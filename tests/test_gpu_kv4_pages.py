"""Pages of the 4-bit cache on the GPU against the CPU bookkeeping (equal tables, references, lengths and bytes after every call), and the
operators together as a decoding program uses them: layers, branches, roll-backs, graph replays, two streams."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as K
from oracle import larosa_oracle as O
from tests import kv4_util as U
from tests.gpu_util import check_layer_trace, to_bits, to_dev

pytestmark = pytest.mark.gpu


def new_status():
    return torch.full((1,), 99, dtype=torch.int32, device="cuda:0")


class Twin:
    """A cache on the GPU and its CPU statement, driven by the same calls and compared after each."""

    def __init__(self, C):
        from paper_2507_01299_amd import api
        self.api, self.C, self.cache = api, C, U.device_cache(C)
        self.ws = api.kv4_pages_workspace(self.cache)

    def same(self, got=None, want=None):
        torch.cuda.synchronize()
        if want is not None:
            assert int(got) == want, (int(got), want)
        U.same_state(self.cache, self.C)

    def trim(self, slots, keep=None):
        K.trim(self.C, slots, keep)
        self.api.kv4_trim(self.cache, U.int32(slots), U.int32(keep))
        self.same()

    def fork(self, src, dst):
        want, status = K.fork(self.C, src, dst), new_status()
        self.api.kv4_fork(self.cache, U.int32(src), U.int32(dst), status)
        self.same(status, want)
        return want

    def grow(self, slots, counts=None):
        want, status = K.grow(self.C, slots, counts or [1] * len(slots)), new_status()
        self.api.kv4_grow(self.cache, U.int32(slots), status, self.ws, U.int32(counts))
        self.same(status, want)
        return want

    def compact(self):
        want, live = K.compact(self.C), new_status()
        self.api.kv4_compact(self.cache, live, self.ws)
        self.same(live, want)
        return want


@pytest.mark.parametrize("seed,pages,slots,max_pages,P", [(1, 20, 6, 5, 32), (2, 40, 12, 7, 64), (3, 13, 5, 9, 32)])
def test_random_walk(gpu_device, seed, pages, slots, max_pages, P):
    rng = np.random.default_rng(seed)
    C = K.Cache(2, pages, P, slots, max_pages, 2, 64, "f16")
    C.data[:] = rng.integers(0, 256, C.data.shape, dtype=np.uint8)
    t = Twin(C)
    seen = {"grown": 0, "missing": 0, "bad": 0, "forked": 0}
    for step in range(120):
        op = rng.integers(9)
        some = [int(s) for s in rng.permutation(slots)[:rng.integers(1, slots)]]
        if op < 2:
            t.trim(some, (rng.integers(-3, max_pages * P, len(some)) * rng.integers(0, 2, len(some))).tolist())
        elif op < 4:
            free = [s for s in range(slots) if C.length[s] == 0]
            used = [s for s in range(slots) if C.length[s] > 0]
            if free and used:
                dst = free[:rng.integers(1, len(free) + 1)]
                seen["forked"] += t.fork([int(s) for s in rng.choice(used, len(dst))], dst) == 0
        elif op < 8:
            rc = t.grow(some, rng.integers(0, P + 9, len(some)).tolist())
            seen["grown" if rc == 0 else "missing" if rc > 0 else "bad"] += 1
        else:
            t.compact()
    print(seen, flush=True)
    assert seen["grown"] and seen["forked"] and seen["missing"]


def test_lists_out_of_order(gpu_device):
    """The same slot twice, slots that do not exist, destinations in use, rows too short, negative numbers."""
    t = Twin(K.Cache(1, 8, 32, 5, 3, 1, 64, "f16"))
    assert t.grow([0, 1], [40, 33]) == 0
    for bad in ([0, 0], [1, 5], [-1], [0, 1, 0]):
        assert t.grow(bad) == -1
    assert t.grow([2, 3], [1, -1]) == t.grow([0], [57]) == t.grow([2], [2 ** 31 - 1]) == -1
    assert t.grow([2, 3, 4], [96, 1, 64]) == 2
    for src, dst in (([0], [1]), ([0, 0], [2, 2]), ([0, 2], [2, 3]), ([5], [2]), ([0], [-1]), ([3], [3])):
        assert t.fork(src, dst) == -1
    assert t.fork([0, 0, 4], [2, 3, 1]) == -1
    assert t.fork([0, 0], [2, 3]) == 0
    t.trim([0, 7, -2, 0, 1, 1], [5, 5, 5, 33, 0, 10])
    t.trim([2, 2, 3])
    assert t.grow([0], [0]) == 0 and t.grow([0, 1, 2], [27, 0, 1]) == 0
    t.compact()
    t.trim([0, 1, 2, 3, 4])
    assert t.compact() == 0
    assert t.fork([0], [1]) == 0                  # an empty sequence


def test_more_sharers_than_pages(gpu_device):
    """Forty slots share the one page: a grow of all would need 39 copies, which there is no room for; of one it fits."""
    t = Twin(K.Cache(1, 2, 32, 40, 2, 1, 64, "bf16"))
    assert t.grow([0], [7]) == 0
    assert t.fork([0] * 39, list(range(1, 40))) == 0
    assert t.grow(list(range(40))) == 38
    assert t.grow([17]) == 0 and t.grow([18]) == 1


def test_large_pool(gpu_device):
    """More pages than one step of the bookkeeping covers, and more listed slots than its lanes."""
    rng = np.random.default_rng(4)
    C = K.Cache(1, 20000, 32, 1500, 16, 1, 64, "f16")
    t = Twin(C)
    assert t.grow(list(range(1500)), rng.integers(0, 400, 1500).tolist()) == 0
    t.trim([int(s) for s in rng.permutation(1500)[:700]], None)
    free = [s for s in range(1500) if C.length[s] == 0]
    used = [s for s in range(1500) if C.length[s] > 0]
    assert t.fork([int(s) for s in rng.choice(used, 600)], free[:600]) == 0
    assert t.grow([int(s) for s in rng.permutation(1500)], None) == 0
    t.compact()


def test_copy_pages(gpu_device):
    from paper_2507_01299_amd import api
    rng = np.random.default_rng(5)
    for P, kv, D, layers in ((32, 1, 64, 3), (64, 3, 128, 2), (256, 2, 256, 1)):
        C = K.Cache(layers, 9, P, 1, 1, kv, D, "f16")
        C.data[:] = rng.integers(0, 256, C.data.shape, dtype=np.uint8)
        cache = U.device_cache(C)
        api.kv4_copy_pages(cache, U.int32([0, 5, 9, 3, 0]), U.int32([1, 8, 2, -1, 4]))
        torch.cuda.synchronize()
        C.data[:, [1, 8, 4]] = C.data[:, [0, 5, 0]]
        U.same_state(cache, C)


# ---- together ---------------------------------------------------------------------------------------------

def small_layer(dtype, seed, shortcut):
    from paper_2507_01299_amd import synth
    from tests import cases
    from tests.gpu_util import device_layer
    shape = synth.LayerShape("small", 256, 256, 128, 704, 64, dtype)
    if shortcut:
        layers, bits, _, _, src = cases.build_shortcut_stack(shape, 1, 0.4, seed=seed, n_cal=512)
        case = cases.LayerCase(shape, bits[0], layers[0], {}, src)
    else:
        case = cases.build_block_layer(shape, 0.4, seed=seed, n_cal=512)
    return case, device_layer(case)


@pytest.mark.parametrize("dtype,shortcut", [("f16", True), ("bf16", False)])
def test_layer_decodes_prompts_branches_and_roll_backs(gpu_device, dtype, shortcut):
    """A program's decoding: prompts in, a fork, steps of all sequences, a roll-back, packing, a further step, one layer after the other.
    Every step's layer output is checked stage by stage, its attention against fp64 over what the cache holds."""
    from paper_2507_01299_amd import api
    rng = np.random.default_rng(31)
    heads, kv, D = 4, 2, 64
    built = [small_layer(dtype, 61 + i, shortcut) for i in range(2)]
    C = K.Cache(2, 16, 32, 4, 6, kv, D, dtype)
    cache = U.device_cache(C)
    ws = api.kv4_pages_workspace(cache)
    table = torch.from_numpy(np.concatenate([np.cos(np.outer(np.arange(200), 0.5 ** np.arange(32))), np.sin(np.outer(np.arange(200), 0.5 ** np.arange(32)))], 1)
                             .astype(np.float32)).to("cuda:0")
    status = new_status()

    def step(slots, counts):
        api.kv4_grow(cache, U.int32(slots), status, ws, U.int32(counts))
        assert int(status) == 0
        starts = [0] + np.cumsum(counts).tolist()
        rows, max_new = starts[-1], max(counts)
        one = max_new == 1
        batch = api.KvBatch(U.int32(slots), rows, starts=None if one else U.int32(starts), max_new=max_new)
        x = to_dev(U.random_rows(rng, rows, 256, dtype), dtype)
        for i, (case, layer) in enumerate(built):
            # by hand
            lw = api.Workspace(layer.workspace_bytes(rows))
            tr = layer.trace_buffers(rows)
            qkv = torch.zeros(rows, (heads + 2 * kv) * D, dtype=x.dtype, device="cuda:0")
            s1 = torch.zeros_like(x) if shortcut else None
            attn, x_out, x_all = (torch.zeros(rows, n, dtype=x.dtype, device="cuda:0") for n in (heads * D, 256, 256))
            api.layer_qkv(layer, x, qkv, s1, lw, tr)
            turned = torch.zeros_like(qkv)
            before = cache.data.clone()
            api.kv4_append(cache, i, batch, qkv, heads, out=turned, rotary=api.Rotary(table))
            aw = api.kv4_attention_workspace(cache, batch, heads)
            api.kv4_attention(cache, i, batch, turned, heads, attn, aw)
            api.layer_after_attention(layer, s1 if shortcut else x, attn, x_out, lw, tr)
            after = cache.data.clone()
            # in one call, from the same start
            cache.data.copy_(before)
            api.layer_forward_kv4(layer, cache, i, batch, x, x_all, api.layer_kv4_workspace(layer, cache, batch), rotary=api.Rotary(table))
            torch.cuda.synchronize()
            assert torch.equal(x_all.view(torch.int16), x_out.view(torch.int16)) and torch.equal(cache.data, after)
            # against the statement
            tr["qkv"] = qkv
            if shortcut:
                tr["s1"] = s1
            check_layer_trace(case.layer, to_bits(x), tr, x_out, attn_bits=to_bits(attn))
            C.data = cache.data.cpu().numpy().reshape(C.data.shape)
            C.table, C.length, C.refs = (t.cpu().numpy() for t in (cache.table, cache.length, cache.refs))
            q = O.decode16(to_bits(turned[:, :heads * D].contiguous()), dtype).reshape(rows, heads, D)
            got = O.decode16(to_bits(attn), dtype).reshape(rows, heads, D)
            want = U.attention_want(C, i, slots, None if one else starts, q, heads, D ** -0.5, 0, max_new)
            for row, (o, tol) in want.items():
                assert (np.abs(got[row] - o) <= tol).all()
            x = x_out
        return x

    step([0, 3], [33, 5])
    api.kv4_fork(cache, U.int32([0, 3]), U.int32([1, 2]), status)
    step([0, 1, 2, 3], [1, 1, 1, 1])
    step([1, 2], [4, 3])
    api.kv4_trim(cache, U.int32([1]), U.int32([35]))          # two of slot 1's four drafted tokens fall
    api.kv4_trim(cache, U.int32([3]))
    api.kv4_compact(cache, None, ws)
    step([1, 0, 2], [1, 1, 1])
    assert cache.length.tolist() == [35, 36, 10, 0]


def test_graph_replays_of_a_decode_step(gpu_device):
    """grow, append and attention captured once and replayed, with eager work between: every replay equals the eager run."""
    from paper_2507_01299_amd import api
    rng = np.random.default_rng(41)
    heads, kv, D, dtype = 4, 2, 128, "bf16"
    C, slots = U.random_cache(rng, [63, 20, 600], 64, kv, D, dtype, headroom=20, spare_pages=8)
    eager, graphed = U.device_cache(C), U.device_cache(C)
    table = torch.randn(700, D, device="cuda:0")
    qkv = to_dev(U.random_rows(rng, 3, (heads + 2 * kv) * D, dtype), dtype)
    sl = U.int32(slots)
    runs = []
    for cache in (eager, graphed):
        batch = api.KvBatch(sl, 3)
        buf = dict(cache=cache, batch=batch, pw=api.kv4_pages_workspace(cache), aw=api.kv4_attention_workspace(cache, batch, heads),
                   status=new_status(), turned=torch.zeros_like(qkv), out=torch.zeros(3, heads * D, dtype=qkv.dtype, device="cuda:0"))

        def one(b=buf):
            api.kv4_grow(b["cache"], sl, b["status"], b["pw"])
            api.kv4_append(b["cache"], 0, b["batch"], qkv, heads, out=b["turned"], rotary=api.Rotary(table))
            api.kv4_attention(b["cache"], 0, b["batch"], b["turned"], heads, b["out"], b["aw"])
        runs.append((one, buf))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        runs[1][0]()
    for i in range(4):
        qkv.copy_(to_dev(U.random_rows(rng, 3, (heads + 2 * kv) * D, dtype), dtype))
        runs[0][0]()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        a, b = runs[0][1], runs[1][1]
        assert int(a["status"]) == int(b["status"]) == 0
        assert torch.equal(a["out"].view(torch.int16), b["out"].view(torch.int16))
        for name in ("table", "length", "refs", "data"):
            assert torch.equal(getattr(eager, name), getattr(graphed, name)), name


def test_two_streams_with_a_cache_and_workspace_each(gpu_device):
    from paper_2507_01299_amd import api
    rng = np.random.default_rng(42)
    heads, kv, D, dtype = 8, 2, 128, "f16"
    jobs = []
    for i in range(2):
        C, slots = U.random_cache(rng, [2000, 900, 5], 64, kv, D, dtype)
        cache = U.device_cache(C)
        batch = api.KvBatch(U.int32(slots), 3)
        q = to_dev(U.random_rows(rng, 3, heads * D, dtype), dtype)
        jobs.append(dict(cache=cache, batch=batch, q=q, out=torch.zeros_like(q), alone=torch.zeros_like(q),
                         ws=api.kv4_attention_workspace(cache, batch, heads), stream=torch.cuda.Stream()))
    for j in jobs:
        api.kv4_attention(j["cache"], 0, j["batch"], j["q"], heads, j["alone"], j["ws"])
    torch.cuda.synchronize()
    for _ in range(20):
        for j in jobs:
            with torch.cuda.stream(j["stream"]):
                api.kv4_attention(j["cache"], 0, j["batch"], j["q"], heads, j["out"], j["ws"])
    torch.cuda.synchronize()
    for j in jobs:
        assert torch.equal(j["out"].view(torch.int16), j["alone"].view(torch.int16))


def test_trim_that_keeps_more_than_there_is(gpu_device):
    """keep up to the largest int32, for used and free slots, beside a smaller keep of the same slot: nothing else may change."""
    t = Twin(K.Cache(1, 12, 32, 6, 4, 1, 64, "f16"))
    assert t.grow([0, 1, 2], [70, 128, 32]) == 0
    for keep in (71, 129, 2 ** 31 - 33, 2 ** 31 - 32, 2 ** 31 - 31, 2 ** 31 - 1):
        t.trim([0, 1, 2, 3, 5], [keep] * 5)
    t.trim([1, 1, 4, 2], [2 ** 31 - 1, 40, 2 ** 31 - 1, 2 ** 31 - 2])
    t.trim([0, 3], [2 ** 31 - 32, -2 ** 31])
    assert t.cache.length.tolist() == [70, 40, 32, 0, 0, 0]


def test_binding_refuses_lists_on_another_device(gpu_device):
    from paper_2507_01299_amd import api
    c = api.KvCache(1, 4, 32, 4, 1, 1, 64, "f16")
    here, status = torch.tensor([0], dtype=torch.int32), torch.zeros(1, dtype=torch.int32, device="cuda:0")
    ws = api.kv4_pages_workspace(c)
    for call in (lambda: api.kv4_trim(c, here), lambda: api.kv4_trim(c, here.cuda(), here), lambda: api.kv4_grow(c, here, status, ws),
                 lambda: api.kv4_grow(c, here.cuda(), status.cpu(), ws), lambda: api.kv4_fork(c, here, here.cuda() + 1, status),
                 lambda: api.kv4_copy_pages(c, here.cuda(), here), lambda: api.kv4_compact(c, status.cpu(), ws),
                 lambda: api.KvBatch(here.cuda(), 2, starts=here.new_zeros(2))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        api.KvCache(1, 4, 32, 4, 1, 1, 64, "f16", data=c.data, refs=c.refs, table=c.table.cpu(), length=c.length)


def test_binding_refuses_rows_on_another_device(gpu_device):
    from paper_2507_01299_amd import api
    c = api.KvCache(1, 4, 32, 4, 1, 1, 64, "f16")
    slots = torch.tensor([0], dtype=torch.int32)
    batch, away = api.KvBatch(slots.cuda(), 1), api.KvBatch(slots, 1)
    rows, table = torch.zeros(1, 192, dtype=torch.float16), torch.zeros(8, 64)
    ws = api.kv4_attention_workspace(c, batch, 1)
    for call in (lambda: api.kv4_append(c, 0, batch, rows, 1), lambda: api.kv4_append(c, 0, batch, rows.cuda(), 1, out=rows),
                 lambda: api.kv4_append(c, 0, away, rows.cuda(), 1),
                 lambda: api.kv4_append(c, 0, batch, rows.cuda(), 1, out=rows.cuda(), rotary=api.Rotary(table)),
                 lambda: api.Rotary(table.cuda(), positions=slots[None]),
                 lambda: api.kv4_attention(c, 0, batch, rows, 1, rows.cuda(), ws), lambda: api.kv4_attention(c, 0, batch, rows.cuda(), 1, rows, ws),
                 lambda: api.kv4_attention(c, 0, away, rows.cuda(), 1, rows.cuda(), ws)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("dtype,shortcut,n", [("f16", True, 2900), ("bf16", False, 2900), ("f16", False, 70)])
def test_layer_with_one_row(gpu_device, dtype, shortcut, n):
    """One token at a time, the kernels of a single row: their key histograms and the attention's partial sums lie in one workspace, one
    after the other.  Three steps through two layers and that workspace, against the split calls with workspaces of their own."""
    from paper_2507_01299_amd import api
    rng = np.random.default_rng(51)
    heads, kv, D = 4, 2, 64
    built = [small_layer(dtype, 81 + i, shortcut) for i in range(2)]
    C, slots = U.random_cache(rng, [n], 64, kv, D, dtype, n_layers=2, headroom=8, spare_pages=4)
    cache = U.device_cache(C)
    ws, status = api.kv4_pages_workspace(cache), new_status()
    sl = U.int32(slots)
    batch = api.KvBatch(sl, 1)
    angles = np.outer(np.arange(n + 8), 0.9 ** np.arange(32))
    rotary = api.Rotary(torch.from_numpy(np.concatenate([np.cos(angles), np.sin(angles)], 1).astype(np.float32)).to("cuda:0"))
    assert (api.kv4_attention_plan(cache, batch, heads)["splits"] > 1) == (n > 1000)
    whole = api.layer_kv4_workspace(built[0][1], cache, batch)
    for _ in range(3):
        api.kv4_grow(cache, sl, status, ws)
        assert int(status) == 0
        x = to_dev(U.random_rows(rng, 1, 256, dtype), dtype)
        for i, (case, layer) in enumerate(built):
            before = cache.data.clone()
            x_all = torch.zeros_like(x)
            api.layer_forward_kv4(layer, cache, i, batch, x, x_all, whole, rotary=rotary)
            after = cache.data.clone()
            cache.data.copy_(before)
            lw, tr = api.Workspace(layer.workspace_bytes(1)), layer.trace_buffers(1)
            qkv = torch.zeros(1, (heads + 2 * kv) * D, dtype=x.dtype, device="cuda:0")
            s1 = torch.zeros_like(x) if shortcut else None
            attn, x_out = torch.zeros(1, heads * D, dtype=x.dtype, device="cuda:0"), torch.zeros_like(x)
            api.layer_qkv(layer, x, qkv, s1, lw, tr)
            turned = torch.zeros_like(qkv)
            api.kv4_append(cache, i, batch, qkv, heads, out=turned, rotary=rotary)
            api.kv4_attention(cache, i, batch, turned, heads, attn, api.kv4_attention_workspace(cache, batch, heads))
            api.layer_after_attention(layer, s1 if shortcut else x, attn, x_out, lw, tr)
            torch.cuda.synchronize()
            assert torch.equal(x_all.view(torch.int16), x_out.view(torch.int16)) and torch.equal(cache.data, after)
            tr["qkv"] = qkv
            if shortcut:
                tr["s1"] = s1
            check_layer_trace(case.layer, to_bits(x), tr, x_out, attn_bits=to_bits(attn))
            C.data = cache.data.cpu().numpy().reshape(C.data.shape)
            C.table, C.length, C.refs = (t.cpu().numpy() for t in (cache.table, cache.length, cache.refs))
            q = O.decode16(to_bits(turned[:, :heads * D].contiguous()), dtype).reshape(1, heads, D)
            o, tol = U.attention_want(C, i, slots, None, q, heads, D ** -0.5, 0, 1)[0]
            assert (np.abs(O.decode16(to_bits(attn), dtype).reshape(heads, D) - o) <= tol).all()
            x = x_out
