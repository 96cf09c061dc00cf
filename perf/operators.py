"""The operators around a key/value cache held in 4 bits: attention over it, the new tokens' rotary positions and
quantised append, and the handling of its pages (fork, grow with copy on write, trim, compaction).

`listed()` names twelve cases, `draw(rng)` gives another one of the same ranges.  `run` computes the operators in
plain torch where `own` is false and calls `paper_2507_01299_amd.api` where it is true; `exact` states attention and
append in 64 bits; `work` gives the bytes and operations of one pass.

The cache.  A page holds `page` tokens of one layer, per key/value head one block of 34 D bytes for every 32 tokens:
the codes of K (16 D bytes) and of V (16 D), then the scales of K (D) and of V (D).  32 neighbouring values of a head share a scale
2^(byte - 127); byte 255 stands for NaN.  A code is a sign and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
TYPE = {"f16": torch.float16, "bf16": torch.bfloat16}
EXPONENTS = {"f16": (-23, 13), "bf16": (-100, 125)}      # of the scales: the values stay inside the 16-bit type
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---- the cases ------------------------------------------------------------------------------------------

HEADS_7B = dict(heads=32, kv_heads=32, dim=128)
HEADS_8B = dict(heads=32, kv_heads=8, dim=128)
HEADS_70B = dict(heads=64, kv_heads=8, dim=128)


def listed():
    return [
        # one chat turn of an 8B model, a few hundred tokens in: all latency
        dict(name="attention_8b_b1_short", op="attention", n_seq=1, longest=333, new=1, window=0, page=64, dtype="f16", **HEADS_8B),
        # one long document in front of a 70B model
        dict(name="attention_70b_b1_long", op="attention", n_seq=1, longest=100003, new=1, window=0, page=64, dtype="bf16", **HEADS_70B),
        # a ragged decode batch of a 7B model, a head of keys for every head of queries
        dict(name="attention_7b_b32", op="attention", n_seq=32, longest=4096, new=1, window=0, page=32, dtype="f16", **HEADS_7B),
        # a server's large ragged batch
        dict(name="attention_8b_b64", op="attention", n_seq=64, longest=16384, new=1, window=0, page=128, dtype="bf16", **HEADS_8B),
        # checking up to seven drafted tokens of every sequence at once
        dict(name="attention_8b_b9_draft", op="attention", n_seq=9, longest=8191, new=7, window=0, page=64, dtype="bf16", **HEADS_8B),
        # a small model with a sliding window
        dict(name="attention_d64_window", op="attention", n_seq=16, longest=6000, new=1, window=2048, page=64, dtype="f16", heads=16, kv_heads=4, dim=64),
        # the append of a decode step: one token for each of 13 sequences
        dict(name="append_8b_b13", op="append", n_seq=13, longest=5000, new=1, axes=1, page=64, dtype="bf16", **HEADS_8B),
        # the append of a prompt with pictures: three axes of positions, three ragged prompts
        dict(name="append_70b_prompt", op="append", n_seq=3, longest=2500, new=2500, axes=3, page=64, dtype="f16", **HEADS_70B),
        # one step of a search with four branches on an 8B model: losers freed, winners forked, all grown by a token
        dict(name="branch_8b_4", op="branch", n_seq=4, longest=700, layers=32, page=64, dtype="bf16", **HEADS_8B),
        # the same for 48 branches of long sequences
        dict(name="branch_8b_48", op="branch", n_seq=48, longest=4096, layers=8, page=64, dtype="bf16", **HEADS_8B),
        # a few short requests end: the pool is packed again
        dict(name="compact_8b_small", op="compact", n_seq=8, longest=500, layers=32, page=64, dtype="bf16", **HEADS_8B),
        # long requests of a 7B model end
        dict(name="compact_7b_large", op="compact", n_seq=12, longest=3000, layers=16, page=32, dtype="f16", **HEADS_7B),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    heads = dict(rng.choice([HEADS_7B, HEADS_8B, HEADS_70B, dict(heads=16, kv_heads=4, dim=64), dict(heads=8, kv_heads=1, dim=256),
                             dict(heads=28, kv_heads=4, dim=128), dict(heads=12, kv_heads=12, dim=64)]))
    case = dict(heads, page=rng.choice([32, 64, 128, 256]), dtype=rng.choice(["f16", "bf16"]))
    op = case["op"] = rng.choice(["attention", "attention", "attention", "append", "branch", "compact"])
    width = heads["kv_heads"] * heads["dim"]
    if op == "attention":
        n = case["n_seq"] = _log_int(rng, 1, 64)
        case["longest"] = _log_int(rng, 1, min(100000, int(64 * 16384 * 1024 / (n * width))))
        case["new"] = rng.choice([1, 1, 1, rng.randint(2, 9)])
        case["window"] = rng.choice([0, 0, 0, _log_int(rng, 16, 8192)])
    elif op == "append":
        n = case["n_seq"] = _log_int(rng, 1, 64)
        case["new"] = rng.choice([1, _log_int(rng, 2, 2048)]) if n < 4 else rng.choice([1, rng.randint(2, 9)])
        case["longest"] = max(case["new"], _log_int(rng, 1, 6000))
        case["axes"] = rng.choice([1, 1, 3])
    else:
        n = case["n_seq"] = _log_int(rng, 4, 32)
        case["layers"] = rng.choice([4, 8, 16])
        tokens = 1.0e9 / (case["layers"] * width * 34 / 32)
        case["longest"] = _log_int(rng, 40, max(64, min(4096, int(tokens / n))))
    return case


def _lengths(case):
    """Tokens of each sequence: the longest, and others down to a sixteenth of it.  Given by the case alone."""
    r = random.Random(case["n_seq"] * 7919 + case["longest"])
    return [case["longest"]] + [_log_int(r, max(1, case["longest"] // 16), case["longest"]) for _ in range(case["n_seq"] - 1)]


def _news(case):
    """New tokens of each sequence (among its tokens)."""
    r = random.Random(case["longest"] * 31 + case["n_seq"])
    return [min(n, case["new"] if i == 0 else r.randint(1, case["new"])) for i, n in enumerate(_lengths(case))]


def _pages(n, page):
    return -(-n // page)


# ---- the format ----------------------------------------------------------------------------------------

def _quantise(x, dtype):
    """x [..., D] in 32 bits -> codes and scale bytes, nearest code, ties to the even one."""
    lowest, highest = EXPONENTS[dtype]
    a = x.abs().unflatten(-1, (-1, 32))
    top = a.amax(-1, keepdim=True)
    part, power = torch.frexp(top)
    e = torch.where(top == 0, lowest, power - 3 + (part > 0.875).to(power.dtype)).clamp(lowest, highest)
    whole = torch.isfinite(top)
    unit = torch.where(whole, torch.exp2(e.to(x.dtype)), float("nan"))
    code = ((a > 0.25 * unit).to(torch.uint8) + (a >= 0.75 * unit) + (a > 1.25 * unit) + (a >= 1.75 * unit)
            + (a > 2.5 * unit) + (a >= 3.5 * unit) + (a > 5.0 * unit))
    code = code.flatten(-2) + 8 * torch.signbit(x).to(torch.uint8)
    return code.to(torch.uint8), torch.where(whole, e + 127, 255).squeeze(-1).to(torch.uint8)


def _values(code, scale):
    """Codes and scale bytes -> what they stand for, in 32 bits."""
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=code.device)
    unit = torch.where(scale == 255, float("nan"), torch.exp2(scale.to(torch.float32) - 127))
    return (level[code.int()].unflatten(-1, (-1, 32)) * unit[..., None]).flatten(-2)


def _pack(kc, vc, ks, vs):
    """Codes [..., 32, D] and scale bytes [..., 32, D/32] of whole blocks -> bytes [..., 34 D]."""
    D = kc.shape[-1]
    W = min(16, D // 8)
    parts = D // 8 // W
    lead = kc.shape[:-2]
    n = len(lead)
    two = lambda c: c[..., 0::2] | (c[..., 1::2] << 4)                                  # noqa: E731
    order = lambda t, o: t.permute(*range(n), *(n + i for i in o)).reshape(*lead, -1)   # noqa: E731
    k = order(two(kc).reshape(*lead, 2, 16, 4, parts, W), (0, 3, 2, 1, 4))
    v = order(two(vc).reshape(*lead, 2, 4, parts, 4 // parts, 16, D // 32), (0, 2, 1, 4, 3, 5))
    a = order(ks.reshape(*lead, 2, 16, D // 32), (0, 2, 1))
    b = order(vs.reshape(*lead, 2, 4, 4, D // 32), (0, 1, 3, 2))
    return torch.cat([k, v, a, b], -1)


def _unpack(block, D):
    """Bytes [..., 34 D] -> K and V [..., 32, D] in 32 bits."""
    W = min(16, D // 8)
    parts = D // 8 // W
    lead = block.shape[:-1]
    n = len(lead)
    order = lambda t, o: t.permute(*range(n), *(n + i for i in o))                      # noqa: E731
    two = lambda t: torch.stack([t & 15, t >> 4], -1).flatten(-2)                       # noqa: E731
    k = order(block[..., :16 * D].reshape(*lead, 2, parts, 4, 16, W), (0, 3, 2, 1, 4)).reshape(*lead, 32, D // 2)
    v = order(block[..., 16 * D:32 * D].reshape(*lead, 2, parts, 4, 16, 4 // parts, D // 32), (0, 2, 1, 4, 3, 5)).reshape(*lead, 32, D // 2)
    a = order(block[..., 32 * D:33 * D].reshape(*lead, 2, D // 32, 16), (0, 2, 1)).reshape(*lead, 32, D // 32)
    b = order(block[..., 33 * D:].reshape(*lead, 2, 4, D // 32, 4), (0, 1, 3, 2)).reshape(*lead, 32, D // 32)
    return _values(two(k), a), _values(two(v), b)


# ---- what a program has in hand ------------------------------------------------------------------------

def _pool(case, g, n_layers, n_pages):
    """A pool of pages whose tokens hold keys with a few strong channels, and values."""
    H, D, P = case["kv_heads"], case["dim"], case["page"]
    data = torch.empty(n_layers, n_pages, H, P // 32, 34 * D, dtype=torch.uint8, device=DEV)
    strong = torch.where(torch.rand(H, 1, 1, D, generator=g, device=DEV) < 0.04, 5.0, 1.0)
    step = max(1, (1 << 26) // (H * P * D))
    for layer in range(n_layers):
        if layer >= 2:                 # deep pools repeat two layers' pages, which nothing but copies reads
            data[layer] = data[layer % 2]
            continue
        for at in range(0, n_pages, step):
            shape = (min(step, n_pages - at), H, P // 32, 32, D)
            k, ks = _quantise(torch.randn(shape, generator=g, device=DEV) * strong, case["dtype"])
            v, vs = _quantise(torch.randn(shape, generator=g, device=DEV), case["dtype"])
            data[layer, at:at + step] = _pack(k, v, ks, vs)
    return data


def _place(case, g, lengths, n_slots, n_pages, slots):
    """Pages in a random order for the sequences in `slots`."""
    need = [_pages(n, case["page"]) for n in lengths]
    max_pages = max(need) + 2
    table = torch.full((n_slots, max_pages), -1, dtype=torch.int32)
    length = torch.zeros(n_slots, dtype=torch.int32)
    refs = torch.zeros(n_pages, dtype=torch.int32)
    ids = torch.randperm(n_pages, generator=g).int()
    at = 0
    for s, n, p in zip(slots, lengths, need):
        table[s, :p] = ids[at:at + p]
        refs[ids[at:at + p].long()] = 1
        length[s] = n
        at += p
    return table.to(DEV), length.to(DEV), refs.to(DEV)


def _rotary_table(n_pos, D):
    angle = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device=DEV) / D)
    return torch.cat([angle.cos(), angle.sin()], -1).float()


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    c = torch.Generator().manual_seed(seed)
    H, D, P, N = case["kv_heads"], case["dim"], case["page"], case["n_seq"]
    T = TYPE[case["dtype"]]
    lengths = _lengths(case)
    s = dict(case=case)
    if case["op"] in ("attention", "append"):
        n_slots, n_layers, layer = N + 3, 1, 0
        slots = torch.randperm(n_slots, generator=c)[:N].tolist()
        n_pages = sum(_pages(n, P) for n in lengths) + 3
        table, length, refs = _place(case, c, lengths, n_slots, n_pages, slots)
        news = _news(case)
        rows = sum(news)
        s.update(layer=layer, rows=rows, max_new=max(news), max_len=max(lengths), slots=torch.tensor(slots, dtype=torch.int32, device=DEV),
                 starts=None if case["new"] == 1 else torch.tensor([0] + news, device=DEV).cumsum(0).int(),
                 qkv=(torch.randn(rows, (case["heads"] + 2 * H) * D, generator=g, device=DEV) * 1.2).to(T))
        if case["op"] == "append":
            s["out"] = torch.empty_like(s["qkv"])
            s["rotary"] = _rotary_table(max(lengths), D)
            s["axis_pairs"], s["positions"] = None, None
            if case["axes"] == 3:      # a picture's tokens in rows of 40 between text
                first = torch.tensor([n - k for n, k in zip(lengths, news)], device=DEV).repeat_interleave(torch.tensor(news, device=DEV))
                i = torch.cat([torch.arange(k, device=DEV) for k in news])
                s["axis_pairs"] = (D // 8, D * 3 // 16, D // 2 - D // 8 - D * 3 // 16)
                s["positions"] = torch.stack([first, first + i // 40, first + i % 40]).clamp(max=max(lengths) - 1).int().contiguous()
        else:
            s["out"] = torch.empty(rows, case["heads"] * D, dtype=T, device=DEV)
    elif case["op"] == "branch":
        # the first half of the slots live on, each forked into one of the second half
        n_layers, half = case["layers"], N // 2
        n_slots = N
        n_pages = sum(_pages(n + 1, P) for n in lengths[:half]) + 2 * N + 8
        table, length, refs = _place(case, c, lengths[:half], n_slots, n_pages, range(half))
        s.update(winners=torch.arange(half, dtype=torch.int32, device=DEV), losers=torch.arange(half, 2 * half, dtype=torch.int32, device=DEV),
                 everyone=torch.arange(2 * half, dtype=torch.int32, device=DEV), back=torch.tensor(lengths[:half], dtype=torch.int32, device=DEV),
                 status=torch.zeros(2, dtype=torch.int32, device=DEV))
    else:
        # every other request ends, and as many tokens come anew; the next pass ends the others
        n_layers, half = case["layers"], N // 2
        n_slots = N
        both = [n for n in lengths[:half] for _ in range(2)]
        n_pages = sum(_pages(n, P) for n in both) * 5 // 4
        table, length, refs = _place(case, c, both, n_slots, n_pages, range(2 * half))
        s.update(turns=[torch.arange(i, 2 * half, 2, dtype=torch.int32, device=DEV) for i in (0, 1)], turn=0,
                 tokens=torch.tensor(lengths[:half], dtype=torch.int32, device=DEV), status=torch.zeros(1, dtype=torch.int32, device=DEV),
                 live=torch.zeros(1, dtype=torch.int32, device=DEV))
    s.update(data=_pool(case, g, n_layers, n_pages), table=table, length=length, refs=refs)
    if own:
        from paper_2507_01299_amd import api
        s["cache"] = api.KvCache(n_layers, n_pages, P, n_slots, table.shape[1], H, D, case["dtype"], data=s["data"], refs=refs, table=table, length=length)
        if "slots" in s:
            s["batch"] = api.KvBatch(s["slots"], s["rows"], starts=s["starts"], max_new=s["max_new"])
        if case["op"] == "attention":
            s["ws"] = api.kv4_attention_workspace(s["cache"], s["batch"], case["heads"], max_len=s["max_len"])
        if case["op"] == "append":
            s["angles"] = api.Rotary(s["rotary"], positions=s["positions"], axis_pairs=s["axis_pairs"])
        if "status" in s:
            s["ws"] = api.kv4_pages_workspace(s["cache"])
    return s


# ---- the plain forms -----------------------------------------------------------------------------------

def _rows(s):
    """Sequence number and place in its sequence of every row of the batch."""
    N, rows = s["case"]["n_seq"], s["rows"]
    r = torch.arange(rows, device=DEV)
    starts = s["starts"] if s["starts"] is not None else torch.arange(N + 1, device=DEV)
    seq = torch.searchsorted(starts[1:].contiguous(), r, right=True)
    ends = starts[1:][seq]
    return seq, s["length"][s["slots"].long()][seq] - ends + r


def _plain_attention(s):
    case = s["case"]
    D, P, Hq, H = case["dim"], case["page"], case["heads"], case["kv_heads"]
    n = _pages(s["max_len"], P)
    pages = s["table"][s["slots"].long(), :n].clamp(min=0).long()
    seq, at = _rows(s)
    k, v = _unpack(s["data"][s["layer"]][pages], D)                                        # [N, n, H, P/32, 32, D]
    k, v = (t.permute(0, 2, 1, 3, 4, 5).reshape(case["n_seq"], H, n * P, D) for t in (k, v))
    # the rows of each sequence side by side: [N, H, max_new * group, D]
    first = s["starts"][:-1].long() if s["starts"] is not None else torch.arange(case["n_seq"], device=DEV)
    j = torch.arange(s["rows"], device=DEV) - first[seq]
    q = torch.zeros(case["n_seq"], s["max_new"], H, Hq // H, D, device=DEV)
    q[seq, j] = s["qkv"][:, :Hq * D].float().reshape(-1, H, Hq // H, D)
    place = torch.full((case["n_seq"], s["max_new"]), -1, dtype=torch.int64, device=DEV)
    place[seq, j] = at.long()
    t = torch.arange(n * P, device=DEV)
    seen = t <= place[..., None]
    if case["window"]:
        seen = seen & (t > place[..., None] - case["window"])
    seen = seen[:, None, :, None, :].expand(-1, H, -1, Hq // H, -1).flatten(2, 3)
    score = torch.matmul(q.permute(0, 2, 1, 3, 4).flatten(2, 3), k.transpose(-1, -2)) * D ** -0.5
    score = torch.where(seen, score, float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = torch.where(seen, torch.exp(score - torch.where(torch.isfinite(top), top, 0.0)), 0.0)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    o = o.unflatten(2, (s["max_new"], Hq // H)).permute(0, 2, 1, 3, 4)[seq, j]
    return o.reshape(s["rows"], Hq * D).to(s["qkv"].dtype)


def _plain_append(s):
    case = s["case"]
    D, P, Hq, H = case["dim"], case["page"], case["heads"], case["kv_heads"]
    seq, at = _rows(s)
    x = s["qkv"].float().reshape(s["rows"], Hq + 2 * H, D)
    if s["positions"] is None:
        turn = s["rotary"][at.long()]
    else:
        axis = torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor(s["axis_pairs"], device=DEV)).repeat(2)
        turn = s["rotary"][s["positions"].long()[axis].T, torch.arange(D, device=DEV)]
    cos, sin = turn[:, None, :D // 2], turn[:, None, D // 2:]
    a, b = x[:, :Hq + H, :D // 2], x[:, :Hq + H, D // 2:]
    qk = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    kc, ks = _quantise(qk[:, Hq:], case["dtype"])
    vc, vs = _quantise(x[:, Hq + H:], case["dtype"])
    out = torch.cat([qk[:, :Hq], _values(kc, ks), _values(vc, vs)], 1).to(s["qkv"].dtype).flatten(1)
    page = s["table"][s["slots"].long()[seq], at // P].long()
    block, t = at % P // 32, (at % 32).long()
    # each token's bytes in its block
    D2, W, n = D // 2, min(16, D // 8), s["rows"]
    byte = torch.arange(D2, device=DEV)
    lane = byte // (D // 8) * 16 + (t % 16)[:, None]
    within = byte % (D // 8)
    k_at = (t // 16)[:, None] * 8 * D + within // W * (64 * W) + lane * W + within % W
    lane = (t % 16 // 4)[:, None] * 16 + byte // (D // 32)
    within = (t % 4)[:, None] * (D // 32) + byte % (D // 32)
    v_at = 16 * D + (t // 16)[:, None] * 8 * D + within // W * (64 * W) + lane * W + within % W
    group = torch.arange(D // 32, device=DEV)
    ks_at = 32 * D + (t // 16)[:, None] * (D // 2) + group * 16 + (t % 16)[:, None]
    vs_at = 33 * D + (t // 16)[:, None] * (D // 2) + ((t % 16 // 4)[:, None] * (D // 32) + group) * 4 + (t % 4)[:, None]
    where = torch.cat([k_at, v_at, ks_at, vs_at], -1)[:, None, :]
    what = torch.cat([kc[..., 0::2] | (kc[..., 1::2] << 4), vc[..., 0::2] | (vc[..., 1::2] << 4), ks, vs], -1)
    heads = torch.arange(H, device=DEV)[None, :, None]
    s["data"][s["layer"]][page[:, None, None].expand(n, H, 1), heads, block[:, None, None].long(), where] = what
    return out


def _plain_trim(s, slots, keep):
    P, table, length, refs = s["case"]["page"], s["table"], s["length"], s["refs"]
    slots = slots.long()
    had = length[slots]
    kept = torch.minimum(had, keep) if keep is not None else torch.zeros_like(had)
    col = torch.arange(table.shape[1], device=DEV)
    mine = table[slots]
    gone = (col >= ((kept + P - 1) // P)[:, None]) & (col < ((had + P - 1) // P)[:, None])
    refs.index_add_(0, torch.where(gone, mine, 0).flatten().long(), -gone.flatten().int())
    table[slots] = torch.where(gone, -1, mine)
    length[slots] = kept


def _plain_fork(s, src, dst):
    table, length, refs = s["table"], s["length"], s["refs"]
    mine = table[src.long()]
    refs.index_add_(0, mine.clamp(min=0).flatten().long(), (mine >= 0).flatten().int())
    table[dst.long()] = mine
    length[dst.long()] = length[src.long()]


def _plain_grow(s, slots, count):
    """Pages for `count` more tokens of every slot: the lowest free ones in the order of the list.  A shared last page that is
    not full is copied first, except by the last slot of the list where all that share it grow."""
    P, table, length, refs, data = s["case"]["page"], s["table"], s["length"], s["refs"], s["data"]
    n_pages, slots = refs.shape[0], slots.long()
    had = length[slots]
    old, new = (had + P - 1) // P, (had + count + P - 1) // P
    mine = table[slots]
    last = mine.gather(1, (old - 1).clamp(min=0)[:, None].long())[:, 0].clamp(min=0).long()
    i = torch.arange(slots.shape[0], device=DEV)
    shared = (count > 0) & (had % P != 0) & (refs[last] > 1)
    at = torch.where(shared, last, n_pages)
    growing = torch.zeros(n_pages + 1, dtype=torch.int32, device=DEV).index_add_(0, at, torch.ones_like(at, dtype=torch.int32))
    final = torch.full((n_pages + 1,), -1, device=DEV).scatter_reduce_(0, at, i, "amax")
    copy = shared & ~((growing[last] == refs[last]) & (final[last] == i))
    need = new - old + copy
    at = torch.cumsum(need, 0) - need
    free = refs == 0
    rank = torch.where(free, torch.cumsum(free, 0) - 1, n_pages)
    ids = torch.zeros(n_pages + 1, dtype=torch.int32, device=DEV).scatter_(0, rank, torch.arange(n_pages, dtype=torch.int32, device=DEV))
    fits = (need.sum() <= free.sum()) & (new <= table.shape[1]).all()
    col = torch.arange(table.shape[1], device=DEV)
    fresh = (col >= old[:, None]) & (col < new[:, None]) | (copy[:, None] & (col == (old - 1)[:, None]))
    fresh = fresh & fits
    given = ids[torch.where(fresh, at[:, None] + col - old[:, None] + copy[:, None], n_pages).long()]
    to = given.gather(1, (old - 1).clamp(min=0)[:, None].long())[:, 0].long()
    moved = copy & fits
    data[:, to[moved]] = data[:, last[moved]]
    refs.index_add_(0, last, -moved.int())
    refs.index_add_(0, torch.where(fresh, given, 0).flatten().long(), fresh.flatten().int())
    table[slots] = torch.where(fresh, given, mine)
    length[slots] = torch.where(fits, had + count, had).int()
    return torch.where(fits, 0, need.sum() - free.sum()).int()


def _plain_compact(s):
    table, refs, data = s["table"], s["refs"], s["data"]
    n_pages = refs.shape[0]
    ids = torch.arange(n_pages, device=DEV)
    live = refs > 0
    n = live.sum()
    holes = (~live & (ids < n)).nonzero()[:, 0]
    movers = (live & (ids >= n)).nonzero()[:, 0]
    data[:, holes] = data[:, movers]
    to = ids.scatter(0, movers, holes)
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].int(), table))
    refs.copy_(torch.zeros_like(refs).index_add_(0, to, refs))
    return n.int().reshape(1)


def run(s):
    op = s["case"]["op"]
    if own:
        return _run_own(s, op)
    if op == "attention":
        return _plain_attention(s)
    if op == "append":
        return dict(out=_plain_append(s), data=s["data"].view(torch.int32))
    if op == "branch":
        _plain_trim(s, s["losers"], None)
        _plain_trim(s, s["winners"], s["back"])
        _plain_fork(s, s["winners"], s["losers"])
        return _state(s, status=_plain_grow(s, s["everyone"], torch.ones_like(s["everyone"])))
    ended = s["turns"][s["turn"]]
    s["turn"] ^= 1
    _plain_trim(s, ended, None)
    live = _plain_compact(s)
    return _state(s, status=_plain_grow(s, ended, s["tokens"]), live=live)


def _state(s, **more):
    return dict(more, table=s["table"], length=s["length"], refs=s["refs"], data=s["data"].view(torch.int32))


def _run_own(s, op):
    from paper_2507_01299_amd import api
    cache, case = s["cache"], s["case"]
    if op == "attention":
        return api.kv4_attention(cache, s["layer"], s["batch"], s["qkv"], case["heads"], s["out"], s["ws"], window=case["window"], max_len=s["max_len"])
    if op == "append":
        api.kv4_append(cache, s["layer"], s["batch"], s["qkv"], case["heads"], out=s["out"], rotary=s["angles"])
        return dict(out=s["out"], data=s["data"].view(torch.int32))
    if op == "branch":
        api.kv4_trim(cache, s["losers"])
        api.kv4_trim(cache, s["winners"], s["back"])
        api.kv4_fork(cache, s["winners"], s["losers"], s["status"][1:])
        api.kv4_grow(cache, s["everyone"], s["status"][:1], s["ws"])
        return _state(s, status=s["status"][0])
    ended = s["turns"][s["turn"]]
    s["turn"] ^= 1
    api.kv4_trim(cache, ended)
    api.kv4_compact(cache, s["live"], s["ws"])
    api.kv4_grow(cache, ended, s["status"], s["ws"], s["tokens"])
    return _state(s, status=s["status"][0], live=s["live"])


# ---- the work of one pass ------------------------------------------------------------------------------

def work(case):
    H, D, P, Hq = case["kv_heads"], case["dim"], case["page"], case["heads"]
    lengths = _lengths(case)
    if case["op"] in ("attention", "append"):
        news = _news(case)
        rows = sum(news)
        if case["op"] == "append":
            return dict(bytes=rows * (Hq + 2 * H) * D * 4 + rows * D * 4 + rows * H * D * 34 // 32, flops=rows * (Hq + H) * D * 3)
        seen = [sum(min(n - k + j + 1, case["window"] or n) for j in range(k)) for n, k in zip(lengths, news)]
        read = [min(n, case["window"] + k - 1 if case["window"] else n) for n, k in zip(lengths, news)]
        return dict(bytes=sum(read) * H * D * 34 // 32 + rows * Hq * D * 4, flops=sum(seen) * Hq * D * 4)
    page = H * P // 32 * 34 * D * case["layers"]
    half = case["n_seq"] // 2
    own_pages = sum(_pages(n, P) for n in lengths[:half])
    if case["op"] == "branch":
        return dict(bytes=2 * page * sum(n % P != 0 for n in lengths[:half]) + 16 * own_pages, flops=0)
    # every pass after the first finds the requests that go on behind as many free pages
    return dict(bytes=2 * page * own_pages + 16 * own_pages, flops=0)


# ---- the definition in 64 bits -------------------------------------------------------------------------

def _token_values(case, data, table_row, n, head, which):
    """K (0) or V (1) of the first n tokens of one head, by the address of every code."""
    D, P = case["dim"], case["page"]
    W, per = min(16, D // 8), D // 8
    t = torch.arange(n, device=DEV)[:, None]
    d = torch.arange(D, device=DEV)[None, :]
    half, m = t % 32 // 16, t % 16
    if which == 0:
        lane, byte = d // (D // 4) * 16 + m, d % (D // 4) // 2
        scale_at = 32 * D + half * (D // 2) + d // 32 * 16 + m
    else:
        lane, byte = m // 4 * 16 + d // (D // 16), t % 4 * (D // 32) + d % (D // 16) // 2
        scale_at = 33 * D + half * (D // 2) + (m // 4 * (D // 32) + d // 32) * 4 + t % 4
    at = which * 16 * D + half * 64 * per + byte // W * 64 * W + lane * W + byte % W
    page = table_row[(t // P).flatten()].long()[:, None]
    base = ((page * case["kv_heads"] + head) * (P // 32) + t % P // 32) * 34 * D
    flat = data.reshape(-1)
    nibble = flat[base + at].long() >> (4 * (d % 2)) & 15
    exponent = flat[base + scale_at].double() - 127
    low = nibble & 7
    size = torch.where(low < 2, low * 0.5, (1 + (low & 1) * 0.5) * torch.exp2((low // 2 - 1).double()))
    return torch.where(nibble >= 8, -size, size) * torch.exp2(exponent)


def _nearest(x, dtype):
    """x [..., D] in 64 bits -> the nearest values that the format holds."""
    lowest, highest = EXPONENTS[dtype]
    g = x.unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(torch.where(top > 0, top, 1.0)))
    e = torch.where(top >= torch.exp2(e + 1), e + 1, torch.where(top < torch.exp2(e), e - 1, e))
    e = torch.where(top > 0, torch.where(top > 1.75 * torch.exp2(e), e - 1, e - 2), lowest).clamp(lowest, highest)
    level = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    away = ((g.abs() / torch.exp2(e))[..., None] - level).abs()
    away[..., 0::2] -= 1e-12 * away[..., 0::2]
    return (torch.copysign(level[away.argmin(-1)], g) * torch.exp2(e)).flatten(-2)


def exact(case, seed):
    if case["op"] not in ("attention", "append"):
        return None
    s = prepare(case, seed)
    D, P, Hq, H = case["dim"], case["page"], case["heads"], case["kv_heads"]
    lengths, news, slots = _lengths(case), _news(case), s["slots"].tolist()
    x = s["qkv"].double().reshape(s["rows"], Hq + 2 * H, D)
    row = 0
    if case["op"] == "append":
        out = x.clone()
        axis = torch.zeros(D // 2, dtype=torch.int64, device=DEV)
        if s["positions"] is not None:
            ends = s["axis_pairs"][0], s["axis_pairs"][0] + s["axis_pairs"][1]
            axis[ends[0]:] = 1
            axis[ends[1]:] = 2
        pair = torch.arange(D // 2, device=DEV)
        for n, k in zip(lengths, news):
            r = torch.arange(row, row + k, device=DEV)
            at = (r - row + n - k)[:, None].expand(k, D // 2) if s["positions"] is None else s["positions"][axis[None, :], r[:, None]].long()
            z = torch.complex(s["rotary"][at, pair].double(), s["rotary"][at, pair + D // 2].double())[:, None]
            y = z * torch.complex(x[r, :Hq + H, :D // 2], x[r, :Hq + H, D // 2:])
            out[r, :Hq + H] = torch.cat([y.real, y.imag], -1)
            row += k
        out[:, Hq:] = _nearest(out[:, Hq:], case["dtype"])
        return dict(out=out.flatten(1), data=None)
    out = torch.zeros(s["rows"], Hq, D, dtype=torch.float64, device=DEV)
    for i, (n, k) in enumerate(zip(lengths, news)):
        place = torch.arange(n - k, n, device=DEV)[:, None]
        t = torch.arange(n, device=DEV)[None, :]
        hidden = (t > place) | (t <= place - case["window"] if case["window"] else t < 0)
        for h in range(H):
            keys, values = (_token_values(case, s["data"][0], s["table"][slots[i]], n, h, w) for w in (0, 1))
            q = x[row:row + k, h * (Hq // H):(h + 1) * (Hq // H)]
            score = (q.reshape(-1, D) @ keys.T / math.sqrt(D)).reshape(k, Hq // H, n).masked_fill(hidden[:, None], -math.inf)
            out[row:row + k, h * (Hq // H):(h + 1) * (Hq // H)] = (torch.softmax(score, -1).reshape(-1, n) @ values).reshape(k, Hq // H, D)
        row += k
    return out.flatten(1)
