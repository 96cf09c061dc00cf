"""The operators behind a model's last layer, on weights in 8-bit floating point: a weight and rows brought to 8 bits with
a scale for each block of 128, their product, the log probabilities of given tokens with entropy and top alternatives,
and all of it in one call, from hidden rows to log probabilities.

`listed()` names twelve cases, `draw(rng)` gives another one of the same ranges.  `run` computes the operators in
plain torch where `own` is false and calls `paper_2507_01299_amd.api` where it is true; `exact` states them in 64 bits;
`work` gives the bytes and operations of one pass.

The format.  A code is an e4m3 number (4 exponent bits, 3 of mantissa, at most 448).  A block of values (128 x 128 of a weight,
128 neighbours of a row) has the scale 2^e with the least e >= -64 for which its largest magnitude is at most 448 * 2^e, held as the
byte e + 127; its codes are the numbers nearest to value / 2^e, ties to the even one.  Codes of a weight [d_in, d_out] are stored [d_out, d_in],
d_in rounded up to 16 (zeros), its scales by block [d_out / 128, d_in / 128], the latter rounded up to 4 (127); codes of rows [n, d] and
their scales [n, d / 128] the same way.
"""
import math

import torch
import torch.nn.functional as F

own = False

DEV = "cuda:0"
TYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
E4M3 = torch.float8_e4m3fn
LEAST = -64          # exponent of a scale


# ---- the cases ------------------------------------------------------------------------------------------

def listed():
    return [
        # the attention output projection of a 7B or 8B model, one token: latency
        dict(name="dense_7b_o_1", op="dense", rows=1, d_in=4096, d_out=4096, dtype="bf16"),
        # the down projection of a 7B model over a short prompt: rows that fill no tile, few output columns, a long sum
        dict(name="dense_7b_down_333", op="dense", rows=333, d_in=11008, d_out=4096, dtype="f16"),
        # gate|up of a 70B model over a long prompt: the largest product
        dict(name="dense_70b_gate_up_4096", op="dense", rows=4096, d_in=8192, d_out=57344, dtype="bf16"),
        # a decode batch's rows to 8 bits, once for several products
        dict(name="rows_5x4096", op="rows", rows=5, d=4096, dtype="f16"),
        # the same for the MLP's inner rows of a 70B model's prompt
        dict(name="rows_4096x28672", op="rows", rows=4096, d=28672, dtype="bf16"),
        # preparing the weight of q|k|v of an 8B model
        dict(name="weight_8b_qkv", op="weight", d_in=4096, d_out=6144, dtype="bf16"),
        # preparing an odd weight: sides that are no multiples of 128
        dict(name="weight_odd", op="weight", d_in=11016, d_out=13832, dtype="f16"),
        # one generated token: its log probability and the five best alternatives
        dict(name="logprobs_1x32000", op="logprobs", rows=1, vocab=32000, given=1, top=5, masked=0.0, dtype="f16"),
        # scored answers over a grammar's mask: 32-bit logits, an odd vocabulary, four candidates a row
        dict(name="logprobs_77x50257", op="logprobs", rows=77, vocab=50257, given=4, top=8, masked=0.4, dtype="f32"),
        # a document's log probabilities with twenty alternatives for each token
        dict(name="logprobs_2048x128256", op="logprobs", rows=2048, vocab=128256, given=1, top=20, masked=0.0, dtype="bf16"),
        # a decode batch through the head of an 8B model: last hidden rows to the sampled tokens' log probabilities
        dict(name="score_13x128256", op="score", rows=13, d=4096, vocab=128256, given=1, dtype="bf16"),
        # perplexity of a document by the head of a 70B model
        dict(name="score_2048x32000", op="score", rows=2048, d=8192, vocab=32000, given=1, dtype="f16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["dense", "dense", "dense", "dense", "rows", "weight", "logprobs", "logprobs", "score", "score"])
    dtype = rng.choice(["f16", "bf16"])
    eight = lambda lo, hi: 8 * _log_int(rng, lo // 8, hi // 8)   # noqa: E731
    if op == "dense":
        d_in, d_out = eight(512, 28672), eight(512, 57344)
        rows = _log_int(rng, 1, min(8192, int(4096 * 8192 * 57344 / (d_in * d_out))))
        return dict(op=op, rows=rows, d_in=d_in, d_out=d_out, dtype=dtype)
    if op == "rows":
        d = eight(512, 28672)
        return dict(op=op, rows=_log_int(rng, 1, 4096 * 28672 // d), d=d, dtype=dtype)
    if op == "weight":
        return dict(op=op, d_in=eight(512, 14336), d_out=eight(512, 28672), dtype=dtype)
    vocab = _log_int(rng, 4000, 200000)
    if op == "logprobs":
        dtype = rng.choice(["f16", "bf16", "f32"])
        rows = _log_int(rng, 1, 2048 * 128256 // vocab // (2 if dtype == "f32" else 1))
        return dict(op=op, rows=rows, vocab=vocab, given=rng.choice([1, 1, rng.randint(2, 9)]), top=rng.choice([0, 1, rng.randint(2, 32)]),
                    masked=rng.choice([0.0, 0.0, 0.4]), dtype=dtype)
    d = 128 * rng.choice([16, 20, 32, 40, 64])
    rows = _log_int(rng, 1, min(4096, int(4096 * 8192 * 57344 / (4 * d * vocab))))
    return dict(op=op, rows=rows, d=d, vocab=vocab, given=rng.choice([1, 1, 4]), dtype=dtype)


# ---- the format ----------------------------------------------------------------------------------------

def _blocks(n):
    return -(-n // 128)


def _exponents(m):
    """Largest magnitudes of blocks -> the exponents of their scales."""
    part, power = torch.frexp(m.clamp(min=2.0 ** -70))
    return (power - 9 + (part > 0.875).to(power.dtype)).clamp(min=LEAST)


def _bytes(e):
    """Exponents [rows, blocks] -> scale bytes, blocks rounded up to 4."""
    return F.pad(e + 127, (0, -e.shape[1] % 4), value=127).to(torch.uint8)


def _codes_of_rows(v):
    """v [n, d] in 32 bits -> codes [n, d up to 16] and scale bytes [n, d / 128 up to 4]."""
    n, d = v.shape
    v = F.pad(v, (0, 128 * _blocks(d) - d)).unflatten(1, (-1, 128))
    e = _exponents(v.abs().amax(-1))
    codes = (v * torch.exp2(-e.float())[..., None]).to(E4M3).flatten(1)
    return codes[:, :-(-d // 16) * 16].contiguous(), _bytes(e)


def _codes_of_weight(W):
    """W [d_in, d_out] in 32 bits -> codes [d_out, d_in up to 16] and scale bytes [d_out / 128, d_in / 128 up to 4]."""
    d_in, d_out = W.shape
    v = F.pad(W.t(), (0, 128 * _blocks(d_in) - d_in, 0, 128 * _blocks(d_out) - d_out))
    v = v.unflatten(0, (-1, 128)).unflatten(2, (-1, 128))
    e = _exponents(v.abs().amax((1, 3)))
    codes = (v * torch.exp2(-e.float())[:, None, :, None]).to(E4M3).flatten(2).flatten(0, 1)
    return codes[:d_out, :-(-d_in // 16) * 16].contiguous(), _bytes(e)


def _values(codes, scales, rows_of_block, d):
    """What codes stand for, in 32 bits."""
    unit = torch.exp2(scales[:, :_blocks(d)].float() - 127.0).repeat_interleave(rows_of_block, 0)[:codes.shape[0]]
    return codes[:, :d].float() * unit.repeat_interleave(128, 1)[:, :d]


# ---- what a program has in hand ------------------------------------------------------------------------

def _hidden(g, rows, d, dtype):
    """Rows behind a norm: every channel about 1, a few channels 20 times that."""
    strong = torch.where(torch.rand(d, generator=g, device=DEV) < 4 / 4096, 20.0, 1.0)
    return (torch.randn(rows, d, generator=g, device=DEV) * strong).to(TYPE[dtype])


def _given(g, rows, n, vocab):
    """Tokens whose log probability is asked for; one place in sixteen is padding."""
    ids = torch.randint(vocab, (rows, n), generator=g, device=DEV)
    pad = (torch.rand(rows, n, generator=g, device=DEV) < 1 / 16) & (torch.arange(rows * n, device=DEV).view(rows, n) > 0)
    return torch.where(pad, -1, ids).int()


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    op, s = case["op"], dict(case=case)
    if op == "rows":
        s["x"] = _hidden(g, case["rows"], case["d"], case["dtype"])
    elif op == "weight":
        s["W"] = (torch.randn(case["d_in"], case["d_out"], generator=g, device=DEV) * 0.02).to(TYPE[case["dtype"]])
    elif op == "dense":
        s["x"] = _hidden(g, case["rows"], case["d_in"], case["dtype"])
        W = (torch.randn(case["d_in"], case["d_out"], generator=g, device=DEV) * 0.02).to(TYPE[case["dtype"]])
        s["codes"], s["scales"] = _codes_of_weight(W.float())
        s["y"] = torch.empty(case["rows"], case["d_out"], dtype=TYPE[case["dtype"]], device=DEV)
    else:
        rows, V, n = case["rows"], case["vocab"], case["given"]
        s["given"] = _given(g, rows, n, V)
        if op == "score":          # rows that lean towards their first token, as a trained model's do
            W = (torch.randn(case["d"], V, generator=g, device=DEV) * 0.02).to(TYPE[case["dtype"]])
            x = torch.randn(rows, case["d"], generator=g, device=DEV)
            lean = W.t()[s["given"][:, 0].clamp(min=0).long()].float() / (0.0004 * case["d"])
            x = x + lean * (12.0 * torch.rand(rows, 1, generator=g, device=DEV))
            s["x"] = x.to(TYPE[case["dtype"]])
            s["codes"], s["scales"] = _codes_of_weight(W.float())
        else:
            z = torch.randn(rows, V, generator=g, device=DEV) * 2.2
            best = torch.randint(V, (rows, 8), generator=g, device=DEV)
            z.scatter_add_(1, best, 12.0 * torch.rand(rows, 8, generator=g, device=DEV))
            if case["masked"]:     # tokens that a grammar forbids at this place
                z.masked_fill_(torch.rand(rows, V, generator=g, device=DEV) < case["masked"], -math.inf)
            s["logits"] = z.to(TYPE[case["dtype"]])
            s["top_id"] = torch.empty(rows, case["top"], dtype=torch.int32, device=DEV)
            s["top_logp"] = torch.empty(rows, case["top"], device=DEV)
        s["logp"] = torch.empty(rows, n, device=DEV)
        s["entropy"] = torch.empty(rows, device=DEV)
    return s


# ---- the operators ---------------------------------------------------------------------------------------

def _logprobs(z, given):
    """z [n, V] in 32 bits -> (log probabilities of the given tokens, entropy, what to take from a logit for its own)."""
    m = z.amax(-1, keepdim=True)
    e = (z - m).exp()
    total = e.sum(-1, keepdim=True)
    entropy = total.log()[:, 0] - torch.where(e > 0, e * (z - m), 0.0).sum(-1) / total[:, 0]
    base = m + total.log()
    logp = z.gather(1, given.clamp(min=0).long()) - base
    return torch.where(given < 0, 0.0, logp), entropy, base


def _top(z, n):
    """The ids of the n largest of each row, the lower id first among equals."""
    bits = (z + 0.0).view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() << 32
    return (order | (0xFFFFFFFF - torch.arange(z.shape[1], device=DEV))).topk(n, 1).indices


def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    op = case["op"]
    if op == "rows":
        return dict(zip(("codes", "scales"), _codes_of_rows(s["x"].float())))
    if op == "weight":
        return dict(zip(("codes", "scales"), _codes_of_weight(s["W"].float())))
    if op == "logprobs":
        z = s["logits"].float()
        logp, entropy, base = _logprobs(z, s["given"])
        if not case["top"]:
            return dict(logp=logp, entropy=entropy)
        ids = _top(z, case["top"])
        return dict(logp=logp, entropy=entropy, top_id=ids.int(), top_logp=z.gather(1, ids) - base)
    d = s["x"].shape[1]
    y = _values(*_codes_of_rows(s["x"].float()), 1, d) @ _values(s["codes"], s["scales"], 128, d).t()
    if op == "dense":
        return y.to(TYPE[case["dtype"]])
    return dict(zip(("logp", "entropy"), _logprobs(y, s["given"])))


def _run_own(s, case):
    from paper_2507_01299_amd import api
    op, dtype = case["op"], case["dtype"]
    if op == "rows":
        return dict(zip(("codes", "scales"), api.quantize_rows8(s["x"], dtype)))
    if op == "weight":
        return dict(zip(("codes", "scales"), api.quantize_w8(s["W"], dtype)))
    if op == "dense":
        if "ws" not in s:
            s["ws"] = api.dense_w8_workspace(case["rows"], case["d_in"], case["d_out"])
        return api.dense_w8(s["codes"], s["scales"], s["x"], s["y"], dtype, s["ws"])
    if op == "logprobs":
        if "ws" not in s:
            s["ws"] = api.logprobs_workspace(case["rows"], case["vocab"], case["top"])
        if not case["top"]:
            api.logprobs(s["logits"], s["given"], s["logp"], s["ws"], entropy=s["entropy"])
            return dict(logp=s["logp"], entropy=s["entropy"])
        api.logprobs(s["logits"], s["given"], s["logp"], s["ws"], entropy=s["entropy"], top_id=s["top_id"], top_logp=s["top_logp"])
        return dict(logp=s["logp"], entropy=s["entropy"], top_id=s["top_id"], top_logp=s["top_logp"])
    if "ws" not in s:
        s["ws"] = api.score_w8_workspace(case["rows"], case["d"], case["vocab"])
    api.score_w8(s["codes"], s["scales"], s["x"], s["given"], s["logp"], dtype, s["ws"], entropy=s["entropy"])
    return dict(logp=s["logp"], entropy=s["entropy"])


# ---- the work of one pass ------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "rows":
        n, d = case["rows"], case["d"]
        return dict(bytes=n * d * 3 + n * _blocks(d), flops=4 * n * d)
    if op == "logprobs":
        n, V = case["rows"], case["vocab"]
        return dict(bytes=n * (V * (4 if case["dtype"] == "f32" else 2) + 8 * case["given"] + 4 + 8 * case["top"]), flops=6 * n * V)
    d_in, d_out = (case["d"], case["vocab"]) if op == "score" else (case["d_in"], case["d_out"])
    scales = _blocks(d_in) * _blocks(d_out)
    if op == "weight":
        return dict(bytes=3 * d_in * d_out + scales, flops=4 * d_in * d_out)
    n = case["rows"]
    held = d_in * d_out + scales + 2 * n * d_in
    if op == "score":
        return dict(bytes=held + n * (8 * case["given"] + 4), flops=2 * n * d_in * d_out + 6 * n * d_out)
    return dict(bytes=held + 2 * n * d_out, flops=2 * n * d_in * d_out)


# ---- the definition in 64 bits --------------------------------------------------------------------------

def _nearest_e4m3(v):
    """The nearest number with four significant bits, exponents from -6 on, at most 448; ties to the even one."""
    unit = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return ((v / unit).round() * unit).clamp(-448.0, 448.0)


def _held(v, rows_of_block):
    """What blocks of rows_of_block x 128 of v [n, d] (64 bits) hold: codes, scale bytes, and the values."""
    n, d = v.shape
    p = v.new_zeros(-(-n // rows_of_block) * rows_of_block, _blocks(d) * 128)
    p[:n, :d] = v
    p = p.view(-1, rows_of_block, _blocks(d), 128)
    top = p.abs().amax((1, 3))
    e = torch.full_like(top, LEAST)
    for k in range(LEAST, 121):
        e = torch.where(top > 448.0 * 2.0 ** k, k + 1.0, e)
    unit = torch.exp2(e)[:, None, :, None]
    codes = _nearest_e4m3(p / unit)
    scales = torch.full((e.shape[0], -(-e.shape[1] // 4) * 4), 127, dtype=torch.uint8, device=v.device)
    scales[:, :e.shape[1]] = (e + 127).to(torch.uint8)
    return codes.flatten(2).flatten(0, 1)[:n], scales, (codes * unit).flatten(2).flatten(0, 1)[:n, :d]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("rows", "weight"):
        v, high = (s["x"].double(), 1) if op == "rows" else (s["W"].double().t(), 128)
        codes, scales, _ = _held(v, high)
        return dict(codes=codes[:, :-(-v.shape[1] // 16) * 16].contiguous(), scales=scales)
    if op == "logprobs":
        z = s["logits"].double()
    else:
        _, _, x = _held(s["x"].double(), 1)
        W = s["codes"][:, :x.shape[1]].double()
        unit = 2.0 ** (s["scales"].double() - 127.0)
        at_in = torch.arange(W.shape[1], device=DEV) // 128
        for i in range(unit.shape[0]):
            W[128 * i:128 * i + 128] *= unit[i][at_in]
        z = x @ W.t()
        if op == "dense":
            return z
    p = torch.log_softmax(z, -1)
    logp = p.gather(1, s["given"].long().clamp(min=0)).masked_fill(s["given"] < 0, 0.0)
    entropy = -(p.exp() * p.masked_fill(p == -math.inf, 0.0)).sum(-1)
    if op == "score" or not case["top"]:
        return dict(logp=logp, entropy=entropy)
    return dict(logp=logp, entropy=entropy, top_id=None, top_logp=p.topk(case["top"], 1).values)
