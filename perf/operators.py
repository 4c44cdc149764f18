"""The operators with which one batch of the library's layers serves many requests, as their users call them.

Three kinds of case, all through the public entry points of paper_2505_00232_amd.binding:

"append"  the QKV layer's output for the new tokens of a batch of requests: queries and keys rotated (pairs half a
          rotation apart or side by side, all of the head or its first values, frequencies scaled for long contexts), keys
          and values appended to a paged cache held in 4 bits.  Returned: the queries, and the values the cache now holds.
"attend"  attention of the new tokens of a batch of requests over that cache, each request with a length of its own.
"adapt"   low-rank adapters beside a shared layer: out = y + scale[a] B[a] (A[a] x), row by row, a = ids[row].

The plain forms hold the cache as codes, steps and offsets side by side, in pages of the same 64 positions.
Shapes: the Llama-3.1-8B and Gemma2-2B layers of this repository's benchmark, and generic ones.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE, GROUP = 64, 32
LLAMA = dict(h_q=32, h_kv=8, d=128)
GEMMA = dict(h_q=8, h_kv=4, d=256)


def listed():
    return [
        # one user's next token in a chat: nothing but latency
        dict(name="append_one", kind="append", batch=1, tokens=1, fewest=1, context=1279, shortest=1279, rot=128, pairs="half", stretch=8.0, **LLAMA),
        # a server's decode step: the next token of 64 requests
        dict(name="append_64_requests", kind="append", batch=64, tokens=1, fewest=1, context=4000, shortest=33, rot=128, pairs="half", stretch=8.0, **LLAMA),
        # prompts of odd lengths, half of the head rotated, pairs side by side
        dict(name="append_prompts_part", kind="append", batch=3, tokens=777, fewest=61, context=900, shortest=400, rot=128, pairs="interleaved", stretch=1.0, **GEMMA),
        # a long prompt behind another, far out in a long context
        dict(name="append_4096_far", kind="append", batch=1, tokens=4096, fewest=4096, context=100000, shortest=100000, rot=128, pairs="half", stretch=8.0, **LLAMA),
        # one user's next token
        dict(name="attend_one", kind="attend", batch=1, tokens=1, fewest=1, context=1280, shortest=1280, **LLAMA),
        # a server's decode step, requests of every length
        dict(name="attend_32_requests", kind="attend", batch=32, tokens=1, fewest=1, context=8192, shortest=100, **LLAMA),
        # the smaller model's decode step: large heads, few of them
        dict(name="attend_20_gemma", kind="attend", batch=20, tokens=1, fewest=1, context=1500, shortest=700, **GEMMA),
        # prompts read from their first token on
        dict(name="attend_prompts", kind="attend", batch=2, tokens=1024, fewest=601, context=1024, shortest=601, **LLAMA),
        # a chunk of a long prompt beside the next tokens of other requests
        dict(name="attend_chunk_and_tokens", kind="attend", batch=6, tokens=300, fewest=1, context=6300, shortest=500, others=1, **LLAMA),
        # one request's adapter beside the QKV layer
        dict(name="adapt_one", kind="adapt", M=1, K=4096, N=6144, rank=16, count=32, requests=1),
        # 64 requests with 40 adapters among them, some with none
        dict(name="adapt_64_requests", kind="adapt", M=64, K=4096, N=4096, rank=16, count=40, requests=64),
        # prompts of five requests, a wide layer, adapters of a higher rank
        dict(name="adapt_prompts", kind="adapt", M=2048, K=4096, N=28672, rank=64, count=8, requests=5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    pick = rng.random()
    if pick < 0.35:
        return dict(LLAMA)
    if pick < 0.6:
        return dict(GEMMA)
    d, h_kv = rng.choice([64, 128, 256]), rng.choice([1, 2, 4, 8])
    return dict(h_q=h_kv * rng.choice([1, 2, 3, 4, 8]), h_kv=h_kv, d=d)


def draw(rng):
    pick = rng.random()
    if pick < 0.3:
        h = _heads(rng)
        few = rng.random() < 0.5
        batch = _log_int(rng, 1, 96) if few else rng.randint(1, 4)
        tokens = rng.choice([1, 1, 1, 2, 5]) if few else _log_int(rng, 16, 1024)
        context = tokens + _log_int(rng, 1, 4000 if few else 30000)
        return dict(kind="append", batch=batch, tokens=tokens, fewest=rng.randint(1, tokens), context=context, shortest=rng.randint(tokens, context),
                    rot=h["d"] if rng.random() < 0.6 else 16 * rng.randint(1, h["d"] // 16), pairs=rng.choice(["half", "interleaved"]),
                    stretch=rng.choice([1.0, 4.0, 8.0]), **h)
    if pick < 0.72:
        h = _heads(rng)
        if rng.random() < 0.6:
            batch, tokens = _log_int(rng, 1, 32), rng.choice([1, 1, 1, 2, 4])
            context = tokens + _log_int(rng, 1, 8000 // (1 + h["d"] // 200))
        else:
            batch, tokens = rng.randint(1, 3), _log_int(rng, 9, 1000)
            context = tokens + (0 if rng.random() < 0.5 else _log_int(rng, 10, 4000))
        return dict(kind="attend", batch=batch, tokens=tokens, fewest=rng.randint(1, tokens), context=context, shortest=rng.randint(tokens, context), **h)
    few = rng.random() < 0.6
    M = _log_int(rng, 1, 128) if few else _log_int(rng, 128, 2048)
    return dict(kind="adapt", M=M, K=32 * _log_int(rng, 16, 300), N=_log_int(rng, 100, 12000), rank=rng.choice([8, 16, 32, 64]), count=rng.randint(1, 48 if few else 8),
                requests=M if few else rng.randint(1, 6))


# ---------------------------------------------------------------- what the cases are made of
def _spread(n, most, least, step):
    """n lengths of a batch's requests, the first the longest."""
    return [most if b == 0 else least + int((most - least + 1) * ((b * step + 0.37) % 1.0)) for b in range(n)]


def _lengths(c):
    """(new tokens, positions with them) of each request."""
    S = [c["tokens"]] + [c["others"]] * (c["batch"] - 1) if "others" in c else _spread(c["batch"], c["tokens"], c["fewest"], 0.7548776662)
    n = _spread(c["batch"], c["context"], c["shortest"], 0.6180339887)
    return S, [max(a, b) for a, b in zip(S, n)]


def _row_adapters(c):
    """The adapter of each row: requests one behind the other, every ninth without one."""
    r = (np.arange(c["M"]) * c["requests"]) // c["M"]
    return np.where(r % 9 == 8, -1, r % c["count"]).astype(np.int32)


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float16)


def _frequencies(c):
    """Parameters of the rotation's table: base, and frequencies lowered by `stretch` where a wave is long against 8192 positions."""
    return dict(base=500000.0, factor=c["stretch"], original_positions=8192 if c["stretch"] > 1.0 else 0, low_turns=1.0, high_turns=4.0)


def _batch(c, gen):
    """The requests of a batch: new tokens one behind the other, positions, and a page table over shuffled pages."""
    S, n = _lengths(c)
    width = max((x + PAGE - 1) // PAGE for x in n)
    used = [(x + PAGE - 1) // PAGE for x in n]
    total = sum(used) + 3  # (a cache is larger than what a batch uses)
    order = torch.randperm(total, generator=gen, device="cuda").int().cpu()
    table, at = torch.full((c["batch"], width), -1, dtype=torch.int32), 0
    for b, u in enumerate(used):
        table[b, :u] = order[at:at + u]
        at += u
    start = torch.tensor([0] + list(np.cumsum(S)), dtype=torch.int32)
    return dict(token_start=start.cuda(), context=torch.tensor(n, dtype=torch.int32).cuda(), page_table=table.cuda(), pages=total, tokens=sum(S), most=max(S), longest=max(n))


def _inputs(c, seed):
    gen = _generator(seed)
    if c["kind"] == "adapt":
        x, y = _normal(gen, c["M"], c["K"]), _normal(gen, c["M"], c["N"])
        a = _normal(gen, c["count"], c["rank"], c["K"]) * (1.0 / math.sqrt(c["K"]))
        b = _normal(gen, c["count"], c["N"], c["rank"]) * (1.0 / math.sqrt(c["rank"]))
        scale = torch.rand(c["count"], generator=gen, device="cuda") + 0.5
        return dict(x=x, y=y, a=a, b=b, scale=scale, ids=torch.from_numpy(_row_adapters(c)).cuda())
    s = _batch(c, gen)
    h_kv, d = c["h_kv"], c["d"]
    # keys have channels of their own size and mean, as trained layers give them
    size, mean = torch.exp(0.4 * torch.randn((h_kv, d), generator=gen, device="cuda")), 0.5 * torch.randn((h_kv, d), generator=gen, device="cuda")
    if c["kind"] == "append":
        s["qkv"] = _normal(gen, s["tokens"], (c["h_q"] + 2 * h_kv) * d)
        k = s["qkv"][:, c["h_q"] * d:(c["h_q"] + h_kv) * d]
        k.copy_(k.float() * size.flatten() + mean.flatten())
        return s
    s["q"] = _normal(gen, s["tokens"], c["h_q"] * d)
    rows = int(sum(_lengths(c)[1]))
    s["k"] = (_normal(gen, rows, h_kv, d) * size + mean).half()  # of request 0's positions, then request 1's ...
    s["v"] = _normal(gen, rows, h_kv, d)
    return s


# ---------------------------------------------------------------- the plain forms
def _to_half(y):
    """64-bit values rounded to binary16 once: to 32 bits by rounding to odd, then to the nearest."""
    f = y.float()
    f64, bits = f.double(), f.view(torch.int32)
    odd = torch.where(f64.abs() > y.abs(), bits - 1, bits) | 1
    return torch.where(f64 == y, bits, odd).view(torch.float32).half()


def _quantize(x):
    """Codes 0 .. 15, and a step and an offset for each 32 values: value = offset + step (code - 8)."""
    g = x.float().unflatten(-1, (-1, GROUP))
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    step = ((hi - lo) / 15.0).half()
    offset = (lo + 8.0 * step.float()).half()
    inv = torch.where(step > 0, 1.0 / step.float(), 0.0)
    code = (torch.round((g - offset.float()) * inv) + 8.0).clamp(0.0, 15.0)
    return code.to(torch.uint8).flatten(-2), step.squeeze(-1), offset.squeeze(-1)


def _values(code, step, offset):
    g = code.float().unflatten(-1, (-1, GROUP)) - 8.0
    return (offset.float().unsqueeze(-1) + step.float().unsqueeze(-1) * g).flatten(-2)


def _plain_cache(c, pages):
    shape, e = (pages, PAGE, c["h_kv"]), torch.zeros
    return [(e((*shape, c["d"]), dtype=torch.uint8, device="cuda"), e((*shape, c["d"] // GROUP), dtype=torch.float16, device="cuda"),
             e((*shape, c["d"] // GROUP), dtype=torch.float16, device="cuda")) for _ in range(2)]


def _places(s):
    """Request, position, page and place in it of each new token."""
    row = torch.arange(s["tokens"], device="cuda")
    b = torch.bucketize(row, s["token_start"][1:].long(), right=True)
    pos = s["context"].long()[b] - (s["token_start"].long()[b + 1] - row)
    return b, pos, s["page_table"].long()[b, pos // PAGE], pos % PAGE


def _store(cache, page, place, rows):
    for held, new in zip(cache, _quantize(rows)):
        held[page, place] = new


def _append(s):
    c = s["case"]
    h_q, h_kv, d, rot = c["h_q"], c["h_kv"], c["d"], c["rot"]
    _, pos, page, place = _places(s)
    x = s["qkv"].view(s["tokens"], h_q + 2 * h_kv, d)
    qk = x[:, :h_q + h_kv].double()
    cos, sin = (s["table"][pos, :, i].double().unsqueeze(1) for i in (0, 1))
    first, second = (qk[..., :rot // 2], qk[..., rot // 2:rot]) if c["pairs"] == "half" else (qk[..., 0:rot:2], qk[..., 1:rot:2])
    a, b = first * cos - second * sin, second * cos + first * sin
    turned = torch.cat([a, b], -1) if c["pairs"] == "half" else torch.stack([a, b], -1).flatten(-2)
    qk = torch.cat([_to_half(turned), x[:, :h_q + h_kv, rot:]], -1)
    for cache, rows in zip(s["cache"], (qk[:, h_q:], x[:, h_q + h_kv:])):
        _store(cache, page, place, rows)
    k, v = (_values(*(held[page, place] for held in cache)).half() for cache in s["cache"])
    return {"q": qk[:, :h_q].reshape(s["tokens"], h_q * d), "k": k, "v": v}


def _attend(s):
    c = s["case"]
    B, h_q, h_kv, d, most = c["batch"], c["h_q"], c["h_kv"], c["d"], s["most"]
    g = h_q // h_kv
    start, n = s["token_start"].long(), s["context"].long()
    S = start[1:] - start[:-1]
    at = torch.arange(most, device="cuda")
    row = (start[:-1, None] + at).clamp(max=s["tokens"] - 1)
    q = s["q"].float()[row].view(B, most, h_kv, g, d).permute(0, 2, 1, 3, 4).reshape(B, h_kv, most * g, d)
    page = s["page_table"].long().clamp(min=0)
    k, v = (_values(*(held[page] for held in cache)).flatten(1, 2).transpose(1, 2).contiguous() for cache in s["cache"])  # [B, h_kv, positions, d]
    sees = torch.arange(k.shape[2], device="cuda") < (n - S)[:, None, None] + at[None, :, None] + 1
    sees = sees.repeat_interleave(g, 1).unsqueeze(1)
    score = (torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(d)).masked_fill_(~sees, -torch.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    out = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    b, pos, _, _ = _places(s)
    out = out.view(B, h_kv, most, g, d).transpose(1, 2)[b, pos - (n - S)[b]]
    return {"out": out.reshape(s["tokens"], h_q * d).half()}


def _adapt(s):
    c = s["case"]
    ids = s["ids"]
    held = torch.arange(c["count"], device="cuda").repeat_interleave(c["rank"])
    low = torch.matmul(s["x"].float(), s["a"].float().flatten(0, 1).t())
    low = low * (ids[:, None] == held) * s["scale"][held]
    more = torch.matmul(low, s["b"].float().transpose(1, 2).flatten(0, 1))
    return {"out": torch.where(ids[:, None] >= 0, s["y"].float() + more, s["y"].float()).half()}


# ---------------------------------------------------------------- the calls a user's program makes
def _rotary(c):
    from paper_2505_00232_amd import binding as B
    f = _frequencies(c)
    return B.make_rotary(c["rot"], f["base"], layout=B.QFC_ROPE_HALF if c["pairs"] == "half" else B.QFC_ROPE_INTERLEAVED, factor=f["factor"],
                         original_positions=f["original_positions"], low_turns=f["low_turns"], high_turns=f["high_turns"])


def _own_prepare(s):
    from paper_2505_00232_amd import binding as B
    c = s["case"]
    if c["kind"] == "adapt":
        s["adapters"] = B.Adapters(s["a"], s["b"], s["scale"])
        s["workspace"] = torch.empty(B.qfc_adapters_workspace_size(s["adapters"], c["M"]), dtype=torch.uint8, device="cuda")
        s["out"] = torch.empty_like(s["y"])
        return
    h_q, h_kv, d = c["h_q"], c["h_kv"], c["d"]
    s["cache"] = B.PagedCache(s["pages"], h_kv, d)
    s["requests"] = B.Requests(s["token_start"], s["context"], s["page_table"], s["tokens"], s["most"], s["longest"])
    E = lambda *shape: torch.empty(shape, dtype=torch.float16, device="cuda")
    if c["kind"] == "append":
        s["rotary"] = _rotary(c)
        s["table"] = B.qfc_rotary_table(s["rotary"], s["longest"])
        s["q"], s["k"], s["v"] = E(s["tokens"], h_q * d), E(s["tokens"], h_kv, d), E(s["tokens"], h_kv, d)
        return
    # the positions that are in the cache already, without a rotation: they are what the cache is said to hold
    rows = s["k"].shape[0]
    qkv = torch.cat([s["k"].view(rows, -1), s["k"].view(rows, -1), s["v"].view(rows, -1)], 1)
    start = torch.nn.functional.pad(s["context"].cumsum(0, dtype=torch.int32), (1, 0))
    B.qfc_append_q4(qkv, B.Requests(start, s["context"], s["page_table"], rows, s["longest"], s["longest"]), h_kv, None, None, s["cache"], E(rows, h_kv * d))
    s["workspace"] = torch.empty(B.qfc_attention_q4_workspace_size(s["requests"], h_q, s["cache"]), dtype=torch.uint8, device="cuda")
    s["out"] = E(s["tokens"], h_q * d)
    torch.cuda.synchronize()


def _own_run(s):
    from paper_2505_00232_amd import binding as B
    c = s["case"]
    if c["kind"] == "append":
        B.qfc_append_q4(s["qkv"], s["requests"], c["h_q"], s["rotary"], s["table"], s["cache"], s["q"])
        B.qfc_read_q4(s["requests"], s["cache"], s["k"], s["v"])
        return {"q": s["q"], "k": s["k"], "v": s["v"]}
    if c["kind"] == "attend":
        B.qfc_attention_q4(s["q"], s["requests"], c["h_q"], s["cache"], s["workspace"], s["out"])
    else:
        B.qfc_add_adapters(s["x"], s["ids"], s["adapters"], s["y"], s["workspace"], s["out"])
    return {"out": s["out"]}


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = dict(case)
    if own:
        _own_prepare(s)
    elif case["kind"] != "adapt":
        s["cache"] = _plain_cache(case, s["pages"])
        if case["kind"] == "append":
            f, i = _frequencies(case), torch.arange(case["rot"] // 2, device="cuda", dtype=torch.float64)
            freq = torch.exp(i * (-2.0 / case["rot"] * math.log(f["base"])))
            if f["original_positions"]:
                keep = ((f["original_positions"] * freq / (2.0 * math.pi) - f["low_turns"]) / (f["high_turns"] - f["low_turns"])).clamp(0.0, 1.0)
                freq = freq * (keep + (1.0 - keep) / f["factor"])
            angle = torch.arange(s["longest"], device="cuda", dtype=torch.float64)[:, None] * freq
            s["table"] = torch.stack([angle.cos(), angle.sin()], -1).float()
        else:
            every = dict(tokens=s["k"].shape[0], token_start=torch.nn.functional.pad(s["context"].cumsum(0), (1, 0)), context=s["context"], page_table=s["page_table"])
            _, _, page, place = _places(every)
            for cache, rows in zip(s["cache"], (s["k"], s["v"])):
                _store(cache, page, place, rows)
    s.pop("k", None) if case["kind"] == "attend" else None
    s.pop("v", None) if case["kind"] == "attend" else None
    return s


def run(state):
    if own:
        return _own_run(state)
    return {"append": _append, "attend": _attend, "adapt": _adapt}[state["case"]["kind"]](state)


def work(case):
    c = case
    if c["kind"] == "adapt":
        ids = _row_adapters(c)
        used, rows = len(set(ids[ids >= 0].tolist())), int((ids >= 0).sum())
        return {"bytes": 2 * used * c["rank"] * (c["K"] + c["N"]) + 2 * rows * c["K"] + 4 * c["M"] * c["N"], "flops": 2 * rows * c["rank"] * (c["K"] + c["N"])}
    S, n = _lengths(c)
    T, h_q, h_kv, d = sum(S), c["h_q"], c["h_kv"], c["d"]
    held = 2 * h_kv * (d // 2 + 4 * d // GROUP)  # bytes of a position in the cache, keys and values
    if c["kind"] == "append":
        return {"bytes": T * (2 * (2 * h_q + 2 * h_kv) * d + held + 4 * h_kv * d + 4 * c["rot"]), "flops": T * (h_q + h_kv) * c["rot"] * 3}
    seen = sum(s * (m - s) + s * (s + 1) // 2 for s, m in zip(S, n))
    return {"bytes": sum(n) * held + 4 * T * h_q * d, "flops": 4 * seen * h_q * d}


# ---------------------------------------------------------------- the definitions in 64 bits
def _exact_values(rows):
    """What the cache holds for binary16 rows: every rounding that the format names, in its place."""
    g = rows.double().reshape(*rows.shape[:-1], -1, GROUP)
    lo, hi = g.min(-1, keepdim=True).values, g.max(-1, keepdim=True).values
    step = ((hi - lo).float().double() / 15.0).float().half().double()
    offset = (lo + step * 8.0).float().half().double()
    inv = torch.where(step > 0.0, (1.0 / step.clamp(min=2.0 ** -24)).float().double(), torch.zeros_like(step))
    code = torch.round(((g - offset).float().double() * inv).float().double()).clamp(-8.0, 7.0)
    return (offset + step * code).reshape(rows.shape)


def _exact_append(c, s):
    S, n = _lengths(c)
    h_q, h_kv, d, half, f = c["h_q"], c["h_kv"], c["d"], c["rot"] // 2, _frequencies(c)
    x = s["qkv"].cpu().numpy().reshape(-1, h_q + 2 * h_kv, d)
    pos = np.concatenate([np.arange(m - t, m) for t, m in zip(S, n)]).astype(np.float64)
    i = np.arange(half, dtype=np.float64)
    freq = f["base"] ** (-i / half)
    if f["original_positions"]:
        turns = f["original_positions"] * freq / (2.0 * np.pi)
        share = np.clip((turns - f["low_turns"]) / (f["high_turns"] - f["low_turns"]), 0.0, 1.0)
        freq = (1.0 - share) * freq / f["factor"] + share * freq
    angle = pos[:, None] * freq
    cos, sin = (t.astype(np.float32).astype(np.float64)[:, None] for t in (np.cos(angle), np.sin(angle)))  # the table holds 32 bits
    qk = x[:, :h_q + h_kv].copy()
    i0, i1 = (np.arange(half), np.arange(half) + half) if c["pairs"] == "half" else (2 * np.arange(half), 2 * np.arange(half) + 1)
    x0, x1 = x[:, :h_q + h_kv][..., i0].astype(np.float64), x[:, :h_q + h_kv][..., i1].astype(np.float64)
    qk[..., i0] = (x0 * cos - x1 * sin).astype(np.float16)
    qk[..., i1] = (x1 * cos + x0 * sin).astype(np.float16)
    q = torch.from_numpy(qk[:, :h_q].reshape(-1, h_q * d).astype(np.float64))
    return {"q": q, "k": _exact_values(torch.from_numpy(qk[:, h_q:])), "v": _exact_values(torch.from_numpy(x[:, h_q + h_kv:].copy()))}


def _exact_attend(c, s):
    S, n = _lengths(c)
    h_q, h_kv, d, g = c["h_q"], c["h_kv"], c["d"], c["h_q"] // c["h_kv"]
    out, at, row = torch.empty((sum(S), h_q, d), dtype=torch.float64), 0, 0
    for t, m in zip(S, n):
        K, V = (_exact_values(s[x][at:at + m]) for x in ("k", "v"))
        unseen = torch.arange(m, device="cuda")[None, :] > torch.arange(m - t, m, device="cuda")[:, None]
        for h in range(h_q):
            q = s["q"][row:row + t, h * d:(h + 1) * d].double()
            score = (q @ K[:, h // g].T.contiguous()) * d ** -0.5
            weight = torch.softmax(score.masked_fill(unseen, float("-inf")), -1)
            out[row:row + t, h] = (weight @ V[:, h // g].contiguous()).cpu()
        at, row = at + m, row + t
    return {"out": out.reshape(sum(S), h_q * d)}


def _exact_adapt(c, s):
    out = s["y"].double()
    for a in range(c["count"]):
        rows = (s["ids"] == a).nonzero().flatten()
        out[rows] += float(s["scale"][a]) * ((s["x"][rows].double() @ s["a"][a].double().T.contiguous()) @ s["b"][a].double().T.contiguous())
    return {"out": out}


def exact(case, seed):
    return {"append": _exact_append, "attend": _exact_attend, "adapt": _exact_adapt}[case["kind"]](case, _inputs(case, seed))
