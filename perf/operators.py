"""The operators of the cloud's verification step, as their speed and their outputs are measured.

The step that the drafted windows of image tokens go through: the cache's pages and slots are planned on the GPU from the
accepted lengths (``plan``), queries and keys are turned by their positions and the new keys and values laid into the
pages (``rotary``), every new token attends to what its request has in the cache (``attention``), and the verifier's
logits pass their penalties, biases and grammar masks before the accept test (``logits``).

Layout of the cache, an atom of 16 tokens of one head at a time, each atom contiguous:
  keys   [pages, kv_heads, page_size / 16, head_dim / 8, 16, 8]   token t of the atom, dimension d: [d / 8, t, d % 8]
  values [pages, kv_heads, page_size / 16, 2, head_dim, 8]        token t of the atom, dimension d: [t / 8, d, t % 8]
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DTYPE = {"float32": torch.float32, "bfloat16": torch.bfloat16}
_BASE = 10000.0


# ---- the cases ----------------------------------------------------------------------------------------------------

def listed() -> list[dict]:
    return [
        # Eight requests, each about to verify a window of eight drafted tokens: what a tight decoding loop plans.
        {"name": "plan_window", **_plan(requests=8, new=8, context=600, page=16, ragged=False)},
        # A large fleet: some requests draft, some have just been filled, some roll pages back, none or a few hundred tokens each.
        {"name": "plan_fleet", **_plan(requests=1000, new=64, context=8192, page=16, ragged=True)},
        # One token for each of sixteen requests, far into a long context, keys and values laid into the cache.
        {"name": "rotary_step", **_rotary(tokens=16, q_heads=32, kv_heads=8, dim=128, rotary=128, far=120000)},
        # A prompt of many tokens: pairs interleaved, half of the head turned, frequencies scaled for a long context.
        {"name": "rotary_prompt", **_rotary(tokens=8192, q_heads=32, kv_heads=8, dim=128, rotary=64, far=30000,
                                            layout="interleaved", scaled=True, page=32)},
        # The gradient of the rotation for a training batch in 32 bits: ragged tokens, a head of 80.
        {"name": "rotary_gradient", **_rotary(tokens=4099, q_heads=16, kv_heads=4, dim=80, rotary=80, far=4099,
                                              dtype="float32", inverse=True)},
        # The first window of one small request, one key head for each query head: all latency.
        {"name": "attention_first", **_attention(requests=1, new=8, context=40, q_heads=8, kv_heads=8, dim=64)},
        # Single tokens of 64 requests with ragged contexts: reading the cache is the work.
        {"name": "attention_token", **_attention(requests=64, new=1, context=4096, q_heads=32, kv_heads=8, dim=128)},
        # Windows of eight drafted tokens of 32 requests, eight query heads to a key head: the verification itself.
        {"name": "attention_window", **_attention(requests=32, new=8, context=4100, q_heads=32, kv_heads=4, dim=128, page=32)},
        # One token at the end of a very long context: few rows, a long axis.
        {"name": "attention_long", **_attention(requests=1, new=1, context=200001, q_heads=16, kv_heads=2, dim=128, page=64)},
        # Chunks of prompts, ragged, with what earlier chunks have left in the cache: the matrix cores' work.
        {"name": "attention_prompt", **_attention(requests=3, new=2048, context=8192, q_heads=32, kv_heads=8, dim=128, page=64)},
        # One window's verifier rows in 32 bits with everything switched on.
        {"name": "logits_window", **_logits(rows=8, vocab=16384, window=8, history=300)},
        # Many windows of a large vocabulary in bf16, long histories, grammar masks shared by the rows of a window.
        {"name": "logits_batch", **_logits(rows=4096, vocab=65536, window=8, history=4000, dtype="bfloat16")},
    ]


def _plan(*, requests, new, context, page, ragged, spread=1):
    return {"op": "plan", "requests": requests, "new": new, "context": context, "page": page, "ragged": ragged, "spread": spread}


def _rotary(*, tokens, q_heads, kv_heads, dim, rotary, far, dtype="bfloat16", layout="half", scaled=False, inverse=False,
            page=16, spread=1):
    return {"op": "rotary", "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "rotary": rotary, "far": far,
            "dtype": dtype, "layout": layout, "scaled": scaled, "inverse": inverse, "page": page, "spread": spread}


def _attention(*, requests, new, context, q_heads, kv_heads, dim, page=16, spread=1):
    return {"op": "attention", "requests": requests, "new": new, "context": context, "q_heads": q_heads, "kv_heads": kv_heads,
            "dim": dim, "page": page, "spread": spread}


def _logits(*, rows, vocab, window, history, dtype="float32", penalties=True, biases=True, masks=True, spread=1):
    return {"op": "logits", "rows": rows, "vocab": vocab, "window": window, "history": history, "dtype": dtype,
            "penalties": penalties, "biases": biases, "masks": masks, "spread": spread}


def draw(rng) -> dict:
    """One more case of the same ranges: every operator, odd sizes, ragged lengths."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["plan", "rotary", "attention", "attention", "logits"])
    mark = rng.randrange(1 << 30)                              # which lengths a ragged case gets
    if op == "plan":
        return _plan(requests=spread(1, 1000), new=spread(1, 64), context=spread(16, 8192), page=rng.choice([16, 32, 64]),
                     ragged=rng.random() < 0.7, spread=mark)
    kv_heads = rng.choice([1, 2, 4, 5, 8])
    q_heads = kv_heads * rng.choice([1, 2, 3, 4, 7, 8] if kv_heads < 5 else [1, 3, 4])
    if op == "rotary":
        inverse = rng.random() < 0.3
        dim = 32 * rng.randint(1, 6) if not inverse else 2 * rng.randint(16, 96)
        part = rng.random() < 0.4
        return _rotary(tokens=spread(1, 4096), q_heads=q_heads, kv_heads=kv_heads, dim=dim,
                       rotary=2 * rng.randint(4, dim // 2) if part else dim, far=spread(100, 200000),
                       dtype=rng.choice(["float32", "bfloat16"]) if inverse else "bfloat16",
                       layout=rng.choice(["half", "interleaved"]), scaled=rng.random() < 0.4, inverse=inverse,
                       page=rng.choice([16, 32, 64]), spread=mark)
    if op == "attention":
        dim = rng.choice([64, 64, 96, 128, 128, 128, 192, 256])
        new = rng.choice([1, 1, spread(2, 32), spread(32, 1024)])
        context = new + spread(1, 16384)
        # as many requests as keep the queries' work and the cache under the largest listed case's
        if new * q_heads * context * dim > 48 * 10 ** 9:
            q_heads = kv_heads
        most = min(48 * 10 ** 9 / (new * q_heads * context * dim), 2 ** 27 / (context * kv_heads * dim))
        return _attention(requests=spread(1, max(1, min(128, int(most)))), new=new, context=context, q_heads=q_heads,
                          kv_heads=kv_heads, dim=dim, page=rng.choice([16, 32, 64]), spread=mark)
    dtype = rng.choice(["float32", "bfloat16"])
    vocab = spread(1024, 32768 if dtype == "float32" else 65536)
    window = rng.choice([1, 2, 4, 5, 8, 8, 16])
    rows = window * spread(1, max(1, min(2048, (1 << 27) // vocab) // window))
    return _logits(rows=rows, vocab=vocab, window=window, history=spread(1, 4000), dtype=dtype, penalties=rng.random() < 0.8,
                   biases=rng.random() < 0.6, masks=rng.random() < 0.6, spread=mark)


def _lengths(case):
    """The lengths of a case's requests: part of the case, the same for every seed."""
    rng, n = random.Random(str(sorted(case.items()))), case["requests"]
    if case["op"] == "plan":
        if not case["ragged"]:
            return [case["context"]] * n, [case["new"]] * n
        # the last is what a request kept of its previous window; now and then a request has just been emptied
        return ([rng.choice([0, rng.randint(1, case["context"])]) if rng.random() < 0.1 else rng.randint(1, case["context"])
                 for _ in range(n)], [rng.choice([0, 1, rng.randint(0, case["new"]), case["new"]]) for _ in range(n)])
    new = [case["new"] if n == 1 or case["new"] == 1 else rng.randint(max(1, case["new"] // 2), case["new"]) for _ in range(n)]
    if n > 1 and case["new"] > 1:
        new[rng.randrange(n)] = case["new"]
    total = [case["context"] if n == 1 else rng.randint(max(c, case["context"] // 2), max(c, case["context"])) for c in new]
    total[rng.randrange(n)] = case["context"]
    return [max(t, c) for t, c in zip(total, new)], new


# ---- inputs -------------------------------------------------------------------------------------------------------

def _maker(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 29)
    return gen


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _frequencies(case):
    """Radians per position of each pair, and what the turned values are multiplied by."""
    half = case["rotary"] // 2
    f = _BASE ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    if not case["scaled"]:
        return f, 1.0
    # four times the positions of the training length of 8192: pairs that turn less than once in it are slowed by 4,
    # pairs that turn more than 32 times keep their pace, those between are blended
    turns = 8192 * f / (2 * math.pi)
    keep = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)
    return f / 4.0 * (1.0 - keep) + f * keep, 1.1386


def prepare(case, seed) -> dict:
    gen, op = _maker(seed), case["op"]
    return {"op": op, "case": case, **{"plan": _prepare_plan, "rotary": _prepare_rotary, "attention": _prepare_attention,
                                       "logits": _prepare_logits}[op](case, gen)}


def _empty(n, dtype=torch.int32):
    return torch.empty(n, dtype=dtype, device="cuda")


def _prepare_plan(case, gen):
    R, page = case["requests"], case["page"]
    context, new = _lengths(case)
    width = -(-(case["context"] + 2 * case["new"]) // page) + 2                # columns of the block table
    pages = R * width + 64
    length, new = _ints(context), _ints(new)
    kept = torch.minimum(torch.randint(0, case["new"] + 1, (R,), generator=gen, device="cuda", dtype=torch.int32), length)
    length = length - kept                                                     # what was there before the last window
    held = ((length + case["new"] + page - 1) // page).int()                   # the last window was drafted in full
    order = torch.randperm(pages, generator=gen, device="cuda").int()
    table = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
    used = torch.arange(width, device="cuda")[None, :] < held[:, None]
    at = torch.cumsum(held.long(), 0) - held
    table = torch.where(used, order[(at[:, None] + torch.arange(width, device="cuda")).clamp(max=pages - 1)], table)
    # the free pages wait in a ring, first come first served; its counters have been running for a while
    taken = held.sum().long()
    head = torch.randint(0, 1 << 20, (1,), generator=gen, device="cuda")
    j = torch.arange(pages, device="cuda")
    ring = torch.zeros(pages, dtype=torch.int32, device="cuda")
    ring[(head + j) % pages] = torch.where(j < pages - taken, order[(taken + j).clamp(max=pages - 1)], -1)
    tokens = R * case["new"]
    return {"lengths": length, "kept": kept, "new": new, "held": held, "table": table, "ring": ring,
            "ring_state": torch.cat([head, head + pages - taken]), "tokens": tokens,
            "out": {"lengths": _empty(R), "kv_len": _empty(R), "cu_new": _empty(R + 1), "held": _empty(R),
                    "granted": _empty(R, torch.uint8), "ring_state": _empty(2, torch.int64), "slots": _empty(tokens),
                    "positions": _empty(tokens), "requests": _empty(tokens)}}


def _cache(pages, case, gen):
    """A cache as it is after long use: every slot holds something."""
    H, D, atoms = case["kv_heads"], case["dim"], case["page"] // 16
    k = torch.empty((pages, H, atoms, D // 8, 16, 8), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    v = torch.empty((pages, H, atoms, 2, D, 8), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    return k, v


def _prepare_rotary(case, gen):
    T, Hq, Hk, D, dtype = case["tokens"], case["q_heads"], case["kv_heads"], case["dim"], _DTYPE[case["dtype"]]
    # queries, keys and values as one projection leaves them: side by side
    qkv = torch.randn((T, Hq + 2 * Hk, D), generator=gen, device="cuda").to(dtype)
    s = {"q": qkv[:, :Hq], "k": qkv[:, Hq:Hq + Hk], "v": qkv[:, Hq + Hk:]}
    if T < 64:                                                                 # single tokens of as many requests
        s["positions"] = torch.randint(0, case["far"], (T,), generator=gen, device="cuda", dtype=torch.int32)
    else:                                                                      # a chunk that ends at a far position
        s["positions"] = torch.arange(T, device="cuda", dtype=torch.int32) + max(0, case["far"] - T)
    s["inv_freq"], s["magnitude"] = _frequencies(case)
    s["out"] = {"q": torch.empty((T, Hq, D), dtype=dtype, device="cuda")}
    if case["inverse"]:
        s["out"]["k"] = torch.empty((T, Hk, D), dtype=dtype, device="cuda")
        return s
    page = case["page"]
    pages = -(-T // page) + 4 if T >= 64 else T + 4
    s["k_cache"], s["v_cache"] = _cache(pages, case, gen)
    own_page = torch.randperm(pages, generator=gen, device="cuda")
    i = torch.arange(T, device="cuda")
    if T < 64:
        s["slots"] = (own_page[:T] * page + torch.randint(0, page, (T,), generator=gen, device="cuda")).int()
    else:
        i = i + min(5, page * pages - T)                                       # the chunk starts inside a page
        s["slots"] = (own_page[i // page] * page + i % page).int()
    return s


def _prepare_attention(case, gen):
    total, new = _lengths(case)
    R, D, page = case["requests"], case["dim"], case["page"]
    need = [-(-t // page) for t in total]
    width, pages = max(need) + 1, sum(need) + 3
    k, v = _cache(pages, case, gen)
    order = torch.randperm(pages, generator=gen, device="cuda").int()
    begin = _ints([sum(need[:r]) for r in range(R)], torch.int64)
    col = torch.arange(width, device="cuda")
    used = col[None, :] < _ints(need)[:, None]
    table = torch.where(used, order[(begin[:, None] + col).clamp(max=pages - 1)], -1)
    cu = [0]
    for c in new:
        cu.append(cu[-1] + c)
    # a row's scores spread as in use: some heads look at few tokens, some at many
    sharp = 0.5 + 2.0 * torch.rand((1, case["q_heads"], 1), generator=gen, device="cuda")
    q = (torch.randn((cu[-1], case["q_heads"], D), generator=gen, device="cuda") * sharp).bfloat16()
    return {"q": q, "k_cache": k, "v_cache": v, "table": table, "cu_new": _ints(cu), "kv_len": _ints(total),
            "max_new": max(new), "max_len": max(total), "scale": 1.0 / math.sqrt(D),
            "out": {"out": torch.empty_like(q), "lse": _empty((cu[-1], case["q_heads"]), torch.float32)}}


def _prepare_logits(case, gen):
    N, V, K, dtype = case["rows"], case["vocab"], case["window"], _DTYPE[case["dtype"]]
    R, rng = -(-N // K), random.Random(str(sorted(case.items())))
    per = 4 if case["dtype"] == "float32" else 8
    stride = -(-V // per) * per
    x = torch.empty((N, stride), dtype=dtype, device="cuda")
    x.normal_(0.0, 2.5, generator=gen)
    s = {"logits": x[:, :V], "out": {"logits": torch.empty((N, stride), dtype=dtype, device="cuda")[:, :V], "left": _empty(N)}}

    def tokens(n):                                                             # a few tokens come again and again
        return (V * torch.rand(n, generator=gen, device="cuda") ** 3).int().clamp(max=V - 1)

    args = {}
    if case["penalties"]:
        lens = [rng.randint(case["history"] // 2, case["history"]) for _ in range(R)]
        args["history_start"] = torch.nn.functional.pad(torch.cumsum(_ints(lens, torch.int64), 0), (1, 0))
        args["history"] = tokens(sum(lens))
        args["prompt_len"] = _ints([n // 3 for n in lens])
        args["drafted"] = tokens(N)
        args["repetition"] = 1.0 + 0.3 * torch.rand(R, generator=gen, device="cuda")
        args["presence"] = torch.rand(R, generator=gen, device="cuda")
        args["frequency"] = 0.5 * torch.rand(R, generator=gen, device="cuda")
    if case["biases"]:
        n = min(40, V // 4)
        lens = [rng.randint(0, n) for _ in range(R)]
        step = V // (n + 1)
        args["bias_start"] = torch.nn.functional.pad(torch.cumsum(_ints(lens, torch.int64), 0), (1, 0))
        first = torch.randint(0, step, (sum(lens),), generator=gen, device="cuda")
        at = torch.arange(sum(lens), device="cuda")
        row = torch.searchsorted(args["bias_start"], at, right=True) - 1       # ascending tokens within a request
        args["bias_ids"] = ((at - args["bias_start"][row]) * step + first).int()
        args["bias_values"] = 4.0 * torch.randn(sum(lens), generator=gen, device="cuda")
    if case["masks"]:
        # one grammar state to a window; what a state allows comes in runs, a few tokens to most of them
        words = -(-V // 32)
        share = torch.rand((R, 1), generator=gen, device="cuda") ** 2
        runs = (torch.rand((R, -(-words // 8)), generator=gen, device="cuda") < share).repeat_interleave(8, 1)[:, :words]
        bits = torch.randint(-(1 << 31), 1 << 31, (R, words), generator=gen, device="cuda").int()
        args["allowed"] = torch.where(runs, bits | 1, 0).int()
        args["allowed"][:, 0] |= 2
        args["allowed_row"] = (torch.arange(N, device="cuda") // K).int()
    return {**s, "args": args}


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(s):
    op, case = s["op"], s["case"]
    if own:
        import paper_2603_25463_amd as ciar
        if op == "plan":
            o = ciar.cache_plan(s["lengths"], s["new"], s["held"], s["ring"], s["ring_state"], s["table"], s["tokens"],
                                page_size=case["page"], kept=s["kept"], out=s["out"])
            return {**o, "table": s["table"], "ring": s["ring"]}
        if op == "rotary":
            if case["inverse"]:
                return ciar.rotary(s["q"], s["k"], s["positions"], s["inv_freq"], layout=case["layout"], inverse=True,
                                   magnitude=s["magnitude"], out=s["out"])
            o = ciar.rotary(s["q"], s["k"], s["positions"], s["inv_freq"], layout=case["layout"], magnitude=s["magnitude"],
                            v=s["v"], k_cache=s["k_cache"], v_cache=s["v_cache"], slots=s["slots"], out=s["out"])
            return {"q": o["q"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
        if op == "attention":
            return ciar.paged_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["cu_new"], s["kv_len"],
                                        s["max_new"], s["max_len"], scale=s["scale"], out=s["out"])
        return ciar.adjust_logits(s["logits"], ciar.Params(window=case["window"]), out=s["out"], **s["args"])
    return {"plan": _plain_plan, "rotary": _plain_rotary, "attention": _plain_attention, "logits": _plain_logits}[op](s)


def _plain_plan(s):
    page, T, table, ring = s["case"]["page"], s["tokens"], s["table"], s["ring"]
    P, width, dev = ring.numel(), table.shape[1], table.device
    head, tail = s["ring_state"][0], s["ring_state"][1]
    length, new, held = s["lengths"].long() + s["kept"].long(), s["new"].long(), s["held"].long()
    end = torch.cumsum(new, 0)
    pages = (length + new + page - 1) // page
    fits = (pages <= width) & (end <= T)
    need = torch.where(fits, (pages - held).clamp(min=0), 0)
    upto = torch.cumsum(need, 0)
    granted = fits & ((need == 0) | (upto <= tail - head))
    need = torch.where(granted, need, 0)
    give = torch.where(granted, (held - pages).clamp(min=0), 0)
    col = torch.arange(width, device=dev)
    # pages come from the ring's head ...
    fresh = (col >= held[:, None]) & (col < (held + need)[:, None])
    from_ring = ring[(head + (upto - need)[:, None] + col - held[:, None]) % P]
    # ... and go back to its tail
    back = (col >= pages[:, None]) & (col < (pages + give)[:, None])
    to = (tail + (torch.cumsum(give, 0) - give)[:, None] + col - pages[:, None]) % P
    ring_new = torch.cat([ring, ring[:1]]).index_put((torch.where(back, to, P).flatten(),), table.flatten())[:P]
    table.copy_(torch.where(fresh, from_ring, table))
    ring.copy_(ring_new)
    i = torch.arange(T, device=dev)
    r = torch.searchsorted(end, i, right=True)
    there = r < new.numel()
    r = r.clamp(max=new.numel() - 1)
    pos = length[r] + i - (end - new)[r]
    slot = table[r, (pos // page).clamp(max=width - 1)] * page + pos % page
    cu = torch.nn.functional.pad(end.clamp(max=T), (1, 0))
    return {"lengths": length.int(), "kv_len": torch.where(granted, length + new, 0).int(), "cu_new": cu.int(),
            "held": torch.where(granted, pages, held).int(), "granted": granted.to(torch.uint8),
            "ring_state": torch.stack([head + need.sum(), tail + give.sum()]),
            "slots": torch.where(there & granted[r], slot, -1).int(), "positions": torch.where(there, pos, 0).int(),
            "requests": torch.where(there, r, -1).int(), "table": table, "ring": ring}


def _turned(x, c, sn, case):
    """x [T, H, D] in 32 bits, its first `rotary` dimensions turned; c, sn [T, 1, rotary / 2]."""
    n = case["rotary"]
    if case["layout"] == "half":
        a, b = x[..., :n // 2], x[..., n // 2:n]
        return torch.cat([a * c - b * sn, b * c + a * sn, x[..., n:]], -1)
    a, b = x[..., 0:n:2], x[..., 1:n:2]
    return torch.cat([torch.stack([a * c - b * sn, b * c + a * sn], -1).flatten(-2), x[..., n:]], -1)


def _plain_rotary(s):
    case = s["case"]
    angle = s["positions"].double()[:, None, None] * s["inv_freq"]
    c, sn = (torch.cos(angle) * s["magnitude"]).float(), (torch.sin(angle) * s["magnitude"]).float()
    if case["inverse"]:
        sn = -sn
    dtype = s["q"].dtype
    q, k = _turned(s["q"].float(), c, sn, case).to(dtype), _turned(s["k"].float(), c, sn, case).to(dtype)
    if case["inverse"]:
        return {"q": q, "k": k}
    T, H, D = k.shape
    slot = s["slots"].long()
    page, at = slot // case["page"], slot % case["page"]
    s["k_cache"][page, :, at // 16, :, at % 16] = k.view(T, H, D // 8, 8)
    s["v_cache"][page, :, at // 16, at % 16 // 8, :, at % 8] = s["v"]
    return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attention(s):
    q, table, case = s["q"], s["table"], s["case"]
    T, Hq, D = q.shape
    H, R, n, page = case["kv_heads"], case["requests"], s["max_new"], case["page"]
    L = -(-s["max_len"] // page) * page
    at = table[:, :L // page].clamp(min=0).long()
    k = s["k_cache"][at].permute(0, 2, 1, 3, 5, 4, 6).reshape(R * H, L, D).float()
    v = s["v_cache"][at].permute(0, 2, 1, 3, 4, 6, 5).reshape(R * H, L, D).float()
    # every request's queries in a block of max_new rows
    begin, new = s["cu_new"][:-1].long(), s["cu_new"][1:].long() - s["cu_new"][:-1].long()
    j = torch.arange(n, device=q.device)
    there = j[None, :] < new[:, None]
    qs = q[(begin[:, None] + j).clamp(max=T - 1)].float().reshape(R, n, H, Hq // H, D).permute(0, 2, 1, 3, 4)
    score = torch.bmm(qs.reshape(R * H, n * (Hq // H), D), k.transpose(1, 2).contiguous()).mul_(s["scale"])
    last = s["kv_len"].long()[:, None] - new[:, None] + j                      # the position of each new token
    seen = torch.arange(L, device=q.device) <= last[:, :, None]
    score = score.view(R, H, n, Hq // H, L)
    score.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp_(score.sub_(top))
    total = p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(R * H, n * (Hq // H), L), v).view(R, H, n, Hq // H, D)
    o = torch.where(total > 0, o / total, 0.0)
    lse = (torch.log(total) + top)[..., 0]
    # back to the tokens' own order
    row = torch.searchsorted(s["cu_new"][1:].long(), torch.arange(T, device=q.device), right=True)
    i = torch.arange(T, device=q.device) - begin[row]
    return {"out": o.permute(0, 2, 1, 3, 4)[row, i].reshape(T, Hq, D).bfloat16(),
            "lse": lse.permute(0, 2, 1, 3)[row, i].reshape(T, Hq)}


def _counts(tokens, request, weight, R, V):
    return torch.zeros(R * V, dtype=torch.float32, device=tokens.device).index_add_(
        0, request * V + tokens.long(), weight).view(R, V)


def _plain_logits(s):
    case, a = s["case"], s["args"]
    N, V, K = case["rows"], case["vocab"], case["window"]
    R, dev = -(-N // K), s["logits"].device
    x, n = s["logits"].float(), torch.arange(N, device=dev)
    if case["penalties"]:
        at = torch.arange(a["history"].numel(), device=dev)
        r = torch.searchsorted(a["history_start"], at, right=True) - 1
        said = (at - a["history_start"][r] >= a["prompt_len"][r]).float()
        out = _counts(a["history"], r, said, R, V)[n // K]
        ever = _counts(a["history"], r, torch.ones_like(said), R, V)[n // K]
        # row n's history ends with the drafted tokens before it in its window
        late = torch.arange(K, device=dev)
        m = (n[:, None] // K * K + late).clamp(max=N - 1)
        add = (late[None, :] < (n % K)[:, None]).float().reshape(-1)
        index = (n[:, None] * V + a["drafted"].long()[m]).reshape(-1)
        out.view(-1).index_add_(0, index, add)
        ever.view(-1).index_add_(0, index, add)
        theta = a["repetition"][n // K][:, None]
        x = torch.where(ever > 0, torch.where(x > 0, x / theta, x * theta), x)
        x = x - a["frequency"][n // K][:, None] * out - a["presence"][n // K][:, None] * (out > 0)
    if case["biases"]:
        at = torch.arange(a["bias_ids"].numel(), device=dev)
        x = x + _counts(a["bias_ids"], torch.searchsorted(a["bias_start"], at, right=True) - 1, a["bias_values"], R, V)[n // K]
    if case["masks"]:
        t = torch.arange(V, device=dev)
        bits = (a["allowed"][:, t // 32] >> (t % 32)) & 1
        x = torch.where(bits[a["allowed_row"].long()] != 0, x, -math.inf)
    return {"logits": x.to(s["logits"].dtype), "left": torch.isfinite(x).sum(1).int()}


# ---- what a pass costs at least, and its results in 64 bits -------------------------------------------------------

def work(case) -> dict:
    op = case["op"]
    if op == "plan":
        R, T = case["requests"], case["requests"] * case["new"]
        context, new = _lengths(case)
        # the requests' numbers, a table entry for each new page and for each that the new tokens start in, three words a token
        return {"bytes": R * (16 + 17) + 24 * 2 + sum(8 + 8 * (n // case["page"]) for n in new) + 12 * T, "flops": 0}
    if op == "rotary":
        T, elt = case["tokens"], 4 if case["dtype"] == "float32" else 2
        heads = case["q_heads"] + case["kv_heads"] + (0 if case["inverse"] else case["kv_heads"])
        return {"bytes": 2 * T * heads * case["dim"] * elt + 8 * T + 4 * case["rotary"],
                "flops": 3 * T * (case["q_heads"] + case["kv_heads"]) * case["rotary"]}
    if op == "attention":
        total, new = _lengths(case)
        pairs = sum(c * (t - c) + c * (c + 1) // 2 for t, c in zip(total, new))
        return {"bytes": 4 * sum(total) * case["kv_heads"] * case["dim"] + sum(new) * case["q_heads"] * (4 * case["dim"] + 4)
                + 4 * sum(-(-t // case["page"]) for t in total), "flops": 4 * pairs * case["q_heads"] * case["dim"]}
    N, V, R = case["rows"], case["vocab"], -(-case["rows"] // case["window"])
    b = 2 * N * V * (4 if case["dtype"] == "float32" else 2) + 4 * N
    b += case["penalties"] * (R * (3 * case["history"] + 24) + 4 * N) + case["biases"] * R * 160 + case["masks"] * (R * (V // 8) + 4 * N)
    return {"bytes": b, "flops": 0}


def exact(case, seed):
    if case["op"] == "plan":
        return None                                                            # whole numbers
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "attention": _exact_attention, "logits": _exact_logits}[case["op"]](s)


def _exact_rotary(s):
    case = s["case"]
    n = case["rotary"]
    pair = torch.arange(n // 2, device="cuda")
    one, two = (pair, pair + n // 2) if case["layout"] == "half" else (2 * pair, 2 * pair + 1)
    angle = s["positions"].double()[:, None] * s["inv_freq"][None, :] * (-1.0 if case["inverse"] else 1.0)
    turn = torch.polar(torch.full_like(angle, s["magnitude"]), angle)[:, None, :]
    turned = {}
    for name in ("q", "k"):
        y = s[name].double().clone()
        z = torch.complex(y[..., one], y[..., two]) * turn
        y[..., one], y[..., two] = z.real, z.imag
        turned[name] = y
    if case["inverse"]:
        return turned
    # the caches with tokens in rows, the rows of the slots replaced
    P, H, A, D = s["k_cache"].shape[0], case["kv_heads"], case["page"] // 16, case["dim"]
    k = s["k_cache"].double().permute(0, 2, 4, 1, 3, 5).reshape(P * A * 16, H, D)
    v = s["v_cache"].double().permute(0, 2, 3, 5, 1, 4).reshape(P * A * 16, H, D)
    k[s["slots"].long()], v[s["slots"].long()] = turned["k"], s["v"].double()
    return {"q": turned["q"], "k_cache": k.view(P, A, 16, H, D // 8, 8).permute(0, 3, 1, 4, 2, 5).contiguous(),
            "v_cache": v.view(P, A, 2, 8, H, D).permute(0, 4, 1, 2, 5, 3).contiguous()}


def _exact_attention(s):
    case, q = s["case"], s["q"]
    total, new = _lengths(case)
    H, D, page, g = case["kv_heads"], case["dim"], case["page"], case["q_heads"] // case["kv_heads"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    begin = 0
    for r, (length, c) in enumerate(zip(total, new)):
        pages = s["table"][r, :-(-length // page)].long()
        for h in range(H):
            k = s["k_cache"][pages, h].transpose(2, 3).reshape(-1, D)[:length].double()
            v = s["v_cache"][pages, h].transpose(3, 4).reshape(-1, D)[:length].double()
            for lo in range(0, c, 512):
                m = min(512, c - lo)
                rows = slice(begin + lo, begin + lo + m)
                x = (q[rows, h * g:(h + 1) * g].double().reshape(m * g, D) @ k.T) * s["scale"]
                late = torch.arange(length, device="cuda") > (length - c + lo + torch.arange(m, device="cuda"))[:, None]
                x = x.view(m, g, length).masked_fill_(late[:, None, :], -math.inf)
                lse[rows, h * g:(h + 1) * g] = torch.logsumexp(x, -1)
                out[rows, h * g:(h + 1) * g] = (torch.softmax(x, -1).view(m * g, length) @ v).view(m, g, D)
        begin += c
    return {"out": out, "lse": lse}


def _exact_logits(s):
    case, a, N, V, K = s["case"], s["args"], s["case"]["rows"], s["case"]["vocab"], s["case"]["window"]
    x = s["logits"].double()
    history = a["history"].cpu() if case["penalties"] else None
    start = a["history_start"].tolist() if case["penalties"] else None
    bias = a["bias_start"].tolist() if case["biases"] else None
    for n in range(N):
        r, y = n // K, x[n]
        if case["penalties"]:
            said = torch.cat([history[start[r] + int(a["prompt_len"][r]):start[r + 1]], a["drafted"][r * K:n].cpu()]).long()
            out = torch.bincount(said, minlength=V).cuda()
            seen = torch.cat([history[start[r]:start[r + 1]].long(), said]).unique().cuda()
            theta = a["repetition"][r].double()
            y[seen] = torch.where(y[seen] > 0, y[seen] / theta, y[seen] * theta)
            y -= a["frequency"][r].double() * out + a["presence"][r].double() * (out > 0)
        if case["biases"]:
            y[a["bias_ids"][bias[r]:bias[r + 1]].long()] += a["bias_values"][bias[r]:bias[r + 1]].double()
        if case["masks"]:
            t = torch.arange(V, device="cuda")
            y[((a["allowed"][a["allowed_row"][n].long()][t // 32] >> (t % 32)) & 1) == 0] = -math.inf
    return {"logits": x, "left": None}
