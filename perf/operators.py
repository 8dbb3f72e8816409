"""Measured cases of the KV-page operators: the 4-bit page store (write and read back), attention over a whole
prompt, attention over the 4-bit page cache, and eviction of pages by accumulated attention weight.

Lengths of the requests of a case follow from the case alone; values, page numbers and weights from the seed."""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
NO_SLOT = -1  # 0xFFFFFFFF as int32


def listed():
    return [
        # one decode step's append: one token for each of 64 running requests, 16-token pages
        dict(name="store 64x1 c16", op="store", requests=64, new=1, start=2048, kv_heads=8, head_dim=128, page_tokens=16,
             dtype="bf16", k_scale=1.0, v_scale=1.0),
        # the missed tail of a ragged batch, odd page size, 64-wide heads, calibrated scales
        dict(name="store 24x777 c48 d64", op="store", requests=24, new=777, start=500, kv_heads=4, head_dim=64, page_tokens=48,
             dtype="fp16", k_scale=0.0173, v_scale=0.00391),
        # prompts of the paged-cache workload, written whole and read back by another worker
        dict(name="store 64x2048 c256", op="store", requests=64, new=2048, start=0, kv_heads=8, head_dim=128, page_tokens=256,
             dtype="bf16", k_scale=1.0, v_scale=0.25),
        # a lone short request: latency
        dict(name="cache 1x300 c16", op="cache", requests=1, len=300, queries=1, kv_heads=8, group=4, head_dim=128,
             page_tokens=16, dtype="bf16", weigh=True),
        # a speculative step: four tokens a request, 64-wide heads
        dict(name="cache 32x4000 q4 d64", op="cache", requests=32, len=4000, queries=4, kv_heads=4, group=3, head_dim=64,
             page_tokens=48, dtype="fp16", weigh=False),
        # a decode step of an ordinary batch, small pages, weights accumulated for eviction
        dict(name="cache 128x2048 c16", op="cache", requests=128, len=2048, queries=1, kv_heads=8, group=4, head_dim=128,
             page_tokens=16, dtype="bf16", weigh=True),
        # long contexts, 256-token pages
        dict(name="cache 16x131072 c256", op="cache", requests=16, len=131072, queries=1, kv_heads=8, group=8, head_dim=128,
             page_tokens=256, dtype="bf16", weigh=True),
        # the tiny workload's batch: eight prompts of up to 512 tokens
        dict(name="prompt 8x512", op="prompt", requests=8, len=512, prefix=0, kv_heads=8, group=4, head_dim=128, dtype="bf16"),
        # ragged tails behind cached prefixes (a hit skips the prefix's prefill), 64-wide heads, odd group
        dict(name="prompt 12x1500+2048 d64", op="prompt", requests=12, len=1500, prefix=2048, kv_heads=4, group=3, head_dim=64,
             dtype="fp16"),
        # two long prompts
        dict(name="prompt 2x8192", op="prompt", requests=2, len=8192, prefix=0, kv_heads=8, group=4, head_dim=128, dtype="bf16"),
        # a running batch cut to half its pages
        dict(name="evict 64x128", op="evict", requests=64, pages=128, page_tokens=16, budget=64, sinks=1, recent=4),
        # long contexts in 16-token pages cut to an eighth
        dict(name="evict 512x8192", op="evict", requests=512, pages=8192, page_tokens=16, budget=1024, sinks=4, recent=32),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("store", "cache", "cache", "prompt", "prompt", "evict"))
    head = dict(kv_heads=rng.choice((1, 2, 4, 8)), head_dim=rng.choice((64, 128)), dtype=rng.choice(("bf16", "fp16")))
    if op == "store":
        new = log(1, 4096)
        return dict(op=op, requests=log(1, max(1, 131072 // new)) if new > 128 else log(1, 1024), new=new, start=rng.randrange(3000),
                    page_tokens=rng.choice((16, 32, 48, 64, 256)), k_scale=rng.choice((1.0, 0.0273)),
                    v_scale=rng.choice((1.0, 0.00719)), **head)
    if op == "cache":
        n = log(1, 131072)
        return dict(op=op, requests=log(1, min(256, max(1, 1500000 // n))), len=n, queries=rng.choice((1, 1, 1, 2, 5)),
                    group=rng.choice((1, 2, 4, 5, 8, 16)), page_tokens=rng.choice((16, 32, 48, 128, 256)),
                    weigh=rng.choice((True, False)), **head)
    if op == "prompt":
        n = log(1, 8192)
        head["kv_heads"] = rng.choice((1, 2, 4))
        prefix = rng.choice((0, 0, log(1, 2048)))
        return dict(op=op, requests=log(1, min(64, max(1, (4 << 20) // (n * (n + prefix))))), len=n, prefix=prefix,
                    group=rng.choice((1, 2, 3, 4, 7, 8)), **head)
    pages = log(1, 8192)
    budget = rng.randint(1, pages + pages // 4)
    recent = rng.randint(1, max(1, budget // 4))
    return dict(op=op, requests=log(1, min(4096, max(1, 4000000 // pages))), pages=pages, page_tokens=rng.choice((16, 48, 256)),
                budget=budget, sinks=rng.randint(0, min(4, budget - recent)), recent=recent)


def lengths(case, most, what):
    """A length for each request in [most/2, most], the first `most` itself."""
    r = random.Random("%s %d %d" % (what, most, case["requests"]))
    return [most] + [r.randint((most + 1) // 2, most) for _ in range(case["requests"] - 1)]


def offsets(lens):
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    return off


# ---- the 4-bit format ------------------------------------------------------------------------------------------------------
# A page holds page_tokens tokens: [kv head][granule of 16 tokens][K codes | V codes | K scales | V scales], a granule's parts
# row-major by token. Codes are e2m1, two to a byte (even dimension low), scales e4m3, one for 16 dimensions.
def quantise(x, g):
    """codes (0..15) and e4m3 scales of float32 x [..., D]; value = E2M1[code] * scale * g."""
    b = x.unflatten(-1, (-1, 16))
    a = b.abs().amax(-1)
    s = (a * torch.full_like(a, 1.0 / 6.0)) / torch.full_like(a, g)
    s = s.clamp(max=448.0).to(torch.float8_e4m3fn)
    den = (s.float() * g).unsqueeze(-1)
    y = torch.where(den > 0, b.abs() / den, torch.zeros_like(b))
    # nearest even: a tie goes to the code with the low bit clear
    mag = (y > 0.25).to(torch.uint8)
    for k, t in enumerate((0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        mag += (y >= t) if k % 2 == 0 else (y > t)
    code = mag | (torch.signbit(b).to(torch.uint8) << 3)
    return code.flatten(-2), s


def value(code, s, g):
    m = code & 7  # halves: 0 1 | 2 3 4 6 8 12
    halves = torch.where(m < 2, m, (2 + (m & 1)) << ((m >> 1).clamp(min=1) - 1)).float()
    x = torch.where(code > 7, -0.5 * halves, 0.5 * halves)
    return (x.unflatten(-1, (-1, 16)) * (s.float() * g).unsqueeze(-1)).flatten(-2)


def pack(k, v, gk, gv):
    """float32 k, v [slots, page_tokens, heads, D] -> uint8 [slots, page bytes]."""
    parts = []
    for x, g in ((k, gk), (v, gv)):
        code, s = quantise(x.permute(0, 2, 1, 3).unflatten(2, (-1, 16)), g)
        parts.append(((code[..., 0::2] | (code[..., 1::2] << 4)).flatten(-2), s.view(torch.uint8).flatten(-2)))
    return torch.cat((parts[0][0], parts[1][0], parts[0][1], parts[1][1]), -1).flatten(1)


def unpack(pages, case, g):
    """uint8 [..., page bytes] -> float32 k, v [..., heads, page_tokens, D]."""
    h, c, d = case["kv_heads"], case["page_tokens"], case["head_dim"]
    x = pages.unflatten(-1, (h, c // 16, 16 * (d + d // 8)))
    out = []
    for j in (0, 1):
        codes = x[..., 8 * d * j: 8 * d * (j + 1)].unflatten(-1, (16, d // 2))
        s = x[..., 16 * d + d * j: 16 * d + d * (j + 1)].unflatten(-1, (16, d // 16)).contiguous().view(torch.float8_e4m3fn)
        code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
        out.append(value(code, s, g[j]).flatten(-3, -2))
    return out


# ---- inputs ----------------------------------------------------------------------------------------------------------------
def randn(shape, gen, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def keys_like(shape, gen, dtype):
    """Keys as models make them: a few channels much larger than the others, a common offset."""
    d = shape[-1]
    amp = torch.ones(d, device="cuda")
    amp[torch.randperm(d, generator=gen, device="cuda")[: max(1, d // 32)]] = 3.0
    return (torch.randn(shape, generator=gen, device="cuda") * amp + 0.3 * amp).to(dtype)


def page_table(lens, stride, gen, slots):
    """int32 [requests, stride] of distinct random slots."""
    p = torch.randperm(slots, generator=gen, device="cuda")[: len(lens) * stride]
    return p.to(torch.int32).view(len(lens), stride).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, r = case["op"], case["requests"]
    s = {"case": case}
    i64 = dict(dtype=torch.int64, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    if op in ("store", "cache"):
        c, h, d, dt = case["page_tokens"], case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]]
        page_bytes = h * c * (d + d // 8)
    if op == "store":
        new = lengths(case, case["new"], "new")
        start = [0] + [random.Random("start %d" % j).randint(0, case["start"]) for j in range(r - 1)]
        stride = -(-max(a + b for a, b in zip(start, new)) // c)
        s["tok_off"], s["start"] = torch.tensor(offsets(new), **i64), torch.tensor(start, **i32)
        s["k"] = keys_like((sum(new), h, d), gen, dt)
        s["v"] = randn((sum(new), h, d), gen, dt)
        if case["k_scale"] != 1.0 or case["v_scale"] != 1.0:
            s["v"] = s["v"] * 0.1
        slots = r * stride + 3
        s["pages"] = page_table(new, stride, gen, slots)
        s["pool"] = torch.zeros((slots, page_bytes), dtype=torch.uint8, device="cuda")
    elif op == "cache":
        lens = lengths(case, case["len"], "len")
        stride = -(-max(lens) // c)
        s["kv_len"] = torch.tensor(lens, **i32)
        slots = r * stride + 3
        s["pages"] = page_table(lens, stride, gen, slots)
        pool, step = [], max(1, (1 << 25) // (c * h * d))
        for a in range(0, slots, step):
            n = min(step, slots - a)
            pool.append(pack(keys_like((n, c, h, d), gen, torch.float32), randn((n, c, h, d), gen, torch.float32), 1.0, 1.0))
        s["pool"] = torch.cat(pool)
        s["q"] = randn((r, case["queries"], h * case["group"], d), gen, dt)
        s["scale"] = d ** -0.5
        s["weight"] = torch.rand((r, stride), generator=gen, device="cuda") * 4 if case["weigh"] else None
    elif op == "prompt":
        h, d, dt = case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]]
        ql = lengths(case, case["len"], "len")
        kl = [a + b for a, b in zip(ql, lengths(case, case["prefix"], "prefix"))]
        s["q_off"], s["k_off"] = torch.tensor(offsets(ql), **i64), torch.tensor(offsets(kl), **i64)
        s["most"] = (max(ql), max(kl))
        s["q"] = randn((sum(ql), h * case["group"], d), gen, dt)
        s["k"] = keys_like((sum(kl), h, d), gen, dt)
        s["v"] = randn((sum(kl), h, d), gen, dt)
        s["scale"] = d ** -0.5
    else:
        n, c = lengths(case, case["pages"], "pages"), case["page_tokens"]
        s["kv_len"] = torch.tensor([a * c - random.Random("tail %d" % j).randrange(c) for j, a in enumerate(n)], **i32)
        s["pages"] = page_table(n, case["pages"], gen, r * case["pages"] + 3)
        # accumulated weights are spread over orders of magnitude; a few pages never had any
        w = torch.exp(3 * torch.randn((r, case["pages"]), generator=gen, device="cuda"))
        s["weight"] = torch.where(torch.rand((r, case["pages"]), generator=gen, device="cuda") < 0.02, torch.zeros_like(w), w)
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------------
def softmax_parts(s, mask):
    """exp(s - max), its sum and the log of sum of exponents, over the last axis; rows without a key sum to 0."""
    s = s.masked_fill(~mask, -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = torch.exp(s - m)
    total = p.sum(-1, keepdim=True)
    return p, total, (m + torch.log(total)).squeeze(-1)


def plain_store(s):
    case, dt, out = s["case"], s["k"].dtype, []
    for x, g in ((s["k"], case["k_scale"]), (s["v"], case["v_scale"])):
        code, scale = quantise(x.float(), g)
        out.append(value(code, scale, g).to(dt))
    return out


def plain_cache(s):
    case, q = s["case"], s["q"].float()
    r, n, h, c = case["requests"], case["queries"], case["kv_heads"], case["page_tokens"]
    k, v = unpack(s["pool"][s["pages"].long()], case, (1.0, 1.0))        # [r, stride, h, c, d]
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in (k, v))             # [r, h, tokens, d]
    q = q.unflatten(2, (h, case["group"])).permute(0, 2, 3, 1, 4)        # [r, h, group, n, d]
    pos = torch.arange(k.shape[2], device=q.device)
    last = s["kv_len"].long().view(-1, 1) - n + torch.arange(n, device=q.device)         # [r, n]
    mask = (pos <= last.unsqueeze(-1)).view(r, 1, 1, n, -1)
    p, total, lse = softmax_parts((q.flatten(2, 3) @ k.transpose(2, 3)).unflatten(2, (-1, n)) * s["scale"], mask)
    inv = torch.where(total > 0, 1 / total, torch.zeros_like(total))
    o = (p.flatten(2, 3) @ v).unflatten(2, (-1, n)) * inv
    o = o.permute(0, 3, 1, 2, 4).flatten(2, 3).to(s["q"].dtype)
    lse = lse.permute(0, 3, 1, 2).flatten(2, 3).contiguous()
    if s["weight"] is None:
        return {"out": o, "lse": lse}
    s["weight"] += (p * inv).sum((1, 2, 3)).unflatten(-1, (-1, c)).sum(-1)
    return {"out": o, "lse": lse, "weight": s["weight"]}


def plain_prompt(s):
    case, (lq, lk), h = s["case"], s["most"], s["case"]["kv_heads"]
    q_off, k_off = s["q_off"], s["k_off"]
    dev = q_off.device
    iq, ik = torch.arange(lq, device=dev), torch.arange(lk, device=dev)
    q = s["q"][(q_off[:-1, None] + iq).clamp(max=s["q"].shape[0] - 1)].float()
    k, v = (s[x][(k_off[:-1, None] + ik).clamp(max=s[x].shape[0] - 1)].float().transpose(1, 2) for x in ("k", "v"))
    q = q.unflatten(2, (h, case["group"])).permute(0, 2, 3, 1, 4)
    ql, kl = (x[1:] - x[:-1] for x in (q_off, k_off))
    mask = ik <= (iq + (kl - ql)[:, None])[:, None, None, :, None]
    sc = (q.flatten(2, 3) @ k.transpose(2, 3)).unflatten(2, (-1, lq)) * s["scale"]
    p, total, lse = softmax_parts(sc, mask)
    del sc
    o = (p.flatten(2, 3) @ v).unflatten(2, (-1, lq)) / total
    t = torch.arange(s["q"].shape[0], device=dev)
    r = torch.searchsorted(q_off[1:], t, right=True)
    i = t - q_off[r]
    o = o.permute(0, 3, 1, 2, 4).flatten(2, 3)[r, i].to(s["q"].dtype)
    return {"out": o, "lse": lse.permute(0, 3, 1, 2).flatten(2, 3)[r, i]}


def plain_evict(s):
    case, c = s["case"], s["case"]["page_tokens"]
    pages, w, budget = s["pages"], s["weight"], s["case"]["budget"]
    r, stride = pages.shape
    j = torch.arange(stride, device=pages.device)
    n = ((s["kv_len"] + c - 1) // c).long()[:, None]
    safe = (j < case["sinks"]) | (j >= n - case["recent"])
    rank_by = torch.where(safe, torch.full_like(w, math.inf), w).masked_fill(j >= n, -math.inf)
    order = torch.argsort(rank_by, dim=1, descending=True, stable=True)
    rank = torch.empty_like(order).scatter_(1, order, j.expand(r, stride).contiguous())
    valid = j < n
    keep = valid & ((rank < budget) | (n <= budget))
    gone = valid & ~keep
    out = []
    for flag, width, what, fill in ((keep, budget, pages, NO_SLOT), (keep, budget, w, 0.0), (gone, stride, pages, NO_SLOT)):
        at = torch.where(flag, flag.cumsum(1) - 1, torch.full_like(order, width))  # the place past the end takes what is left out
        out.append(torch.full((r, width + 1), fill, dtype=what.dtype, device=what.device).scatter_(1, at, what)[:, :width])
    count = keep.sum(1)
    kv_len = (s["kv_len"].long() - (n[:, 0] - count) * c).to(torch.int32)
    return {"pages": out[0], "weight": out[1], "evicted": out[2], "kv_len": kv_len}


# ---- the framework's operators ---------------------------------------------------------------------------------------------
def cache_of(s, k_scale=1.0, v_scale=1.0):
    """The cache object that a program keeps for its pool."""
    if "cache" not in s:
        from paper_2609_38706_gb300.service import KVPages
        c = s["case"]
        s["cache"] = KVPages(s["pool"].shape[0], c["page_tokens"], c["kv_heads"], c["head_dim"], k_scale=k_scale,
                             v_scale=v_scale, pool=s["pool"])
    return s["cache"]


def own_run(s):
    case, op = s["case"], s["case"]["op"]
    if op == "store":
        cache = cache_of(s, case["k_scale"], case["v_scale"])
        cache.write(s["k"], s["v"], s["tok_off"], s["start"], s["pages"])
        return list(cache.read(s["tok_off"], s["start"], s["pages"], s["k"].shape[0], s["k"].dtype))
    if op == "cache":
        out, lse = cache_of(s).attend(s["q"], s["kv_len"], s["pages"], s["scale"], weight=s["weight"])
        return {"out": out, "lse": lse} | ({} if s["weight"] is None else {"weight": s["weight"]})
    from paper_2609_38706_gb300 import service
    if op == "prompt":
        out, lse = service.attend_prompt(s["q"], s["k"], s["v"], s["q_off"], s["k_off"], s["scale"])
        return {"out": out, "lse": lse}
    pages, weight, kv_len, evicted = service.evict_pages(s["pages"], s["weight"], s["kv_len"], case["page_tokens"],
                                                         case["budget"], case["sinks"], case["recent"])
    return {"pages": pages, "weight": weight, "evicted": evicted, "kv_len": kv_len}


def run(state):
    if own:
        return own_run(state)
    return {"store": plain_store, "cache": plain_cache, "prompt": plain_prompt, "evict": plain_evict}[state["case"]["op"]](state)


# ---- work ------------------------------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "store":
        t = sum(lengths(case, case["new"], "new")) * case["kv_heads"]
        d = case["head_dim"]
        return {"bytes": t * (2 * 4 * d + 2 * (d + d // 8)), "flops": t * d * 2 * 4}
    if op == "cache":
        n, d = lengths(case, case["len"], "len"), case["head_dim"]
        rows = case["requests"] * case["queries"] * case["kv_heads"] * case["group"]
        pages = sum(-(-a // case["page_tokens"]) for a in n)
        return {"bytes": sum(n) * case["kv_heads"] * (d + d // 8) + rows * (4 * d + 4) + pages * (12 if case["weigh"] else 4),
                "flops": 4 * sum(n) * d * case["queries"] * case["kv_heads"] * case["group"]}
    if op == "prompt":
        ql, d, h = lengths(case, case["len"], "len"), case["head_dim"], case["kv_heads"] * case["group"]
        pre = lengths(case, case["prefix"], "prefix")
        pairs = sum(a * b + a * (a + 1) // 2 for a, b in zip(ql, pre))
        return {"bytes": sum(ql) * h * (4 * d + 4) + sum(a + b for a, b in zip(ql, pre)) * case["kv_heads"] * 4 * d,
                "flops": 4 * pairs * h * d}
    n = sum(lengths(case, case["pages"], "pages"))
    return {"bytes": 8 * n + case["requests"] * (8 * case["budget"] + 4 * case["pages"] + 8), "flops": n}


# ---- from the definitions, in 64 bits --------------------------------------------------------------------------------------
def e4m3_64(x):
    """x >= 0 rounded to the nearest e4m3 value, ties to even, saturating at 448."""
    e = torch.floor(torch.log2(x.clamp(min=2.0 ** -20))).clamp(min=-6.0)
    e = torch.where(torch.exp2(e) > x, (e - 1).clamp(min=-6.0), e)
    step = torch.exp2(e - 3)
    return (torch.round(x / step) * step).clamp(max=448.0)


def stored_64(x, g):
    g = float(torch.tensor(g, dtype=torch.float32))  # the scale is a 32-bit argument
    b = x.double().unflatten(-1, (-1, 16))
    den = (e4m3_64(b.abs().amax(-1) / 6 / g) * g).unsqueeze(-1)
    y = torch.where(den > 0, b / den, torch.zeros_like(b)).clamp(-6, 6)
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
    return (torch.round(y / step) * step * den).flatten(-2)


def attend_64(q, k, v, ok, scale):
    s = (q @ k.T) * scale
    s = torch.where(ok, s, torch.full_like(s, -math.inf))
    lse = torch.logsumexp(s, -1)
    p = torch.where(ok, torch.exp(s - lse[:, None]), torch.zeros_like(s))
    return p @ v, lse, p


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "store":
        return [stored_64(s["k"], case["k_scale"]), stored_64(s["v"], case["v_scale"])]
    if op == "evict":
        keep_w = torch.zeros((case["requests"], case["budget"]), dtype=torch.float64)
        w = s["weight"].double().cpu()
        for r, t in enumerate(s["kv_len"].tolist()):
            n = -(-t // case["page_tokens"])
            if n <= case["budget"]:
                kept = list(range(n))
            else:
                a, b = case["sinks"], n - case["recent"]
                room = case["budget"] - case["sinks"] - case["recent"]
                best = sorted(range(a, b), key=lambda j, row=w[r].tolist(): (-row[j], j))[:room]
                kept = sorted(list(range(a)) + best + list(range(b, n)))
            keep_w[r, : len(kept)] = w[r, kept]
        return {"pages": None, "weight": keep_w, "evicted": None, "kv_len": None}
    h, g, d = case["kv_heads"], case["group"], case["head_dim"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:-1], dtype=torch.float64, device="cuda")
    if op == "prompt":
        qo, ko = s["q_off"].tolist(), s["k_off"].tolist()
        for r in range(case["requests"]):
            a, b, e, f = qo[r], qo[r + 1], ko[r], ko[r + 1]
            ok = torch.arange(f - e, device="cuda") <= torch.arange(b - a, device="cuda")[:, None] + (f - e) - (b - a)
            for x in range(h * g):
                o, z, _ = attend_64(s["q"][a:b, x].double(), s["k"][e:f, x // g].double(), s["v"][e:f, x // g].double(), ok, s["scale"])
                out[a:b, x], lse[a:b, x] = o, z
        return {"out": out, "lse": lse}
    n, c = case["queries"], case["page_tokens"]
    weight = None if s["weight"] is None else s["weight"].double()
    lut = torch.tensor([m * (1 - 2 * b) for b in (0, 1) for m in E2M1], dtype=torch.float64, device="cuda")
    e4m3 = torch.arange(256, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()
    for r, t in enumerate(s["kv_len"].tolist()):
        raw = s["pool"][s["pages"][r, : -(-t // c)].long()].view(-1, h, c // 16, 16 * (d + d // 8))
        for x in range(h):
            gran = raw[:, x].flatten(0, 1)
            kv = []
            for j in (0, 1):
                by = gran[:, 8 * d * j: 8 * d * (j + 1)].reshape(-1, d // 2).int()
                sc = e4m3[gran[:, 16 * d + d * j: 16 * d + d * (j + 1)].reshape(-1, d // 16).int()]
                kv.append(lut[torch.stack((by % 16, by // 16), -1).reshape(-1, d)] * sc.repeat_interleave(16, 1))
            q = s["q"][r, :, x * g: (x + 1) * g].double().reshape(n * g, d)
            ok = torch.arange(kv[0].shape[0], device="cuda") <= (t - n + torch.arange(n * g, device="cuda") // g)[:, None]
            o, z, p = attend_64(q, kv[0], kv[1], ok, s["scale"])
            out[r, :, x * g: (x + 1) * g], lse[r, :, x * g: (x + 1) * g] = o.view(n, g, d), z.view(n, g)
            if weight is not None:
                weight[r, : p.shape[1] // c] += p.sum(0).view(-1, c).sum(1)
    return {"out": out, "lse": lse} | ({} if weight is None else {"weight": weight})
