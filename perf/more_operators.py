"""Measured cases of a serving layer's steps over KV pages: norms of queries and keys with the position rotation in the
same pass, attention of a chunk of new tokens over the 4-bit page cache, and attention with a sliding window and a few
first tokens that stay visible, for chunks and for single tokens.

Lengths of the requests of a case follow from the case alone; values, page numbers and weights from the seed."""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # one decode step of 64 running requests: norms and full rotation, far positions
        dict(name="rotate 64x1", op="rotate", requests=64, new=1, start=130000, q_heads=32, kv_heads=8, head_dim=128, rotary=128,
             interleaved=False, base=500000.0, factor=8.0, context=8192, norm=True, dtype="bf16"),
        # a ragged batch behind cached prefixes: neighbouring pairs, half of the head rotated, no norms, 64-wide heads
        dict(name="rotate 24x777 half d64", op="rotate", requests=24, new=777, start=2500, q_heads=12, kv_heads=4, head_dim=64,
             rotary=32, interleaved=True, base=10000.0, factor=1.0, context=0, norm=False, dtype="fp16"),
        # long prompts, norms and full rotation
        dict(name="rotate 8x8192", op="rotate", requests=8, new=8192, start=0, q_heads=32, kv_heads=8, head_dim=128, rotary=128,
             interleaved=False, base=10000.0, factor=1.0, context=0, norm=True, dtype="bf16"),
        # a lone short follow-up over a cached conversation: latency
        dict(name="chunk 1x16+1000", op="attend", requests=1, new=16, past=1000, kv_heads=8, group=4, head_dim=128, page_tokens=16,
             window=0, sinks=0, packed=True, weigh=False, dtype="bf16"),
        # tails of different lengths behind cached prefixes, odd group, odd page size, 64-wide heads
        dict(name="chunk 12x700+2048 d64", op="attend", requests=12, new=700, past=2048, kv_heads=4, group=3, head_dim=64,
             page_tokens=48, window=0, sinks=0, packed=True, weigh=False, dtype="fp16"),
        # a step of chunked prefill of four long prompts
        dict(name="chunk 4x512+16384", op="attend", requests=4, new=512, past=16384, kv_heads=8, group=4, head_dim=128, page_tokens=256,
             window=0, sinks=0, packed=True, weigh=False, dtype="bf16"),
        # a short question over a long document: few rows, long axis
        dict(name="chunk 1x40+120000", op="attend", requests=1, new=40, past=120000, kv_heads=8, group=8, head_dim=128, page_tokens=256,
             window=0, sinks=0, packed=True, weigh=False, dtype="bf16"),
        # the last large chunk of a long document
        dict(name="chunk 1x2048+60000", op="attend", requests=1, new=2048, past=60000, kv_heads=8, group=4, head_dim=128,
             page_tokens=256, window=0, sinks=0, packed=True, weigh=False, dtype="bf16"),
        # windowed layers: ragged chunks, 64-wide heads, the window ends inside tiles and pages
        dict(name="chunk 8x600+9000 w1000 d64", op="attend", requests=8, new=600, past=9000, kv_heads=4, group=5, head_dim=64,
             page_tokens=48, window=1000, sinks=4, packed=True, weigh=False, dtype="fp16"),
        # windowed layers: chunked prefill of long prompts
        dict(name="chunk 4x2048+32768 w4096", op="attend", requests=4, new=2048, past=32768, kv_heads=8, group=4, head_dim=128,
             page_tokens=256, window=4096, sinks=4, packed=True, weigh=False, dtype="bf16"),
        # windowed layers: a decode step of an ordinary batch, weights accumulated for eviction
        dict(name="step 128x8192 w1024", op="attend", requests=128, new=1, past=8191, kv_heads=8, group=4, head_dim=128, page_tokens=16,
             window=1024, sinks=4, packed=False, weigh=True, dtype="bf16"),
        # windowed layers: a speculative step over long contexts, 64-wide heads
        dict(name="step 16x65536 q4 w4096 d64", op="attend", requests=16, new=4, past=65532, kv_heads=4, group=3, head_dim=64,
             page_tokens=48, window=4096, sinks=64, packed=False, weigh=False, dtype="fp16"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("rotate", "chunk", "chunk", "chunk", "step"))
    head = dict(kv_heads=rng.choice((1, 2, 4, 8)), head_dim=rng.choice((64, 128)), dtype=rng.choice(("bf16", "fp16")))
    group = rng.choice((1, 2, 3, 4, 5, 7, 8, 16))
    if op == "rotate":
        new = log(1, 8192)
        factor = rng.choice((1.0, 4.0, 8.0))
        return dict(op=op, requests=log(1, max(1, 65536 // new)) if new > 64 else log(1, 1024), new=new, start=log(1, 200000),
                    q_heads=head["kv_heads"] * min(group, 8), rotary=16 * rng.randint(1, head["head_dim"] // 16),
                    interleaved=rng.choice((True, False)), base=rng.choice((10000.0, 500000.0)), factor=factor,
                    context=rng.choice((0, 4096)) if factor > 1 else 0, norm=rng.choice((True, False)), **head)
    windowed = rng.choice((True, False)) if op == "chunk" else True
    window = log(1, 8192) if windowed else 0
    more = dict(op="attend", group=group, page_tokens=rng.choice((16, 32, 48, 128, 256)), window=window,
                sinks=rng.choice((0, 1, 4, 100)) if windowed else 0, packed=op == "chunk", **head)
    if op == "step":
        past = log(1, 65536)
        return dict(requests=log(1, min(256, max(1, 1000000 // past))), new=rng.choice((1, 1, 1, 2, 5)), past=past,
                    weigh=rng.choice((True, False)), **more)
    new, past = log(1, 4096), rng.choice((0, log(1, 65536), log(1, 65536)))
    seen = min(window, new + past) if windowed else new + past
    heads = more["kv_heads"] * group
    room = min(2_000_000 // (new + past), 4_000_000_000 // (new * (seen + new) * heads))  # of the cache, of a plain form's scores
    return dict(requests=log(1, min(64, max(1, room))), new=new, past=past, weigh=False, **more)


def lengths(case, most, what):
    """A length for each request in [most/2, most], the first `most` itself."""
    r = random.Random("%s %d %d" % (what, most, case["requests"]))
    return [most] + [r.randint((most + 1) // 2, most) for _ in range(case["requests"] - 1)]


def sizes(case):
    """New tokens of each request, and tokens that it holds with them."""
    new = lengths(case, case["new"], "new") if case["packed"] else [case["new"]] * case["requests"]
    return new, [a + b for a, b in zip(new, lengths(case, case["past"], "past"))]


def offsets(lens):
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    return off


# ---- the 4-bit format ------------------------------------------------------------------------------------------------------
# A page holds page_tokens tokens: [kv head][granule of 16 tokens][K codes | V codes | K scales | V scales], a granule's parts
# row-major by token. Codes are e2m1, two to a byte (even dimension low), scales e4m3, one for 16 dimensions.
def quantise(x):
    """codes (0..15) and e4m3 scales of float32 x [..., D]; value = E2M1[code] * scale."""
    b = x.unflatten(-1, (-1, 16))
    s = (b.abs().amax(-1) / 6).clamp(max=448.0).to(torch.float8_e4m3fn)
    den = s.float().unsqueeze(-1)
    y = torch.where(den > 0, b.abs() / den, torch.zeros_like(b))
    mag = (y > 0.25).to(torch.uint8)
    for k, t in enumerate((0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        mag += (y >= t) if k % 2 == 0 else (y > t)
    return (mag | (torch.signbit(b).to(torch.uint8) << 3)).flatten(-2), s


def pack(k, v):
    """float32 k, v [slots, page_tokens, heads, D] -> uint8 [slots, page bytes]."""
    parts = []
    for x in (k, v):
        code, s = quantise(x.permute(0, 2, 1, 3).unflatten(2, (-1, 16)))
        parts.append(((code[..., 0::2] | (code[..., 1::2] << 4)).flatten(-2), s.view(torch.uint8).flatten(-2)))
    return torch.cat((parts[0][0], parts[1][0], parts[0][1], parts[1][1]), -1).flatten(1)


def unpack(gran, d):
    """uint8 [..., granule bytes] -> float32 k, v [..., 16, D]."""
    out = []
    for j in (0, 1):
        codes = gran[..., 8 * d * j: 8 * d * (j + 1)].unflatten(-1, (16, d // 2))
        s = gran[..., 16 * d + d * j: 16 * d + d * (j + 1)].unflatten(-1, (16, d // 16)).contiguous().view(torch.float8_e4m3fn)
        code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
        m = code & 7  # halves: 0 1 | 2 3 4 6 8 12
        halves = torch.where(m < 2, m, (2 + (m & 1)) << ((m >> 1).clamp(min=1) - 1)).float()
        x = torch.where(code > 7, -0.5 * halves, 0.5 * halves)
        out.append((x.unflatten(-1, (-1, 16)) * s.float().unsqueeze(-1)).flatten(-2))
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


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r, d, dt = case["requests"], case["head_dim"], DTYPES[case["dtype"]]
    s = {"case": case}
    i64 = dict(dtype=torch.int64, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    if case["op"] == "rotate":
        new = lengths(case, case["new"], "new")
        start = [case["start"]] + [random.Random("start %d" % j).randint(0, case["start"]) for j in range(r - 1)]
        s["tok_off"], s["start"] = torch.tensor(offsets(new), **i64), torch.tensor(start, **i32)
        # as a projection leaves them: one row of queries, keys and values a token
        qkv = keys_like((sum(new), case["q_heads"] + 2 * case["kv_heads"], d), gen, dt)
        s["q"], s["k"] = qkv[:, : case["q_heads"]], qkv[:, case["q_heads"]: case["q_heads"] + case["kv_heads"]]
        s["weight"] = [(1 + 0.3 * torch.randn(d, generator=gen, device="cuda")).to(dt) for _ in (0, 1)] if case["norm"] else [None, None]
        return s
    new, held = sizes(case)
    c, h = case["page_tokens"], case["kv_heads"]
    stride = -(-max(held) // c)
    slots = r * stride + 3
    s["pages"] = torch.randperm(slots, generator=gen, device="cuda")[: r * stride].to(torch.int32).view(r, stride).contiguous()
    pool, step = [], max(1, (1 << 25) // (c * h * d))
    for a in range(0, slots, step):
        n = min(step, slots - a)
        pool.append(pack(keys_like((n, c, h, d), gen, torch.float32), randn((n, c, h, d), gen, torch.float32)))
    s["pool"] = torch.cat(pool)
    s["kv_len"], s["q_off"] = torch.tensor(held, **i32), torch.tensor(offsets(new), **i64)
    heads = h * case["group"]
    s["q"] = randn((sum(new), heads, d) if case["packed"] else (r, case["new"], heads, d), gen, dt)
    s["scale"] = d ** -0.5
    s["weight"] = torch.rand((r, stride), generator=gen, device="cuda") * 4 if case["weigh"] else None
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------------
def plain_rotate(s):
    """Norm over the head, then the rotation; angles in 64 bits, as positions are far."""
    case = s["case"]
    rot, dev = case["rotary"], s["q"].device
    f = case["base"] ** (torch.arange(rot // 2, device=dev, dtype=torch.float64) * (-2.0 / rot))
    keep = torch.zeros_like(f)  # how much of a frequency is left as it is: by its turns in the original context
    if case["context"]:
        keep = ((f * (case["context"] / (2 * math.pi)) - 1) / 31).clamp(0, 1)
    f = f * (keep + (1 - keep) / case["factor"])
    t = torch.arange(s["q"].shape[0], device=dev)
    r = torch.searchsorted(s["tok_off"][1:], t, right=True)
    pos = s["start"][r] + t - s["tok_off"][r]
    angle = (pos.double()[:, None] * f)[:, None]
    amp = 0.1 * math.log(case["factor"]) + 1
    cos, sin = (torch.cos(angle) * amp).float(), (torch.sin(angle) * amp).float()

    def one(x, w):
        y = x.float()
        if w is not None:
            y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * w.float()
        head, rest = y[..., :rot], y[..., rot:]
        if case["interleaved"]:
            a, b = head[..., 0::2], head[..., 1::2]
            head = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
        else:
            a, b = head[..., : rot // 2], head[..., rot // 2:]
            head = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
        return torch.cat((head, rest), -1).to(x.dtype)

    return [one(s["q"], s["weight"][0]), one(s["k"], s["weight"][1])]


def plain_attend(s):
    """Granules that some query of a request can see, gathered and unpacked; scores, masks, weights, sums."""
    case, q_off = s["case"], s["q_off"]
    c, h, g, d, dev = case["page_tokens"], case["kv_heads"], case["group"], case["head_dim"], q_off.device
    held, n = s["kv_len"].long(), q_off[1:] - q_off[:-1]
    most, every = case["new"], s["pages"].shape[1] * (c // 16)
    i = torch.arange(most, device=dev)
    if case["window"]:
        first, last = -(-case["sinks"] // 16), -(-(case["window"] + most) // 16) + 1
        low = ((held - n - case["window"] + 1).clamp(min=0) // 16).clamp(min=first)
        at = torch.cat((torch.arange(first, device=dev).expand(len(held), -1), low[:, None] + torch.arange(last, device=dev)), 1)
    else:
        at = torch.arange(every, device=dev).expand(len(held), -1)
    safe = at.clamp(max=every - 1)
    slot = s["pages"].long().gather(1, safe // (c // 16))
    raw = s["pool"].unflatten(-1, (h, c // 16, 18 * d))[slot, :, safe % (c // 16)]                    # [r, granules, h, bytes]
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in unpack(raw, d))                                  # [r, h, tokens, d]
    pos = (at[..., None] * 16 + torch.arange(16, device=dev)).flatten(1)
    pos = torch.where(pos < held[:, None], pos, torch.full_like(pos, 1 << 40))
    q = s["q"][(q_off[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)] if case["packed"] else s["q"]
    q = q.float().unflatten(2, (h, g)).permute(0, 2, 3, 1, 4).flatten(2, 3)                           # [r, h, g n, d]
    mine = ((held - n)[:, None] + i)[..., None]                                                       # [r, n, 1]
    see = pos[:, None] <= mine
    if case["window"]:
        see &= (pos[:, None] > mine - case["window"]) | (pos[:, None] < case["sinks"])
    sc = (q @ k.transpose(2, 3)).unflatten(2, (g, most)).mul_(s["scale"]).masked_fill_(~see[:, None, None], -math.inf)
    m = sc.amax(-1, keepdim=True).clamp(min=-3e38)
    p = sc.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    inv = torch.where(total > 0, 1 / total, torch.zeros_like(total))
    out = ((p.flatten(2, 3) @ v).unflatten(2, (g, most)) * inv).permute(0, 3, 1, 2, 4).flatten(2, 3).to(s["q"].dtype)
    lse = (m + torch.log(total)).squeeze(-1).permute(0, 3, 1, 2).flatten(2, 3).contiguous()
    if not case["packed"]:
        if s["weight"] is None:
            return {"out": out, "lse": lse}
        page = (at[..., None].expand(-1, -1, 16).flatten(1) // (c // 16)).clamp(max=s["pages"].shape[1] - 1)
        s["weight"].scatter_add_(1, page, (p * inv).sum((1, 2, 3)))
        return {"out": out, "lse": lse, "weight": s["weight"]}
    t = torch.arange(s["q"].shape[0], device=dev)
    r = torch.searchsorted(q_off[1:], t, right=True)
    return {"out": out[r, t - q_off[r]], "lse": lse[r, t - q_off[r]]}


# ---- the framework's operators ---------------------------------------------------------------------------------------------
def own_rotate(s):
    from paper_2609_38706_gb300 import service
    case = s["case"]
    if "rotary" not in s:  # the object that a program keeps for its layers
        s["rotary"] = service.Rotary(case["head_dim"], case["rotary"], case["base"], case["interleaved"], factor=case["factor"],
                                     context=case["context"] or None, amplitude=0.1 * math.log(case["factor"]) + 1)
    return list(service.rotate(s["q"], s["k"], s["tok_off"], s["start"], s["rotary"], *s["weight"], eps=1e-6))


def own_attend(s):
    case = s["case"]
    if "cache" not in s:  # the cache object that a program keeps for its pool
        from paper_2609_38706_gb300.service import KVPages
        s["cache"] = KVPages(s["pool"].shape[0], case["page_tokens"], case["kv_heads"], case["head_dim"], pool=s["pool"])
    window = case["window"] or None
    if case["packed"]:
        out, lse = s["cache"].attend_chunk(s["q"], s["q_off"], s["kv_len"], s["pages"], s["scale"], window=window, sinks=case["sinks"])
        return {"out": out, "lse": lse}
    out, lse = s["cache"].attend(s["q"], s["kv_len"], s["pages"], s["scale"], weight=s["weight"], window=window, sinks=case["sinks"])
    return {"out": out, "lse": lse} | ({} if s["weight"] is None else {"weight": s["weight"]})


def run(state):
    if own:
        return own_rotate(state) if state["case"]["op"] == "rotate" else own_attend(state)
    return plain_rotate(state) if state["case"]["op"] == "rotate" else plain_attend(state)


# ---- work ------------------------------------------------------------------------------------------------------------------
def work(case):
    d = case["head_dim"]
    if case["op"] == "rotate":
        values = sum(lengths(case, case["new"], "new")) * (case["q_heads"] + case["kv_heads"]) * d
        return {"bytes": 4 * values, "flops": values * (7 if case["norm"] else 3)}
    new, held = sizes(case)
    w, sinks = case["window"] or 1 << 40, case["sinks"]
    pairs = keys = 0
    for n, t in zip(new, held):
        low = max(0, t - n - w + 1)
        keys += t - low + min(sinks, low)
        full = max(0, min(n, w - (t - n)))  # queries whose window reaches the first token: p + 1 keys each
        pairs += full * (t - n) + full * (full + 1) // 2
        for p in (range(t - n + full, t) if n > full else ()):
            pairs += w + min(sinks, p - w + 1)
    rows = sum(new) * case["kv_heads"] * case["group"]
    pages = -(-keys // case["page_tokens"])
    return {"bytes": keys * case["kv_heads"] * (d + d // 8) + rows * (4 * d + 4) + pages * (12 if case["weigh"] else 4),
            "flops": 4 * pairs * d * case["kv_heads"] * case["group"]}


# ---- from the definitions, in 64 bits --------------------------------------------------------------------------------------
def exact_rotate(case, s):
    rot = case["rotary"]
    freq = []
    for i in range(rot // 2):
        f = math.exp(-2.0 * i / rot * math.log(case["base"]))
        part = min(1.0, max(0.0, (case["context"] * f / (2 * math.pi) - 1.0) / (32.0 - 1.0))) if case["context"] else 0.0
        freq.append(part * f + (1.0 - part) * f / case["factor"])
    pos = torch.cat([torch.arange(a, a + n, dtype=torch.float64) for a, n in
                     zip(s["start"].tolist(), (s["tok_off"][1:] - s["tok_off"][:-1]).tolist())]).cuda()
    turn = torch.polar(torch.full((), 1 + 0.1 * math.log(case["factor"]), dtype=torch.float64, device="cuda"),
                       torch.outer(pos, torch.tensor(freq, dtype=torch.float64, device="cuda")))[:, None]
    out = []
    for x, w in ((s["q"], s["weight"][0]), (s["k"], s["weight"][1])):
        y = x.double()
        if w is not None:
            y = y * torch.rsqrt(y.square().sum(-1, keepdim=True) / y.shape[-1] + 1e-6) * w.double()
        first = torch.arange(0, rot, 2, device="cuda") if case["interleaved"] else torch.arange(rot // 2, device="cuda")
        second = first + (1 if case["interleaved"] else rot // 2)
        z = torch.complex(y[..., first], y[..., second]) * turn
        y = y.clone()
        y[..., first], y[..., second] = z.real, z.imag
        out.append(y)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotate":
        return exact_rotate(case, s)
    h, g, d, c = case["kv_heads"], case["group"], case["head_dim"], case["page_tokens"]
    q = s["q"].flatten(0, 1) if not case["packed"] else s["q"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(q.shape[:-1], dtype=torch.float64, device="cuda")
    weight = None if s["weight"] is None else s["weight"].double()
    lut = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")
    e4m3 = torch.arange(256, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()
    off = s["q_off"].tolist()
    for r, t in enumerate(s["kv_len"].tolist()):
        a, b = off[r], off[r + 1]
        at = torch.arange(t, device="cuda")
        mine = torch.arange(t - (b - a), t, device="cuda")[:, None]
        ok = at <= mine
        if case["window"]:
            ok = ok & ((mine - at < case["window"]) | (at < case["sinks"]))
            at = torch.nonzero(ok.any(0)).flatten()  # keys that nobody sees are left out
            ok = ok[:, at]
        raw = s["pool"][s["pages"][r].long()[at // c]].view(len(at), h, c // 16, 18 * d)[torch.arange(len(at), device="cuda"), :, at % c // 16]
        tok = at % 16
        for x in range(h):
            kv = []
            for j in (0, 1):
                by = raw[:, x, 8 * d * j: 8 * d * (j + 1)].view(-1, 16, d // 2)[torch.arange(len(at), device="cuda"), tok].int()
                sc = e4m3[raw[:, x, 16 * d + d * j: 16 * d + d * (j + 1)].view(-1, 16, d // 16)[torch.arange(len(at), device="cuda"), tok].int()]
                kv.append(lut[torch.stack((by % 16, by // 16), -1).reshape(-1, d)] * sc.repeat_interleave(16, 1))
            for y in range(x * g, (x + 1) * g):
                z = (q[a:b, y].double() @ kv[0].T) * s["scale"]
                z = z.masked_fill(~ok, -math.inf)
                lse[a:b, y] = torch.logsumexp(z, -1)
                p = torch.exp(z - lse[a:b, y, None])
                out[a:b, y] = p @ kv[1]
                if weight is not None:
                    weight[r].index_add_(0, at // c, p.sum(0))
    out, lse = out.view(s["q"].shape), lse.view(s["q"].shape[:-1])
    return {"out": out, "lse": lse} | ({} if weight is None else {"weight": weight})
