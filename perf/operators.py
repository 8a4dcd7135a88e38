"""Cases of the paged 4-bit key/value cache: block tables and slot maps, appending tokens, attention.

A serving step of a model with grouped-query attention keeps its keys and values in
fixed-size pages.  Three operators run per step and layer:

  plan    block tables, slot map, positions and cumulative lengths from the requests' lengths
  append  16-bit keys and values of the step's tokens -> 4-bit Log_b codes in their slots
  attend  attention of the step's queries over the cached tokens of their requests

Cache format: pages of `page` tokens; per page, kv head and token, d/2 bytes of codes
(two 4-bit codes a byte, the even dimension in the low half: sign << 3 | m) and one
16-bit range, the vector's largest magnitude.  A code stands for
range * sign * L_m with L_0 = 0 and L_m = base^(m - 7) rounded to the cache's type,
and m = #{ j < 7 : |x| >= T_j * range } (product in 32 bits) with T_j = base^(j - 6.5)
rounded up to 32 bits.

A query at position p of its request attends to the keys at max(0, p - window + 1) .. p
(window 0: all up to p); the last query of a request sits at its last cached position.
A query that sees no key gives zeros.
"""
import math
import random

import numpy as np
import torch

own = False

BASE_K, BASE_V = 1.5, 1.6          # bases of the key and value codebooks
SKIPPED = 13                       # of the tokens of a padded append, each 13th has no slot


# ------------------------------------------------------------------ cases ---

def listed():
    def plan(name, requests, page, kv_hi, prompts, prompt_hi, ended, pad):
        return {"name": name, "op": "plan", "requests": requests, "page": page, "kv_hi": kv_hi, "prompts": prompts,
                "prompt_hi": prompt_hi, "ended": ended, "pad": pad}

    def append(name, tokens, dtype, h, d, hq, page, padded):
        return {"name": name, "op": "append", "tokens": tokens, "dtype": dtype, "h": h, "d": d, "hq": hq, "page": page,
                "padded": padded}

    def attend(name, dtype, hq, h, d, page, requests, q_lo, q_hi, kv_lo, kv_hi, singles=0, window=0):
        return {"name": name, "op": "attend", "dtype": dtype, "hq": hq, "h": h, "d": d, "page": page,
                "requests": requests, "q_lo": q_lo, "q_hi": q_hi, "kv_lo": kv_lo, "kv_hi": kv_hi, "singles": singles,
                "window": window}

    return [
        # one decode step's bookkeeping: 64 running requests, a token each
        plan("plan-decode-64", 64, 64, 8192, 0, 0, 0, 0),
        # a busy server's step: 1024 requests, some finishing, some starting with prompts, padded token buffers
        plan("plan-mixed-1024", 1024, 16, 8192, 40, 2048, 50, 333),
        # the cache write of one 8B layer in a decode step of 64 requests
        append("append-decode-64", 64, "bf16", 8, 128, 32, 64, False),
        # an odd batch of prompts of the 1B model, in fp16, with padding tokens that have no slot
        append("append-ragged-5003", 5003, "f16", 8, 64, 32, 16, True),
        # the cache write of a full prefill batch of an 8B layer
        append("append-prompt-16384", 16384, "bf16", 8, 128, 32, 64, False),
        # single-user decode, 8B heads: latency
        attend("decode-1x4001", "bf16", 32, 8, 128, 64, 1, 1, 1, 4001, 4001),
        # batched decode, 8B heads, ragged context lengths
        attend("decode-64-ragged", "bf16", 32, 8, 128, 64, 64, 1, 1, 17, 8191),
        # long-document decode, 1B heads in fp16
        attend("decode-4x131000", "f16", 32, 8, 64, 32, 4, 1, 1, 130001, 131072),
        # speculative decoding: a few draft tokens a request are checked at once
        attend("verify-16x5", "bf16", 32, 8, 128, 16, 16, 5, 5, 300, 5000),
        # the next piece of a long prompt beside running requests (chunked prefill)
        attend("chunk-512-of-16k", "bf16", 32, 8, 128, 64, 4, 512, 512, 15000, 16384, 3),
        # a whole prompt, 8B heads
        attend("prompt-8192", "bf16", 32, 8, 128, 64, 1, 8192, 8192, 8192, 8192),
        # a batch of short prompts with as many kv heads as query heads and a sliding window, 1B head size, fp16
        attend("prompts-window-mha", "f16", 16, 16, 64, 16, 8, 60, 1500, 60, 1500, 0, 256),
    ]


def spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "append", "append", "decode", "decode", "verify", "prompt", "prompt"])
    dtype = rng.choice(["bf16", "f16"])
    page = rng.choice([16, 32, 64, 128])
    if kind == "plan":
        requests = spread(rng, 1, 1024)
        prompts = rng.randrange(0, requests // 16 + 1)
        return {"op": "plan", "requests": requests, "page": page, "kv_hi": spread(rng, 64, 8192), "prompts": prompts,
                "prompt_hi": spread(rng, 2, 2048), "ended": rng.randrange(0, requests // 8 + 1), "pad": rng.randrange(0, 500)}
    h, hq = rng.choice([(8, 32), (8, 32), (2, 16), (4, 28), (16, 16)])
    d = rng.choice([64, 128])
    if kind == "append":
        return {"op": "append", "tokens": spread(rng, 1, 16384), "dtype": dtype, "h": min(h, 8), "d": d, "hq": hq,
                "page": page, "padded": rng.random() < 0.5}
    window = rng.choice([0, 0, 0, rng.randrange(50, 3000)])
    case = {"op": "attend", "dtype": dtype, "hq": hq, "h": h, "d": d, "page": page, "requests": 1, "q_lo": 1, "q_hi": 1,
            "kv_lo": 1, "kv_hi": 1, "singles": 0, "window": window}
    if kind in ("decode", "verify"):
        case["requests"] = spread(rng, 1, 64)
        case["kv_hi"] = spread(rng, 20, min(100000, 300000 // case["requests"] + 20))
        case["kv_lo"] = max(1, int(case["kv_hi"] * rng.random()))
        if kind == "verify":
            case["q_lo"], case["q_hi"] = 1, rng.randrange(2, 10)
    else:
        case["requests"] = spread(rng, 1, 8)
        case["q_hi"] = spread(rng, 20, 4096 // case["requests"])
        case["q_lo"] = max(1, int(case["q_hi"] * rng.random()))
        case["kv_lo"] = case["q_lo"] + rng.choice([0, spread(rng, 1, 4096)])
        case["kv_hi"] = max(case["kv_lo"], case["q_hi"]) + rng.randrange(0, 500)
        case["singles"] = rng.randrange(0, case["requests"])
    return case


def lengths(c):
    """(query lengths, cached lengths) of an attend case; (cached, new) lengths of a plan case."""
    r = random.Random(repr(sorted((k, v) for k, v in c.items() if k != "name")))
    if c["op"] == "attend":
        q = [1 if i >= c["requests"] - c["singles"] else r.randint(c["q_lo"], c["q_hi"]) for i in range(c["requests"])]
        kv = [max(n, r.randint(c["kv_lo"], c["kv_hi"])) for n in q]
        return q, kv
    n = c["requests"]
    kind = ["prompt"] * c["prompts"] + ["ended"] * c["ended"] + ["running"] * max(0, n - c["prompts"] - c["ended"])
    kind = kind[:n]
    r.shuffle(kind)
    ctx = [0 if k == "prompt" else r.randint(1, c["kv_hi"]) for k in kind]
    new = [r.randint(1, c["prompt_hi"]) if k == "prompt" else -1 if k == "ended" else 1 for k in kind]
    return ctx, new


def up(a, b):
    return -(-a // b)


def work(case):
    c = case
    if c["op"] == "plan":
        ctx, new = lengths(c)
        taken = sum(up(x + n, c["page"]) - up(x, c["page"]) for x, n in zip(ctx, new) if n > 0)
        freed = sum(up(x, c["page"]) for x, n in zip(ctx, new) if n < 0)
        tokens = sum(n for n in new if n > 0) + c["pad"]
        # lengths in, cumulative and cached lengths out, pages moved, a table entry and two results a token
        return {"bytes": 16.0 * c["requests"] + 8 * (taken + freed) + 16 * tokens, "flops": 0}
    if c["op"] == "append":
        n = c["tokens"] * c["h"]
        # keys and values in; codes, ranges and the values they stand for out
        return {"bytes": 2.0 * n * (2 * c["d"] + c["d"] // 2 + 2 + 2 * c["d"]) + 8 * c["tokens"], "flops": 0}
    q, kv = lengths(c)
    seen = pairs = 0
    for n, m in zip(q, kv):
        w = c["window"] or m
        seen += m - max(0, m - n - w + 1)
        first = m - n
        full = max(0, min(n, w - 1 - first)) if first < w - 1 else 0        # rows that see all keys up to their own
        pairs += full * first + full * (full + 1) // 2 + (n - full) * w
    return {"bytes": 4.0 * sum(q) * c["hq"] * c["d"] + 2.0 * seen * c["h"] * (c["d"] // 2 + 2) + 4 * up(seen, c["page"]),
            "flops": 4.0 * pairs * c["hq"] * c["d"]}


# ----------------------------------------------------------------- inputs ---

def dtype_of(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float16


def levels(base, dtype):
    """The 16 values of a code with range 1, and the 7 boundaries, in 32 bits."""
    pos = np.array([0.0] + [base ** (m - 7) for m in range(1, 8)]).astype(np.float32)
    lv = torch.from_numpy(np.concatenate([pos, -pos])).to(dtype).float()
    t = np.array([base ** (j - 6.5) for j in range(7)])
    t32 = t.astype(np.float32)
    t32 = np.where(t32 < t, np.nextafter(t32, np.float32(np.inf)), t32).astype(np.float32)
    return lv.cuda(), torch.from_numpy(t32).cuda()


def quantise(x, thresh):
    """(codes [..., d] as whole numbers, ranges [...]) of 16-bit vectors."""
    r = x.abs().amax(-1)
    bound = thresh * r.float().unsqueeze(-1)                                  # [..., 7]
    m = (x.float().abs().unsqueeze(-1) >= bound.unsqueeze(-2)).sum(-1, dtype=torch.uint8)
    m = torch.where((r == 0).unsqueeze(-1), torch.zeros_like(m), m)
    return m + 8 * ((x < 0) & (m > 0)).to(torch.uint8), r


def packed(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def fill(pages, c, base, gen, spread_channels):
    """Cached vectors of a layer: codes [pages, h, page, d/2] and ranges [pages, h, page]."""
    dt = dtype_of(c)
    thresh = levels(base, dt)[1]
    codes = torch.empty(pages, c["h"], c["page"], c["d"] // 2, dtype=torch.uint8, device="cuda")
    ranges = torch.empty(pages, c["h"], c["page"], dtype=dt, device="cuda")
    scale = torch.ones(c["h"], 1, c["d"], device="cuda")
    if spread_channels:                                                       # keys have a few large channels
        scale = 0.5 + 2.0 * torch.rand(c["h"], 1, c["d"], generator=gen, device="cuda") ** 4
    step = max(1, (1 << 25) // (c["h"] * c["page"] * c["d"]))
    for a in range(0, pages, step):
        b = min(pages, a + step)
        x = torch.randn(b - a, c["h"], c["page"], c["d"], generator=gen, device="cuda") * scale
        m, r = quantise(x.to(dt), thresh)
        codes[a:b], ranges[a:b] = packed(m), r
    return codes, ranges


def tables(counts, total, spare, gen):
    """Block table [requests, widest + spare] over randomly ordered pages; unused entries -1."""
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    n = torch.tensor(counts, device="cuda")
    col = torch.arange(max(counts) + spare, device="cuda")
    held = col < n.unsqueeze(1)
    at = (n.cumsum(0) - n).unsqueeze(1) + col
    return torch.where(held, order[at.clamp(max=total - 1)], torch.full((), -1, dtype=torch.int32, device="cuda")), order


def handle(s, c):
    """The cache as the framework's calls take it, kept by a program beside its tensors."""
    import paper_2607_01127_gb300 as logq
    return logq.KVCache(s["k_codes"], s["k_range"], s["v_codes"], s["v_range"],
                        logq.logq_build_codebook(4, BASE_K, 1.0), logq.logq_build_codebook(4, BASE_V, 1.0))


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"op": c["op"], "case": c}
    if c["op"] == "plan":
        ctx, new = lengths(c)
        held = [up(x, c["page"]) for x in ctx]
        need = sum(up(x + n, c["page"]) - up(x, c["page"]) for x, n in zip(ctx, new) if n > 0)
        total = sum(held) + need + 37
        width = max(up(max(n, 0) + x, c["page"]) for x, n in zip(ctx, new))
        s["block_table"], order = tables(held, total, max(1, width - max(held)), gen)
        s["ctx_len"] = torch.tensor(ctx, dtype=torch.int32, device="cuda")
        s["new_len"] = torch.tensor(new, dtype=torch.int32, device="cuda")
        # the free pages queue in a ring that has gone round
        free = total - sum(held)
        head = total - free // 2
        s["ring"] = torch.zeros(total, dtype=torch.int32, device="cuda")
        s["ring"][(head + torch.arange(free, device="cuda")) % total] = order[sum(held):]
        s["ring_state"] = torch.tensor([head, free], dtype=torch.int32, device="cuda")
        s["max_tokens"] = sum(n for n in new if n > 0) + c["pad"]
        s["page"] = c["page"]
        return s
    dt = dtype_of(c)
    if c["op"] == "append":
        n, wide = c["tokens"], (c["hq"] + 2 * c["h"]) * c["d"]
        pages = up(n, c["page"]) + 5
        # the step's keys and values are slices of a fused projection's output
        qkv = torch.randn(n, wide, generator=gen, device="cuda").to(dt)
        s["k"] = qkv[:, c["hq"] * c["d"]:(c["hq"] + c["h"]) * c["d"]].view(n, c["h"], c["d"])
        s["v"] = qkv[:, (c["hq"] + c["h"]) * c["d"]:].view(n, c["h"], c["d"])
        order = torch.randperm(pages, generator=gen, device="cuda")
        t = torch.arange(n, device="cuda")
        s["slots"] = order[t // c["page"]] * c["page"] + t % c["page"]
        if c["padded"]:
            s["slots"][SKIPPED - 1::SKIPPED] = -1
        for x in ("k", "v"):
            s[x + "_codes"] = torch.zeros(pages, c["h"], c["page"], c["d"] // 2, dtype=torch.uint8, device="cuda")
            s[x + "_range"] = torch.zeros(pages, c["h"], c["page"], dtype=dt, device="cuda")
        s["k_table"], s["v_table"] = levels(BASE_K, dt), levels(BASE_V, dt)
        if own:
            s["cache"] = handle(s, c)
        return s
    q, kv = lengths(c)
    counts = [up(m, c["page"]) for m in kv]
    pages = sum(counts) + 3
    s["k_codes"], s["k_range"] = fill(pages, c, BASE_K, gen, True)
    s["v_codes"], s["v_range"] = fill(pages, c, BASE_V, gen, False)
    s["block_table"], _ = tables(counts, pages, 1, gen)
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device="cuda")
    s["q_start"] = torch.tensor(np.concatenate([[0], np.cumsum(q)]), dtype=torch.int32, device="cuda")
    wide = (c["hq"] + 2 * c["h"]) * c["d"]
    qkv = (1.5 * torch.randn(sum(q), wide, generator=gen, device="cuda")).to(dt)
    s["q"] = qkv[:, :c["hq"] * c["d"]].view(sum(q), c["hq"], c["d"])
    s["max_q"], s["max_kv"] = max(q), max(kv)
    s["k_table"], s["v_table"] = levels(BASE_K, dt), levels(BASE_V, dt)
    if own:
        import paper_2607_01127_gb300 as logq
        s["cache"] = handle(s, c)
        s["workspace"] = logq.new_kv_workspace(c["hq"], c["h"], c["d"])
    return s


# ------------------------------------------------------------- plain form ---

def plain_plan(s):
    page, ring, table = s["page"], s["ring"], s["block_table"]
    ctx, new = s["ctx_len"].long(), s["new_len"].long()
    cap, width = ring.numel(), table.shape[1]
    n = new.clamp(min=0)
    q_end = n.cumsum(0)
    old, want = (ctx + page - 1) // page, (ctx + n + page - 1) // page
    ok = (want <= width) & (q_end <= s["max_tokens"]) & (new >= 0)
    need = torch.where(ok, want - old, 0)
    first = need.cumsum(0) - need
    head, count = s["ring_state"].long()
    ok = ok & ((need == 0) | (first + need <= count))
    need = torch.where(ok, need, 0)
    kv_len = torch.where(ok, ctx + n, 0)
    q_start = torch.cat([torch.zeros_like(q_end[:1]), q_end.clamp(max=s["max_tokens"])])
    # new pages into the table
    col = torch.arange(width, device="cuda")
    k = col - old.unsqueeze(1)
    fresh = (k >= 0) & (k < need.unsqueeze(1))
    taken = ring[((head + first.unsqueeze(1) + k.clamp(min=0)) % cap)]
    after = torch.where(fresh, taken, table)
    # the pages of ended requests go to the ring's tail
    freed = (new < 0).unsqueeze(1) & (col < old.unsqueeze(1))
    order = freed.flatten().cumsum(0).view_as(freed)
    to = torch.where(freed, (head + count + order - 1) % cap, cap)
    grown = torch.cat([ring, ring[:1]]).scatter(0, to.flatten(), table.flatten())
    s["ring"].copy_(grown[:cap])
    s["block_table"].copy_(after)
    state = torch.stack([(head + need.sum()) % cap, count - need.sum() + freed.sum()]).int()
    # tokens
    t = torch.arange(s["max_tokens"], device="cuda")
    r = torch.searchsorted(q_end, t, right=True)
    live = r < ctx.numel()
    r = r.clamp(max=ctx.numel() - 1)
    live = live & ok[r]
    pos = ctx[r] + t - (q_end - n)[r]
    slot = after[r, (pos // page).clamp(min=0, max=width - 1)].long() * page + pos % page
    return {"q_start": q_start.int(), "kv_len": kv_len.int(), "positions": torch.where(live, pos, -1).int(),
            "slots": torch.where(live, slot, -1), "block_table": s["block_table"], "ring": s["ring"], "ring_state": state}


def plain_append(s):
    c = s["case"]
    out, slots = {}, s["slots"]
    live = slots >= 0
    pages, page = s["k_codes"].shape[0], c["page"]
    at = torch.where(live, slots, pages * page)                               # tokens without a slot: a spare page
    for x in ("k", "v"):
        level, thresh = s[x + "_table"]
        codes, r = quantise(s[x], thresh)
        out[x] = (level[codes.long()] * r.float().unsqueeze(-1)).to(s[x].dtype)
        for name, value in (("_codes", packed(codes)), ("_range", r)):
            buf = s[x + name]
            grown = torch.cat([buf, buf[:1]])
            grown[at // page, :, at % page] = value
            buf.copy_(grown[:-1])
        out[x + "_range"] = s[x + "_range"]
    return out


def plain_attend(s):
    c, q, page = s["case"], s["q"], s["case"]["page"]
    h, g, d, n_q, n_kv = c["h"], c["hq"] // c["h"], c["d"], s["max_q"], s["max_kv"]
    start, kv = s["q_start"].long(), s["kv_len"].long()
    lens = start[1:] - start[:-1]
    requests = kv.numel()
    j = torch.arange(n_kv, device="cuda")
    pages = s["block_table"][:, j // page].long().clamp(min=0)               # [requests, keys]

    def vectors(x):
        level = s[x + "_table"][0]
        b = s[x + "_codes"][pages, :, j % page].transpose(1, 2).int()        # [requests, h, keys, d/2]
        r = s[x + "_range"][pages, :, j % page].transpose(1, 2).float()
        return level[torch.stack([b & 15, b >> 4], -1).flatten(-2)] * r.unsqueeze(-1)

    i = torch.arange(n_q, device="cuda")
    row = (start[:-1].unsqueeze(1) + i).clamp(max=q.shape[0] - 1)
    qs = q[row].float().view(requests, n_q, h, g, d).permute(0, 2, 3, 1, 4).reshape(requests, h, g * n_q, d)
    score = (qs @ vectors("k").transpose(2, 3)).view(requests, h, g, n_q, n_kv).mul_(1.0 / math.sqrt(d))
    pos = (kv - lens).unsqueeze(1) + i                                        # [requests, n_q]
    seen = (j <= pos.unsqueeze(2)) & (i < lens.unsqueeze(1)).unsqueeze(2)
    if c["window"]:
        seen = seen & (j > pos.unsqueeze(2) - c["window"])
    score = score.masked_fill_(~seen.view(requests, 1, 1, n_q, n_kv), -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(requests, h, g * n_q, n_kv) @ vectors("v")).view(requests, h, g, n_q, d)
    o = torch.where(total > 0, o / total, 0.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(requests, n_q, h * g, d)
    t = torch.arange(q.shape[0], device="cuda")
    r = torch.searchsorted(start[1:], t, right=True)
    return o[r, t - start[r]].to(q.dtype)


def run(state):
    s = state
    if own:
        import paper_2607_01127_gb300 as logq
        if s["op"] == "plan":
            q_start, kv_len, positions, slots, ring_state = logq.logq_kv_plan(
                s["ctx_len"], s["new_len"], s["block_table"], s["ring"], s["ring_state"], s["page"], s["max_tokens"],
                inplace=False)
            return {"q_start": q_start, "kv_len": kv_len, "positions": positions, "slots": slots,
                    "block_table": s["block_table"], "ring": s["ring"], "ring_state": ring_state}
        if s["op"] == "append":
            k, v = logq.logq_kv_append(s["cache"], s["k"], s["v"], s["slots"], values=True)
            return {"k": k, "v": v, "k_range": s["k_range"], "v_range": s["v_range"]}
        return logq.logq_kv_attention(s["cache"], s["q"], s["q_start"], s["kv_len"], s["block_table"],
                                      window=s["case"]["window"], max_q=s["max_q"], workspace=s["workspace"])
    return {"plan": plain_plan, "append": plain_append, "attend": plain_attend}[s["op"]](s)


# ------------------------------------------------------------ in 64 bits ---

def exact(case, seed):
    c = case
    if c["op"] == "plan":
        return None                                                           # whole numbers only
    s = prepare(c, seed)
    dt = dtype_of(c)

    def level64(base):
        lv = torch.tensor([base ** (m - 7.0) for m in range(1, 8)], dtype=torch.float64).float().to(dt).double()
        return torch.cat([torch.zeros(1, dtype=torch.float64), lv]).cuda()

    if c["op"] == "append":
        out = {}
        for x, base in (("k", BASE_K), ("v", BASE_V)):
            val = s[x].double()
            r = val.abs().max(-1).values
            # the level whose decision interval holds |x| / range
            m = torch.zeros_like(val, dtype=torch.long)
            for j in range(7):
                m += val.abs() >= base ** (j - 6.5) * r.unsqueeze(-1)
            out[x] = torch.sign(val) * level64(base)[m] * r.unsqueeze(-1)
            held = torch.zeros(s[x + "_range"].shape, dtype=torch.float64, device="cuda")
            for_slot = s["slots"][s["slots"] >= 0]
            held[for_slot // c["page"], :, for_slot % c["page"]] = r[s["slots"] >= 0]
            out[x + "_range"] = held
        return out
    q, kv = lengths(c)
    if 4.0 * sum(a * b for a, b in zip(q, kv)) * c["hq"] * c["d"] > 1.2e13:
        return None
    g, at = c["hq"] // c["h"], 0
    out = torch.zeros(sum(q), c["hq"], c["d"], dtype=torch.float64, device="cuda")
    lk, lv = level64(BASE_K), level64(BASE_V)

    def dense(codes, ranges, ids, head, n, lev):
        b = codes[ids, head].flatten(0, 1)[:n].long()
        nib = torch.empty(n, c["d"], dtype=torch.long, device="cuda")
        nib[:, 0::2], nib[:, 1::2] = b % 16, b // 16
        sign = 1.0 - 2.0 * (nib // 8).double()
        return sign * lev[nib % 8] * ranges[ids, head].flatten()[:n].double().unsqueeze(1)

    for r, (n, m) in enumerate(zip(q, kv)):
        ids = s["block_table"][r, :up(m, c["page"])].long()
        p = torch.arange(m - n, m, device="cuda").unsqueeze(1)
        key = torch.arange(m, device="cuda").unsqueeze(0)
        hidden = key > p
        if c["window"]:
            hidden |= key <= p - c["window"]
        for head in range(c["h"]):
            k = dense(s["k_codes"], s["k_range"], ids, head, m, lk)
            v = dense(s["v_codes"], s["v_range"], ids, head, m, lv)
            for z in range(head * g, head * g + g):
                w = s["q"][at:at + n, z].double() @ k.T / math.sqrt(c["d"])
                out[at:at + n, z] = torch.softmax(w.masked_fill_(hidden, -math.inf), -1) @ v
        at += n
    return out
