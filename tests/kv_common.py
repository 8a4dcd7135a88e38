"""Plain implementations, in 64 bits, of the paged 4-bit key/value cache's operators."""
import math

import numpy as np
import torch


def up(a, b):
    return -(-a // b)


def plan_ref(ctx, new, table, ring, state, page, max_tokens):
    """The bookkeeping of one step, a request at a time.  Returns the outputs and the updated table, ring, state."""
    table, ring = table.copy(), ring.copy()
    cap, width = len(ring), table.shape[1]
    head, count = state
    q_start, kv_len = [0], []
    positions, slots = np.full(max_tokens, -1, np.int64), np.full(max_tokens, -1, np.int64)
    used = freed = asked = 0
    old_table = table.copy()
    for r, (c, n) in enumerate(zip(ctx, new)):
        if n < 0:
            for j in range(min(up(max(c, 0), page), width)):
                ring[(head + count + freed) % cap] = old_table[r, j]
                freed += 1
        q0, q1 = q_start[-1], q_start[-1] + max(n, 0)
        q_start.append(q1)
        fits = n >= 0 and c >= 0 and up(c + n, page) <= width and q1 <= max_tokens
        need = up(c + n, page) - up(c, page) if fits else 0
        asked += need
        if not fits or (need and asked > count):
            kv_len.append(0)
            continue
        for j in range(need):
            table[r, up(c, page) + j] = ring[(head + used) % cap]
            used += 1
        kv_len.append(c + n)
        for i in range(n):
            positions[q0 + i] = c + i
            slots[q0 + i] = int(table[r, (c + i) // page]) * page + (c + i) % page
    q_start = np.minimum(np.array(q_start), max_tokens)
    return q_start, np.array(kv_len), positions, slots, table, ring, ((head + used) % cap, count + freed - used)


def boundaries(base):
    out = []
    for j in range(7):
        t = base ** (j - 6.5)
        f = np.float32(t)
        out.append(f if float(f) >= t else np.nextafter(f, np.float32(np.inf)))
    return np.array(out, np.float32)


def level_values(base, dtype):
    pos = torch.tensor([0.0] + [base ** (m - 7) for m in range(1, 8)], dtype=torch.float64).float().to(dtype).double()
    return torch.cat([pos, -pos])


def quantise_ref(x, base):
    """16-bit vectors [..., d] -> (packed codes, ranges, values), from the definition."""
    a = x.detach().cpu().float().numpy()
    top = np.abs(a).max(-1)
    bad = ~np.isfinite(a).all(-1)
    bound = (boundaries(base) * np.where(bad, 0, top)[..., None].astype(np.float32)).astype(np.float32)
    m = (np.abs(a)[..., None] >= bound[..., None, :]).sum(-1)
    m[(top == 0) | bad] = 0
    c = (m + 8 * ((a < 0) & (m > 0))).astype(np.uint8)
    packed = c[..., 0::2] | (c[..., 1::2] << 4)
    rng = torch.from_numpy(np.where(bad, np.nan, top).astype(np.float32)).to(x.dtype)
    val = level_values(base, x.dtype).numpy()[c] * rng.double().numpy()[..., None]
    return torch.from_numpy(packed), rng, torch.from_numpy(val)


def cached_vectors(codes, ranges, ids, head, base, dtype):
    """[len(ids) * page, d] values in 64 bits of one head of the listed pages."""
    b = codes[ids, head].flatten(0, 1).long()
    c = torch.stack([b & 15, b >> 4], -1).flatten(-2)
    return level_values(base, dtype).to(codes.device)[c] * ranges[ids, head].flatten().double().unsqueeze(-1)


def attention_ref(cache, q, q_start, kv_len, table, scale, window, k_base, v_base):
    """(out, bound) in 64 bits.  bound: what the kernel's arithmetic may differ by, element by element --
    the output's rounding; the rounding of each weight to fp16 (2^-11 of it, or 2^-25 of the largest
    where it is subnormal); 32-bit products, sums and 2^x (a relative 2^-23 for each addition of a chain,
    2^-20 for the rest), scores weighted by how far they move the result."""
    dev = q.device
    tokens, hq, d = q.shape
    g, page = hq // cache.heads, cache.page_size
    out = torch.full((tokens, hq, d), float("nan"), dtype=torch.float64, device=dev)
    bound = torch.zeros_like(out)
    half = 2.0 ** -8 if q.dtype == torch.bfloat16 else 2.0 ** -11
    starts, kvs = [int(x) for x in q_start], [int(x) for x in kv_len]
    for r in range(len(kvs)):
        a, b = starts[r], starts[r + 1]
        n, kv = b - a, max(kvs[r], 0)
        if n <= 0:
            continue
        seen_kv = min(kv, table.shape[1] * page)
        ids = table[r, :up(seen_kv, page)].long()
        real = ((ids >= 0) & (ids < cache.pages)).repeat_interleave(page)[:seen_kv]
        ids = ids.clamp(0, cache.pages - 1)
        p = torch.arange(kv - n, kv, device=dev).unsqueeze(1)
        j = torch.arange(seen_kv, device=dev).unsqueeze(0)
        seen = (j <= p) & real
        if window:
            seen &= j > p - window
        for h in range(cache.heads):
            if seen_kv == 0:
                out[a:b, h * g:(h + 1) * g] = 0
                continue
            k = cached_vectors(cache.k_codes, cache.k_range, ids, h, k_base, q.dtype)[:seen_kv]
            v = cached_vectors(cache.v_codes, cache.v_range, ids, h, v_base, q.dtype)[:seen_kv]
            any_seen = seen.any(0).unsqueeze(1)          # what no query sees may hold anything
            k, v = torch.where(any_seen, k, 0.0), torch.where(any_seen, v, 0.0)
            biggest = cache.v_range[ids, h].flatten()[:seen_kv].double()
            for z in range(h * g, h * g + g):
                x = q[a:b, z].double()
                s = (x @ k.T * scale).masked_fill(~seen, -math.inf)
                size = (x.abs() @ k.abs().T * abs(scale)).masked_fill(~seen, 0.0).amax(1, keepdim=True)
                w = torch.softmax(s, -1).masked_fill(~seen.any(1, keepdim=True), 0.0)
                w = torch.where(seen, w, 0.0)
                # 0 * NaN of a key that another query sees must not reach this one
                o = torch.stack([(w[i].unsqueeze(1) * v)[seen[i]].sum(0) for i in range(n)]) if v.isnan().any() else w @ v
                mass = w @ v.abs().nan_to_num()
                moved = 2.0 ** -20 + (d + 16) * 2.0 ** -23 * size
                top = torch.where(seen, biggest.nan_to_num(), 0.0).amax(1, keepdim=True)
                out[a:b, z] = o
                bound[a:b, z] = (half * o.abs() + (2.0 ** -11 + 2 * moved + (seen_kv / 16 + 64) * 2.0 ** -23) * mass +
                                 seen_kv * 2.0 ** -25 * top + 2.0 ** -24)
    return out, bound


def check_attention(got, ref, bound):
    written = ~ref.isnan()
    err = (got.double() - ref).abs()
    worst = torch.where(written, err / bound, 0.0)
    assert not (worst > 1).any(), f"{int((worst > 1).sum())} outputs beyond the bound, worst {float(worst.max()):.2f} of it"
    assert not got[written].isnan().any()
    return float(worst.max())
