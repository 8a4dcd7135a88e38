"""The paged 4-bit key/value cache on the GPU against plain implementations in 64 bits."""
import math

import numpy as np
import pytest
import torch

from gpu_common import lib
from kv_common import attention_ref, check_attention, plan_ref, quantise_ref, up

pytestmark = pytest.mark.gpu

BF, FH = torch.bfloat16, torch.float16
KB, VB = 1.5, 1.6


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


# -------------------------------------------------------------------- plan ---

def run_plan(logq, ctx, new, table, ring, state, page, max_tokens, inplace):
    t, rg, st = i32(table), i32(ring), i32(state)
    ws = logq.new_workspace()
    got = logq.logq_kv_plan(i32(ctx), i32(new), t, rg, st, page, max_tokens, inplace=inplace, workspace=ws)
    assert (got[4] is st) == inplace
    if not inplace:
        assert st.tolist() == list(state)
    assert int(ws.sum()) == 0                              # the arrival count is back at zero
    return [x.cpu().numpy() for x in (*got[:4], t, rg, got[4])]


def make_plan(rng, requests, page, kv_hi, prompt_hi, free, width_cut=0):
    kind = rng.choice(3, requests, p=[0.7, 0.2, 0.1])
    ctx = np.where(rng.random(requests) < 0.1, 0, rng.integers(0, kv_hi + 1, requests))
    new = np.where(kind == 0, 1, np.where(kind == 1, rng.integers(0, prompt_hi + 1, requests), -1))
    held = -(-ctx // page)
    width = max(1, int((-(-(ctx + np.maximum(new, 0)) // page)).max()) - width_cut)
    held = np.minimum(held, width)
    total = int(held.sum()) + free
    order = rng.permutation(total)
    table = np.full((requests, width), -1)
    at = 0
    for r in range(requests):
        table[r, :held[r]] = order[at:at + held[r]]
        at += held[r]
    cap = max(total, 1)
    head = int(rng.integers(0, cap))
    ring = np.full(cap, -7)
    ring[(head + np.arange(free)) % cap] = order[at:]
    return ctx, new, table, ring, (head, free)


@pytest.mark.parametrize("inplace", [True, False])
@pytest.mark.parametrize("requests,page,kv_hi,prompt_hi,free,cut,pad",
                         [(1, 16, 0, 1, 1, 0, 0), (1, 64, 100, 5000, 200, 0, 7), (7, 16, 40, 20, 30, 0, 1),
                          (64, 64, 8192, 1, 64, 0, 0), (513, 32, 600, 90, 2000, 0, 100), (1300, 16, 300, 30, 5000, 0, 333),
                          (40, 16, 200, 100, 25, 0, 5),           # the ring runs dry
                          (40, 16, 200, 100, 400, 4, 5),          # some requests are too long for the table
                          (40, 128, 1, 300, 100, 0, -500)])       # the token buffers are too short
def test_plan(requests, page, kv_hi, prompt_hi, free, cut, pad, inplace):
    logq = lib()
    rng = np.random.default_rng(requests * 31 + page + cut)
    ctx, new, table, ring, state = make_plan(rng, requests, page, kv_hi, prompt_hi, free, cut)
    max_tokens = max(0, int(np.maximum(new, 0).sum()) + pad)
    want = plan_ref(ctx.tolist(), new.tolist(), table, ring, state, page, max_tokens)
    got = run_plan(logq, ctx, new, table, ring, state, page, max_tokens, inplace)
    for name, x, y in zip(("q_start", "kv_len", "positions", "slots", "block_table", "ring", "ring_state"), got, want):
        np.testing.assert_array_equal(x, np.asarray(y), err_msg=name)


def test_plan_empty_and_zero_lengths():
    logq = lib()
    got = run_plan(logq, [], [], np.zeros((0, 3)), [5, 6], (1, 2), 16, 4, True)
    assert got[0].tolist() == [0] and got[2].tolist() == [-1] * 4 and got[3].tolist() == [-1] * 4 and got[6].tolist() == [1, 2]
    # nothing new: lengths stay, no page is taken; a negative length is refused
    got = run_plan(logq, [16, 0, -3], [0, 0, 2], [[1], [-1], [-1]], [5, 6], (0, 2), 16, 2, False)
    assert got[0].tolist() == [0, 0, 0, 2] and got[1].tolist() == [16, 0, 0]
    assert got[3].tolist() == [-1, -1] and got[6].tolist() == [0, 2]


# ------------------------------------------------------------------ append ---

@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("d,heads,page,tokens,extra", [(128, 8, 64, 1, 0), (64, 8, 16, 37, 512), (128, 1, 32, 5, 8),
                                                       (64, 3, 16, 130, 0), (128, 8, 128, 1000, 4096), (64, 1, 1024, 1, 64)])
@pytest.mark.parametrize("values", [True, False])
def test_append(dtype, d, heads, page, tokens, extra, values):
    logq = lib()
    gen = torch.Generator().manual_seed(tokens * d + heads)
    cache = logq.new_kv_cache(up(tokens, page) + 3, page, heads, d, dtype, KB, VB)
    for x in (cache.k_codes, cache.v_codes):
        x.fill_(0xA5)
    for x in (cache.k_range, cache.v_range):
        x.fill_(3.0)
    wide = heads * d + extra
    kv = torch.randn(2, tokens, wide, generator=gen) * torch.exp(2 * torch.randn(2, tokens, 1, generator=gen))
    kv = kv.to(dtype)
    kv[:, ::5, :d] = 0                                     # zero vectors
    kv[0, tokens // 2, 0] = -0.0
    if tokens > 4:
        kv[0, 1, 3], kv[1, 2, 5], kv[0, 3, 0] = math.nan, math.inf, -math.inf
        kv[0, 4, :d] = torch.linspace(-1, 1, d).to(dtype)
        kv[1, 4, :d] = 2.0 ** -20                          # all at the range; subnormal in fp16
    if tokens > 8:
        kv[0, 6], kv[1, 7] = kv[0, 6] * 2.0 ** -14, kv[1, 7] * 2.0 ** -130   # subnormal in fp16, in bf16
    x = kv.cuda()
    k, v = (x[i, :, extra // 16 * 8:extra // 16 * 8 + heads * d].view(tokens, heads, d) for i in range(2))
    slots = torch.randperm(cache.pages * page, generator=gen)[:tokens].cuda()
    slots[1::7] = -1
    slots[3::11] = cache.pages * page                      # just beyond the cache
    before = [t.clone() for t in (cache.k_codes, cache.k_range, cache.v_codes, cache.v_range)]
    got = logq.logq_kv_append(cache, k, v, slots, values=values)
    assert (got is None) != values
    s = slots.cpu()
    live = (s >= 0) & (s < cache.pages * page)
    for i, (src, base, codes, ranges) in enumerate(((k, KB, cache.k_codes, cache.k_range), (v, VB, cache.v_codes, cache.v_range))):
        want_c, want_r, want_v = quantise_ref(src, base)
        c0, r0 = before[2 * i].cpu(), before[2 * i + 1].cpu()
        c0[s[live] // page, :, s[live] % page] = want_c[live]
        r0[s[live] // page, :, s[live] % page] = want_r[live]
        assert torch.equal(codes.cpu(), c0)
        assert torch.equal(ranges.cpu().isnan(), r0.isnan())
        assert torch.equal(ranges.cpu().nan_to_num(), r0.nan_to_num())
        if values:
            assert torch.equal(got[i].cpu().isnan(), want_v.isnan())
            assert torch.equal(got[i].cpu().nan_to_num().double(), want_v.to(dtype).nan_to_num().double())


# --------------------------------------------------------------- attention ---

def filled(logq, pages, page, heads, d, dtype, seed, v_scale=1.0):
    """A cache whose every slot holds something, some of it large."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    cache = logq.new_kv_cache(pages, page, heads, d, dtype, KB, VB)
    n = pages * page
    x = torch.randn(2, n, heads, d, generator=gen, device="cuda")
    x[1] *= v_scale * torch.exp(torch.randn(n, heads, 1, generator=gen, device="cuda"))
    x.clamp_(-60000, 60000)                                # finite in fp16
    logq.logq_kv_append(cache, x[0].to(dtype), x[1].to(dtype), torch.arange(n, device="cuda"))
    return cache, gen


def attend(logq, cache, gen, q_lens, kv_lens, hq, window=0, scale=None, max_q=None, extra_width=1, poison=True,
           q_scale=1.5):
    page, d = cache.page_size, cache.head_dim
    n = len(q_lens)
    counts = [up(m, page) for m in kv_lens]
    width = max(counts) + extra_width
    order = torch.randperm(cache.pages, generator=gen, device="cuda").to(torch.int32)
    assert sum(counts) <= cache.pages
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for r, c in enumerate(counts):
        table[r, :c] = order[at:at + c]
        if poison and kv_lens[r] % page:                   # what lies behind the last token may be anything
            last = int(order[at + c - 1])
            for x in (cache.k_range, cache.v_range):
                x[last, :, kv_lens[r] % page:] = math.nan
                x[last, :, page - 1] = math.inf
        at += c
    q_start = i32(np.concatenate([[0], np.cumsum(q_lens)]))
    wide = torch.randn(sum(q_lens), (hq + 3) * d, generator=gen, device="cuda") * q_scale
    q = wide.to(cache.dtype)[:, d:(hq + 1) * d].view(-1, hq, d)
    kv = i32(kv_lens)
    ws = logq.new_kv_workspace(hq, cache.heads, d)
    args = dict(scale=scale, window=window, max_q=max(q_lens) if max_q is None else max_q, workspace=ws)
    out = logq.logq_kv_attention(cache, q, q_start, kv, table, **args)
    again = logq.logq_kv_attention(cache, q, q_start, kv, table, **args)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))     # the same call, the same bits
    assert int(ws[:256 + 4096].sum()) == 0                 # no error, every arrival count back at zero
    ref, bound = attention_ref(cache, q, q_start.tolist(), kv_lens, table, d ** -0.5 if scale is None else scale,
                               window, KB, VB)
    return out, ref, bound


ATTEND = [
    # q_lens, kv_lens, hq, heads, page, window
    ([1], [1], 4, 1, 16, 0),
    ([1], [4001], 32, 8, 64, 0),
    ([1] * 9, [1, 15, 16, 17, 255, 256, 257, 1000, 63], 8, 2, 16, 0),
    ([1, 1, 1], [0, 5, 0], 8, 2, 32, 0),                   # requests without keys: rows of zeros
    ([3, 0, 2, 1], [3, 40, 1, 0], 8, 2, 16, 0),            # more queries than keys, no queries, neither
    ([5] * 4, [300, 5, 77, 1025], 32, 8, 16, 0),
    ([2, 7, 1], [2, 700, 33], 28, 4, 128, 0),              # 7 query heads a kv head
    ([33], [133], 16, 16, 64, 0),
    ([200, 1, 63], [200, 190, 500], 8, 2, 64, 0),
    ([65, 130], [65, 400], 5, 5, 32, 20),
    ([1, 1], [900, 130], 8, 2, 16, 100),
    ([40], [300], 40, 1, 16, 1),                           # each query sees its own key alone; 40 heads share one
    ([300], [300], 6, 2, 1024, 77),
]


@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", ATTEND, ids=lambda c: f"q{c[0][0]}x{len(c[0])}-kv{c[1][-1]}-h{c[2]}-{c[3]}-p{c[4]}-w{c[5]}")
def test_attention(case, d, dtype):
    logq = lib()
    q_lens, kv_lens, hq, heads, page, window = case
    cache, gen = filled(logq, sum(up(m, page) for m in kv_lens) + 2, page, heads, d, dtype, len(q_lens) + d)
    check_attention(*attend(logq, cache, gen, q_lens, kv_lens, hq, window))


@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("q_lens,kv_lens,max_q", [([1, 20, 150], [70, 20, 400], 1), ([1, 20, 150], [70, 20, 400], 100000),
                                                  ([1, 2], [70, 20], 100000)])
def test_attention_max_q_is_only_a_hint(q_lens, kv_lens, max_q, dtype):
    logq = lib()
    cache, gen = filled(logq, 20, 64, 2, 128, dtype, 5)
    check_attention(*attend(logq, cache, gen, q_lens, kv_lens, 8, max_q=max_q))


@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("scale,q_scale,v_scale", [(0.0, 1.0, 1.0), (1.0, 3.0, 1.0), (-0.3, 1.0, 1.0), (0.1, 1.0, 1e-6),
                                                   (0.1, 1.0, 700.0)])
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1], [333, 2000]), ([150], [500])])
def test_attention_scales(scale, q_scale, v_scale, q_lens, kv_lens, dtype):
    """Flat and sharp softmax, negative scale, values near the ends of fp16's range."""
    logq = lib()
    cache, gen = filled(logq, 40, 64, 2, 128, dtype, 9, v_scale)
    if dtype == FH:
        assert cache.v_range.isfinite().all()
    check_attention(*attend(logq, cache, gen, q_lens, kv_lens, 8, scale=scale, q_scale=q_scale))


@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1], [100, 333]), ([150, 3], [300, 40])])
def test_attention_nan_reaches_only_who_sees_it(q_lens, kv_lens):
    logq = lib()
    cache, gen = filled(logq, 24, 32, 2, 64, BF, 3)
    n = len(q_lens)
    table = torch.arange(24, dtype=torch.int32, device="cuda").view(n, 12)
    # key 60 of the second request's head 1, and key 120 of the first's head 0
    cache.k_range[int(table[1, 1]), 1, 38 - 32] = math.nan
    q = torch.randn(sum(q_lens), 8, 64, generator=gen, device="cuda").to(BF)
    q_start = i32(np.concatenate([[0], np.cumsum(q_lens)]))
    out = logq.logq_kv_attention(cache, q, q_start, i32(kv_lens), table, max_q=max(q_lens))
    first = q_lens[0]
    assert not out[:first].isnan().any() and not out[first:, :4].isnan().any()
    pos = torch.arange(kv_lens[1] - q_lens[1], kv_lens[1], device="cuda")
    assert torch.equal(out[first:, 4:].isnan().all(-1).all(-1), pos >= 38)
    assert torch.equal(out[first:, 4:].isnan().any(-1).any(-1), pos >= 38)


@pytest.mark.parametrize("q_lens,kv_lens", [([1], [200]), ([140], [200])])
def test_attention_missing_pages_and_long_lengths(q_lens, kv_lens):
    """Table entries outside the cache hide their keys; a length beyond the table ends at the table."""
    logq = lib()
    cache, gen = filled(logq, 8, 32, 2, 128, FH, 4)
    table = i32([[3, 8, 5, -1, 0, 1, 2147483647]])
    q = torch.randn(sum(q_lens), 4, 128, generator=gen, device="cuda").to(FH)
    q_start = i32([0, q_lens[0]])
    for kv in (kv_lens[0], 230, 100000):
        for window in (0, 64):
            out = logq.logq_kv_attention(cache, q, q_start, i32([kv]), table, window=window, max_q=q_lens[0])
            check_attention(out, *attention_ref(cache, q, q_start.tolist(), [kv], table, 128 ** -0.5, window, KB, VB))


def test_attention_leaves_other_rows_alone():
    logq = lib()
    cache, gen = filled(logq, 8, 32, 2, 64, BF, 4)
    q = torch.randn(20, 4, 64, generator=gen, device="cuda").to(BF)
    out = torch.full_like(q, 7.0)
    logq.logq_kv_attention(cache, q, i32([2, 5, 5, 14]), i32([40, 9, 60]), i32([[0, 1], [2, 3], [4, 5]]), out=out)
    assert (out[:2] == 7).all() and (out[14:] == 7).all() and not (out[2:14] == 7).all(-1).any()


def test_attention_offsets_beyond_32_bits():
    """Codes of more than 4 GB: the last pages are read where they are."""
    logq = lib()
    pages, page, heads, d = 9000, 1024, 8, 128
    codes = [torch.empty(pages, heads, page, d // 2, dtype=torch.uint8, device="cuda") for _ in range(2)]
    ranges = [torch.empty(pages, heads, page, dtype=BF, device="cuda") for _ in range(2)]
    assert codes[0].numel() > 2 ** 32
    cache = logq.KVCache(codes[0], ranges[0], codes[1], ranges[1], logq.logq_build_codebook(4, KB, 1.0),
                         logq.logq_build_codebook(4, VB, 1.0))
    gen = torch.Generator(device="cuda").manual_seed(1)
    n = 1500
    table = i32([[8999, 8997]])
    pos = torch.arange(n, device="cuda")
    slots = table[0, pos // page].long() * page + pos % page
    k, v = torch.randn(2, n, heads, d, generator=gen, device="cuda").to(BF).unbind(0)
    logq.logq_kv_append(cache, k, v, slots)
    for nq in (1, 130):
        q = torch.randn(nq, 32, d, generator=gen, device="cuda").to(BF)
        out = logq.logq_kv_attention(cache, q, i32([0, nq]), i32([n]), table, max_q=nq)
        check_attention(out, *attention_ref(cache, q, [0, nq], [n], table, d ** -0.5, 0, KB, VB))


def test_step_on_another_stream_and_in_a_graph():
    """plan -> append -> attention on a side stream, then captured and replayed on new inputs."""
    logq = lib()
    heads, hq, d, page = 2, 8, 64, 16
    side = torch.cuda.Stream()
    cache = logq.new_kv_cache(64, page, heads, d, BF, KB, VB)
    ctx, new = i32([0, 0, 0]), i32([20, 1, 33])
    table, ring, state = i32(np.full((3, 8), -1)), i32(np.arange(64)), i32([0, 64])
    ws, aws = logq.new_workspace(), logq.new_kv_workspace(hq, heads, d)
    gen = torch.Generator(device="cuda").manual_seed(2)
    qkv = torch.randn(54, (hq + 2 * heads) * d, generator=gen, device="cuda").to(BF)
    out = torch.zeros(54, hq, d, dtype=BF, device="cuda")

    def step():
        q_start, kv_len, _, slots, _ = logq.logq_kv_plan(ctx, new, table, ring, state, page, 54, workspace=ws)
        q, k, v = qkv.split([hq * d, heads * d, heads * d], 1)
        logq.logq_kv_append(cache, k.view(54, heads, d), v.view(54, heads, d), slots)
        logq.logq_kv_attention(cache, q.view(54, hq, d), q_start, kv_len, table, out=out, workspace=aws)
        return q_start, kv_len

    def check(q_start, kv_len):
        torch.cuda.synchronize()
        check_attention(out, *attention_ref(cache, qkv[:, :hq * d].view(54, hq, d), q_start.tolist(), kv_len.tolist(),
                                            table, d ** -0.5, 0, KB, VB))

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    check(*got)
    assert got[1].tolist() == [20, 1, 33] and state.tolist() == [6, 58]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step()
    for _ in range(2):
        ctx.copy_(ctx + new)
        new.copy_(i32([1, 1, 1]) if _ else i32([17, 3, 2]))
        qkv.copy_(torch.randn(qkv.shape, generator=gen, device="cuda"))
        out.zero_()
        graph.replay()
        check(*got)
    assert got[1].tolist() == [38, 5, 36]


def test_example_layer():
    """The example's layer: every step's attention against 64 bits over what its cache holds."""
    import os
    import sys
    lib()
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import paged_decode

    seen = []

    def check(layer, q, out, q_start, kv_len, table):
        check_attention(out, *attention_ref(layer.cache, q, q_start.tolist(), kv_len.tolist(), table,
                                            layer.DIM ** -0.5, 0, 1.5, 1.5))
        seen.append(kv_len.tolist())

    y, ctx, layer = paged_decode.run(steps=6, check=check)
    assert y.isfinite().all() and seen[0] == [40, 3, 117, 64]
    assert ctx.tolist() == [25 + 2, 3 + 6, 117 + 6, 64 + 6]
    held = sum(up(n, 16) for n in ctx.tolist())
    assert int(layer.ring_state[1]) == layer.cache.pages - held
    # every page is either held once or free once
    free = layer.ring[(int(layer.ring_state[0]) + torch.arange(int(layer.ring_state[1]), device="cuda")) % layer.ring.numel()]
    used = torch.cat([t[:up(n, 16)] for t, n in zip(layer.block_table, ctx.tolist())])
    assert torch.equal(torch.cat([free, used]).sort().values, torch.arange(layer.cache.pages, dtype=torch.int32, device="cuda"))



def test_empty_calls():
    logq = lib()
    cache = logq.new_kv_cache(4, 16, 2, 64, BF)
    none = torch.empty(0, 2, 64, dtype=BF, device="cuda")
    assert logq.logq_kv_append(cache, none, none, torch.empty(0, dtype=torch.int64, device="cuda")) is None
    q = torch.empty(0, 4, 64, dtype=BF, device="cuda")
    assert logq.logq_kv_attention(cache, q, i32([0, 0]), i32([7]), i32([[0]])).shape == (0, 4, 64)
    q = torch.ones(3, 4, 64, dtype=BF, device="cuda")
    out = torch.full_like(q, 5.0)
    logq.logq_kv_attention(cache, q, i32([0]), i32([]), torch.empty(0, 1, dtype=torch.int32, device="cuda"), out=out)
    assert (out == 5).all()


@pytest.mark.parametrize("tokens", [10, 300])
def test_attention_odd_bounds(tokens):
    """Bounds that do not ascend or leave the tokens are cut to them; a negative length is none."""
    logq = lib()
    cache, gen = filled(logq, 16, 32, 2, 64, FH, 6)
    table = torch.arange(16, dtype=torch.int32, device="cuda").view(4, 4)
    q = torch.randn(tokens, 4, 64, generator=gen, device="cuda").to(FH)
    q_start, kv = [tokens // 2, 2, -7, tokens - 1, 10 ** 6], [100, -5, 128, 90]
    # requests: none (from the middle back to 2), none, tokens 0 .. n - 2, the last token
    out = torch.full_like(q, 5.0)
    logq.logq_kv_attention(cache, q, i32(q_start), i32(kv), table, out=out)
    check_attention(out, *attention_ref(cache, q, [tokens, tokens, 0, tokens - 1, tokens], [100, 0, 128, 90], table,
                                        64 ** -0.5, 0, KB, VB))


@pytest.mark.parametrize("heavy", [150, 9, 1])
def test_attention_of_many_requests(heavy):
    """More requests than a CTA has threads: the scans over them go round."""
    logq = lib()
    q_lens, kv_lens = [1] * 700, [1 + (7 * i) % 40 for i in range(700)]
    for i in (0, 300, 699):
        q_lens[i], kv_lens[i] = heavy, heavy + 90
    q_lens[5] = 0
    cache, gen = filled(logq, sum(up(m, 16) for m in kv_lens), 16, 2, 64, BF, 8)
    check_attention(*attend(logq, cache, gen, q_lens, kv_lens, 8))


def test_stream_argument_orders_a_calls_own_tensors():
    """With stream=, what a call makes for itself is made there: its workspace's zero-fill comes before
    the kernels, and its memory is not given to the current stream while they run."""
    logq = lib()
    cache, gen = filled(logq, 64, 64, 8, 128, BF, 12)
    side = torch.cuda.Stream()
    q = torch.randn(300, 32, 128, generator=gen, device="cuda").to(BF)
    table = torch.arange(64, dtype=torch.int32, device="cuda").view(1, 64)
    q_start, kv = i32([0, 300]), i32([4000])
    ref, bound = attention_ref(cache, q, [0, 300], [4000], table, 128 ** -0.5, 0, KB, VB)
    torch.cuda.synchronize()
    need = logq.logq_kv_attention_workspace_bytes(32, 8, 128)
    for _ in range(3):
        dirty = torch.full((need,), 255, dtype=torch.uint8, device="cuda")         # what the allocator has at hand
        del dirty
        out = logq.logq_kv_attention(cache, q, q_start, kv, table, max_q=300, stream=side)
        other = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        side.synchronize()
        check_attention(out, ref, bound)
        del other


@pytest.mark.parametrize("hq,heads", [(8, 2), (2, 2)])
@pytest.mark.parametrize("window", [1, 63, 64, 200])
def test_attention_windows_narrower_than_a_tile_of_rows(window, hq, heads):
    """Some warps of a row tile see none of a key tile that others see, before and after their own."""
    logq = lib()
    q_lens, kv_lens = [700, 300], [700, 1111]
    cache, gen = filled(logq, sum(up(m, 16) for m in kv_lens), 16, heads, 64, BF, 21)
    check_attention(*attend(logq, cache, gen, q_lens, kv_lens, hq, window=window))


@pytest.mark.parametrize("lens", [[40, 0, 3], [1, 1, 200], [0, 0, 0], [200, 200, 200]])
def test_attention_lengths_below_equal_bounds(lens):
    """max_q * requests = tokens leaves no room for unequal lengths, but the device's may be shorter."""
    logq = lib()
    tokens, kv = 600, [500, 64, 333]
    cache, gen = filled(logq, 64, 16, 2, 128, BF, 23)
    q = torch.randn(tokens, 8, 128, generator=gen, device="cuda").to(BF)
    table = torch.arange(96, dtype=torch.int32, device="cuda").view(3, 32) % 64
    starts = [0, lens[0], lens[0] + lens[1], sum(lens)]
    out = torch.full_like(q, 5.0)
    logq.logq_kv_attention(cache, q, i32(starts), i32(kv), table, max_q=200, out=out)
    if sum(lens):
        ref = attention_ref(cache, q, starts, kv, table, 128 ** -0.5, 0, KB, VB)
        check_attention(out[:sum(lens)], *[x[:sum(lens)] for x in ref])
    assert (out[sum(lens):] == 5.0).all()
