// The paged 4-bit key/value cache: a step's bookkeeping from the requests'
// lengths (block tables, slot map, positions) and the quantisation of its keys
// and values into their slots.
//
// Bookkeeping (plan_kernel).  With n_r = max(new_r, 0):
//   q_start = exclusive sum of n_r;  need_r = ceil((ctx_r + n_r) / P) - ceil(ctx_r / P)
//   new page i of request r = ring[(head + sum_{s < r} need_s + i) mod ring_size]
//   slot of position p = page[p / P] * P + p mod P
// It is bound by latency: a 64-request step moves 2 KB.  So it is one launch
// whose CTAs do not wait for one another: every CTA repeats the scans over the
// requests (8 bytes a request, from L2) and then serves its own slice of the
// tokens and its own share of the ended requests.
//
// Quantisation (append_kernel).  range = max|x|, m = #{ j < 7 : |x| >= fl32(thresh[j] * range) }:
// read once, written once.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>
#include <string.h>

#include "internal.h"
#include "kv_cache.h"

namespace logq {
namespace {

constexpr int kPlanThreads = 512;
constexpr int kPlanSlice = 1024;         // tokens per CTA
constexpr int kPlanWarps = kPlanThreads / 32;

// Inclusive sum over the block; *total is the block's sum.
__device__ __forceinline__ long long block_scan(long long v, long long* warp_sums, long long* total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
    }
    __syncthreads();                     // the previous call's sums are read
    if (lane == 31) warp_sums[warp] = v;
    __syncthreads();
    long long before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kPlanWarps; ++w) {
        const long long s = warp_sums[w];
        before += w < warp ? s : 0;
        all += s;
    }
    *total = all;
    return v + before;
}

// What a token needs to know of its request, kept at the request's first token in the slice.
struct Mark {
    int32_t r, ctx, end, first, ok;      // request, cached tokens, q_start[r + 1], its first new page's rank
    int32_t q0;
};

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const __grid_constant__ KvPlanParams p)
{
    __shared__ long long warp_sums[kPlanWarps];
    __shared__ int32_t mark_at[kPlanSlice];
    __shared__ Mark marks[kPlanSlice];
    __shared__ int32_t ended_r[kPlanThreads];
    __shared__ long long ended_to[kPlanThreads];
    __shared__ int n_ended;
    __shared__ int32_t warp_last[kPlanWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long t0 = (long long)blockIdx.x * kPlanSlice;
    const long long t1 = t0 + kPlanSlice < p.max_tokens ? t0 + kPlanSlice : p.max_tokens;
    const bool first_cta = blockIdx.x == 0;
    const int P = p.page_size, shift = p.page_shift;

    const long long cap = p.ring_size;
    long long head = p.ring_state[0], count = p.ring_state[1];
    head = ((head % cap) + cap) % cap;
    count = count < 0 ? 0 : count > cap ? cap : count;

    for (int k = tid; k < kPlanSlice; k += kPlanThreads) mark_at[k] = -1;
    long long tokens_before = 0, need_before = 0, freed_before = 0;
    long long taken = 0;                 // pages of admitted requests
    for (long long base = 0; base < p.requests; base += kPlanThreads) {
        if (tid == 0) n_ended = 0;       // block_scan's barriers order this
        const long long r = base + tid;
        const bool have = r < p.requests;
        const long long ctx = have ? p.ctx_len[r] : 0, raw = have ? p.new_len[r] : 0;
        const long long n = raw > 0 ? raw : 0;
        const long long old = ctx > 0 ? (ctx + P - 1) >> shift : 0;
        const long long held = old < p.table_width ? old : p.table_width;
        long long all;
        const long long q1 = tokens_before + block_scan(n, warp_sums, &all), q0 = q1 - n;
        tokens_before += all;
        const long long want = (ctx + n + P - 1) >> shift;
        bool ok = have && raw >= 0 && ctx >= 0 && ctx + n <= 0x7fffffffll && want <= p.table_width && q1 <= p.max_tokens;
        const long long need = ok ? want - old : 0;
        const long long first = need_before + block_scan(need, warp_sums, &all) - need;
        need_before += all;
        ok = ok && (need == 0 || first + need <= count);
        // admitted requests that take pages are a prefix of those that want any
        if (ok && need > 0) taken = first + need;
        const bool ended = have && raw < 0;
        const long long freed = ended ? held : 0;
        const long long to = freed_before + block_scan(freed, warp_sums, &all) - freed;
        freed_before += all;
        if (have && first_cta) {
            p.q_start[r] = (int32_t)(q0 < p.max_tokens ? q0 : p.max_tokens);
            p.kv_len[r] = ok ? (int32_t)(ctx + n) : 0;
        }
        if (n > 0 && q0 < t1 && q1 > t0) {
            const int k = (int)((q0 > t0 ? q0 : t0) - t0);
            mark_at[k] = k;
            marks[k] = Mark{(int32_t)r, (int32_t)ctx, (int32_t)(q1 < t1 ? q1 : t1), (int32_t)(ok ? first : 0), ok ? 1 : 0,
                            (int32_t)q0};
        }
        if (ended && freed > 0 && r % gridDim.x == blockIdx.x) {
            const int i = atomicAdd(&n_ended, 1);       // order among them does not matter
            ended_r[i] = tid;
            ended_to[i] = to;
        }
        __syncthreads();
        // the pages of ended requests go behind the ring's tail
        for (int i = 0; i < n_ended; ++i) {
            const long long rr = base + ended_r[i], at = ended_to[i];
            const long long c = p.ctx_len[rr], o = (c + P - 1) >> shift;
            const long long m = o < p.table_width ? o : p.table_width;
            for (long long j = tid; j < m; j += kPlanThreads)
                if (count + at + j < cap) p.ring[(head + count + at + j) % cap] = p.block_table[rr * p.table_width + j];
        }
        __syncthreads();
    }

    if (first_cta && tid == 0)
        p.q_start[p.requests] = (int32_t)(tokens_before < p.max_tokens ? tokens_before : p.max_tokens);

    // this CTA's tokens: the last mark at or before each
    int last[kPlanSlice / kPlanThreads];
    {
        const int k0 = tid * (kPlanSlice / kPlanThreads);
        int m = -1;
#pragma unroll
        for (int i = 0; i < kPlanSlice / kPlanThreads; ++i) {
            const int v = mark_at[k0 + i];
            m = v > m ? v : m;
            last[i] = m;
        }
        int incl = m;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o && u > incl) incl = u;
        }
        if (lane == 31) warp_last[warp] = incl;
        __syncthreads();
        int before = __shfl_up_sync(0xffffffffu, incl, 1);
        if (lane == 0) before = -1;
        for (int w = 0; w < warp; ++w) before = warp_last[w] > before ? warp_last[w] : before;
#pragma unroll
        for (int i = 0; i < kPlanSlice / kPlanThreads; ++i) last[i] = last[i] < 0 ? before : last[i];
    }
#pragma unroll
    for (int i = 0; i < kPlanSlice / kPlanThreads; ++i) {
        const long long t = t0 + tid * (kPlanSlice / kPlanThreads) + i;
        if (t >= t1) continue;
        int32_t pos = -1;
        long long slot = -1;
        if (last[i] >= 0) {
            const Mark m = marks[last[i]];
            if (t < m.end && m.ok) {
                pos = m.ctx + (int32_t)(t - m.q0);
                const int32_t page_i = pos >> shift, off = pos & (P - 1);
                const int32_t old = (m.ctx + P - 1) >> shift;
                int32_t page;
                if (page_i < old) {
                    page = p.block_table[(long long)m.r * p.table_width + page_i];
                } else {
                    page = p.ring[(head + m.first + (page_i - old)) % cap];
                    // each new page has one first token among the new ones
                    if (off == 0) p.block_table[(long long)m.r * p.table_width + page_i] = page;
                }
                slot = (long long)page * P + off;
            }
        }
        p.positions[t] = pos;
        p.slots[t] = slot;
    }

    // The ring's new state.  In place, only the last CTA to arrive may write it:
    // the others have read the old one by then.
    __shared__ long long taken_max[kPlanWarps];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const long long u = __shfl_xor_sync(0xffffffffu, taken, o);
        taken = u > taken ? u : taken;
    }
    if (lane == 0) taken_max[warp] = taken;
    __syncthreads();
    if (tid == 0) {
        for (int w = 0; w < kPlanWarps; ++w) taken = taken_max[w] > taken ? taken_max[w] : taken;
        bool write = first_cta;
        if (p.ws) {
            __threadfence();
            write = atomicInc(&p.ws->ticket, gridDim.x - 1) == gridDim.x - 1;    // wraps to 0
        }
        if (write) {
            const long long full = count + freed_before < cap ? count + freed_before : cap;
            p.ring_state_out[0] = (int32_t)((head + taken) % cap);
            p.ring_state_out[1] = (int32_t)(full - taken);
        }
    }
}

// ------------------------------------------------------------------ append ---

constexpr int kAppendThreads = 256;

template <bool F16>
__device__ __forceinline__ float to_float(uint32_t b)
{
    if constexpr (F16) return __half2float(__ushort_as_half((unsigned short)b));
    else return __uint_as_float(b << 16);
}

template <bool F16>
__device__ __forceinline__ uint32_t to_bits(float v)
{
    if constexpr (F16) return __half_as_ushort(__float2half_rn(v));
    else return __bfloat16_as_ushort(__float2bfloat16_rn(v));
}

// 16 dimensions per thread, D / 16 neighbouring lanes per vector; vector index =
// ((token * 2 + {k, v}) * heads + head), so that a token's reads and writes are
// contiguous runs.
template <int D, bool F16>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const __grid_constant__ KvAppendParams p)
{
    constexpr int kLanes = D / 16;
    __shared__ float level[2][16];
    if (threadIdx.x < 32) {
        const int i = threadIdx.x;
        level[i >> 4][i & 15] = to_float<F16>(p.lvl16[i >> 4][i & 15]);
    }
    __syncthreads();
    const long long vectors = p.tokens * 2 * p.heads;
    const long long per = (long long)gridDim.x * (kAppendThreads / kLanes);
    const int part = threadIdx.x % kLanes;
    const long long page_vecs = (long long)p.heads * p.page_size;
    // every lane of a warp stays in the loop while one of them has a vector: the shuffles need them all
    const long long begin = (long long)blockIdx.x * (kAppendThreads / kLanes) + threadIdx.x / kLanes;
    const long long warp_begin = begin - (threadIdx.x % 32) / kLanes;
    for (long long w = 0; warp_begin + w < vectors; w += per) {
        const long long i = begin + w;
        const bool live = i < vectors;
        const int head = live ? (int)(i % p.heads) : 0;
        const long long tv = live ? i / p.heads : 0;
        const int which = (int)(tv & 1);
        const long long token = tv >> 1;
        uint32_t x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (live) {
            const uint16_t* src = (which ? p.v + token * p.v_stride : p.k + token * p.k_stride) + (long long)head * D + part * 16;
            const uint4 a = __ldg(reinterpret_cast<const uint4*>(src));
            const uint4 b = __ldg(reinterpret_cast<const uint4*>(src) + 1);
            x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
            x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        }
        // magnitudes order like their bit patterns; NaN and Inf lie above all finite ones
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t lo = x[j] & 0x7fffu, hi = (x[j] >> 16) & 0x7fffu;
            top = max(top, max(lo, hi));
        }
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        const bool bad = top >= (F16 ? 0x7c00u : 0x7f80u);
        const float range = to_float<F16>(top);
        float bound[7];
#pragma unroll
        for (int j = 0; j < 7; ++j) bound[j] = p.thresh[which][j] * range;
        uint32_t code[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const uint32_t b = (j & 1) ? x[j >> 1] >> 16 : x[j >> 1] & 0xffffu;
            const float a = to_float<F16>(b & 0x7fffu);
            uint32_t m = 0;
#pragma unroll
            for (int t = 0; t < 7; ++t) m += a >= bound[t] ? 1u : 0u;
            const uint32_t c = m | ((m && (b & 0x8000u)) ? 8u : 0u);
            code[j >> 3] |= c << (4 * (j & 7));
        }
        if (bad || top == 0) code[0] = code[1] = 0;
        if (!live) continue;             // after the shuffles
        const uint32_t range_bits = bad ? 0x7fffu : top;
        const long long slot = p.slots[token];
        if (slot >= 0 && slot < p.pages * p.page_size) {
            const long long page = slot >> p.page_shift, off = slot & (p.page_size - 1);
            const long long vec = page * page_vecs + (long long)head * p.page_size + off;
            uint8_t* codes = which ? p.v_codes : p.k_codes;
            *reinterpret_cast<uint2*>(codes + vec * (D / 2) + part * 8) = make_uint2(code[0], code[1]);
            if (part == 0) (which ? p.v_range : p.k_range)[vec] = (uint16_t)range_bits;
        }
        if (p.k_values) {
            uint32_t y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t two = 0;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int e = 2 * j + h;
                    const float v = level[which][(code[e >> 3] >> (4 * (e & 7))) & 15u] * range;
                    two |= (bad ? 0x7fffu : to_bits<F16>(v)) << (16 * h);
                }
                y[j] = two;
            }
            uint16_t* dst = (which ? p.v_values : p.k_values) + (token * p.heads + head) * D + part * 16;
            reinterpret_cast<uint4*>(dst)[0] = make_uint4(y[0], y[1], y[2], y[3]);
            reinterpret_cast<uint4*>(dst)[1] = make_uint4(y[4], y[5], y[6], y[7]);
        }
    }
}

template <int D, bool F16>
cudaError_t append_launch(const KvAppendParams& p, cudaStream_t s)
{
    const int sms = sm_count() > 0 ? sm_count() : 148;
    const long long vectors = p.tokens * 2 * p.heads;
    const long long per_cta = kAppendThreads / (D / 16);
    long long grid = (vectors + per_cta - 1) / per_cta;
    if (grid > (long long)sms * 8) grid = (long long)sms * 8;
    append_kernel<D, F16><<<(int)grid, kAppendThreads, 0, s>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv_plan(const KvPlanParams& p, cudaStream_t s)
{
    long long grid = (p.max_tokens + kPlanSlice - 1) / kPlanSlice;
    if (grid < 1) grid = 1;
    plan_kernel<<<(int)grid, kPlanThreads, 0, s>>>(p);
    return cudaGetLastError();
}

cudaError_t launch_kv_append(const KvAppendParams& p, int head_dim, bool f16, cudaStream_t s)
{
    if (head_dim == 128) return f16 ? append_launch<128, true>(p, s) : append_launch<128, false>(p, s);
    return f16 ? append_launch<64, true>(p, s) : append_launch<64, false>(p, s);
}

}  // namespace logq
