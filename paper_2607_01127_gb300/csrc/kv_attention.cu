// Attention over the paged 4-bit key/value cache.
//
//   s_j = scale * range_k[j] * (q . level_k[code_k[j]]),  out = sum_j softmax_j(s) range_v[j] level_v[code_v[j]]
//
// The queries of one request that read one kv head (its tokens x the query
// heads of the group) are the columns of a tile; keys and values are decoded
// once per tile of up to NC columns.  A (request, kv head, block of NC columns)
// is a segment; its keys are cut into steps of 16.
//
// Split.  All segments' steps form one line that the CTAs cut into equal
// pieces, so ragged batches balance and one long request uses the whole GPU.
// The lengths are on the device, so every CTA finds its piece by itself (a scan
// over the requests).  A segment that ends up in several CTAs is joined by the
// last of them to arrive, in the order of the keys: results do not depend on
// timing.
//
// Step (one warp, 16 keys).  S^T[16 keys x 8 queries] = K[16 x D] Q^T on
// mma.m16n8k16: with the keys on the 16 side a group of 4 query heads wastes
// half a tile, not three quarters.  The contraction order over D is free, so a
// lane takes contiguous codes: 16 bytes of a key row, each byte one lookup in
// the pair table -> a register of two 16-bit values.  Softmax without a running
// maximum across lanes: a reference value per column is raised (and O rescaled)
// only when a score exceeds it by 2^8, found by one vote per step; the sums stay
// per lane to the end.  O^T[D x 8] += V^T[D x 16] W^T with W = p * range_v in
// fp16; the two codes of a dimension at two neighbouring keys are brought into
// one byte first, so one lookup gives the (key, key + 1) pair that the MMA wants.
// The reference is a maximum of s + log2(range_v), so W never overflows fp16.
//
// Pair table.  As in the decode GEMV: 256 rows of 256 bytes, one copy per lane,
// keys' entries in the first half of a row and values' in the second; the
// offset of an entry is one byte permute.  256 codes (a key and a value) cost
// 128 lookups, 4 cycles of an SM's shared memory, below the 5.6 cycles that
// their 132 bytes take from HBM.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <limits.h>
#include <stdint.h>
#include <string.h>

#include "internal.h"
#include "kv_cache.h"
#include "kv_device.h"
#include "ptx.h"

namespace logq {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kStep = 16;                    // keys per warp step
constexpr int kMinChunk = kWarps;            // steps per CTA, at least
constexpr uint32_t kTabBytes = 256 * 256;

template <uint32_t OFF>
__device__ __forceinline__ uint32_t lds_tab(uint32_t off)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1+%2];" : "=r"(v) : "r"(off), "n"(kTabOff + OFF));
    return v;
}

template <bool F16>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1)
{
    if constexpr (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 8 x 8 matrix of 16-bit values, one row of pairs per four lanes, transposed across the warp.
__device__ __forceinline__ uint32_t transpose8(uint32_t v)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// floor(log2 r) of a range, kept within what the scaled weights and their sums can take.
__device__ __forceinline__ float range_exponent(float r)
{
    int e = (int)((__float_as_uint(r) >> 23) & 0xffu) - 127;
    e = e < -24 ? -24 : e > 100 ? 100 : e;
    return (float)e;
}

// One request's share of the line of steps.
struct Share : Request {
    int32_t lo_step;         // first step any of its tokens sees
    int32_t steps;           // steps per segment (at least one, so that empty rows are answered)
    int32_t blocks;          // segments per kv head (tokens x query heads fit 31 bits)
};

__device__ __forceinline__ Share load_share(const KvAttendParams& p, int64_t r, int nc)
{
    Share q;
    static_cast<Request&>(q) = load_request(p, r);
    const int64_t first = q.kv - q.n;
    int64_t lo = p.window > 0 ? first - p.window + 1 : 0;
    lo = lo < 0 ? 0 : lo;
    q.lo_step = (int32_t)(lo / kStep);
    const int64_t st = (q.hi + kStep - 1) / kStep - q.lo_step;
    q.steps = st < 1 ? 1 : (int32_t)st;
    if (st < 1) q.lo_step = 0;               // no key is seen: one step, hidden whole, inside the table
    const int64_t rows = (int64_t)q.n * p.group;
    q.blocks = rows > p.tile_rows ? 0 : (int32_t)((rows + nc - 1) / nc);
    return q;
}

__device__ __forceinline__ int64_t weight_of(const KvAttendParams& p, const Share& q)
{
    return (int64_t)q.blocks * p.heads * q.steps;
}

__device__ __forceinline__ int64_t warp_sum(int64_t v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The codes and ranges of one step as one lane needs them.
template <int D>
struct StepData {
    uint32_t k[2][D / 32];       // key rows g and g + 8: D / 4 codes from dimension (D / 4) * t
    uint32_t v[4][D / 64];       // key rows 2t, 2t + 1, 2t + 8, 2t + 9: D / 8 codes from dimension (D / 8) * g
    uint16_t kr[2], vr[2];       // ranges of keys g and g + 8
    bool bad;                    // the page does not exist
};

template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const uint8_t* p)
{
    if constexpr (N == 4) {
        asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
    } else if constexpr (N == 2) {
        asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
    } else {
        asm volatile("ld.global.nc.L1::no_allocate.u32 %0, [%1];" : "=r"(w[0]) : "l"(p));
    }
}

template <int D>
__device__ __forceinline__ void load_step(StepData<D>& s, const KvAttendParams& p, int head, int64_t kb, int32_t page,
                                          int g, int t)
{
    s.bad = page < 0 || page >= p.pages;
    const int64_t row = ((int64_t)(s.bad ? 0 : page) * p.heads + head) * p.page_size + (kb & (p.page_size - 1));
    const uint8_t* kc = p.k_codes + (row + g) * (D / 2) + t * (D / 8);
    load_words(s.k[0], kc);
    load_words(s.k[1], kc + 8 * (D / 2));
    const uint8_t* vc = p.v_codes + (row + 2 * t) * (D / 2) + g * (D / 16);
    load_words(s.v[0], vc);
    load_words(s.v[1], vc + D / 2);
    load_words(s.v[2], vc + 8 * (D / 2));
    load_words(s.v[3], vc + 9 * (D / 2));
    s.kr[0] = __ldg(p.k_range + row + g);
    s.kr[1] = __ldg(p.k_range + row + g + 8);
    s.vr[0] = __ldg(p.v_range + row + g);
    s.vr[1] = __ldg(p.v_range + row + g + 8);
}

template <int D, bool F16, int NT>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 2 : 1) attend_kernel(const __grid_constant__ KvAttendParams p)
{
    constexpr int NC = 8 * NT;
    constexpr int kOStride = D + 4;                  // floats per column of the merge buffer
    extern __shared__ __align__(1024) uint8_t smem[];
    // layout: pair table | merge buffer [warp][8 columns][D] | {reference, sum} [warp][NC] | scratch
    float* merge = reinterpret_cast<float*>(smem + kTabBytes);
    float2* stat = reinterpret_cast<float2*>(merge + kWarps * 8 * kOStride);
    int64_t* scratch = reinterpret_cast<int64_t*>(stat + kWarps * NC);      // [kWarps + 4]
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g = lane >> 2, t = lane & 3;

    // pair tables: two codes -> two 16-bit levels, keys then values in each row
    for (int i = tid; i < 256 * 16; i += kThreads) {
        const int e = i >> 4, part = i & 15;
        const uint16_t* lv = part < 8 ? p.k_lvl : p.v_lvl;
        const uint32_t v = (uint32_t)lv[e & 15] | ((uint32_t)lv[e >> 4] << 16);
        *reinterpret_cast<uint4*>(smem + e * 256 + part * 16) = make_uint4(v, v, v, v);
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // this CTA's piece [f, f_end) of the line, and the request it starts in
    int64_t total = 0;
    for (int64_t r = tid; r < p.requests; r += kThreads) total += weight_of(p, load_share(p, r, NC));
    total = warp_sum(total);
    if (lane == 0) scratch[warp] = total;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) total += scratch[w];
    int64_t chunk = (total + gridDim.x - 1) / gridDim.x;
    chunk = chunk < kMinChunk ? kMinChunk : chunk;
    int64_t f = (int64_t)blockIdx.x * chunk;
    const int64_t f_end = f + chunk < total ? f + chunk : total;
    if (f >= f_end) return;
    {
        int64_t before = 0;
        for (int64_t base = 0; base < p.requests; base += kThreads) {
            const int64_t r = base + tid;
            const int64_t w = r < p.requests ? weight_of(p, load_share(p, r, NC)) : 0;
            int64_t incl = w;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t u = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += u;
            }
            __syncthreads();
            if (lane == 31) scratch[warp] = incl;
            __syncthreads();
            int64_t all = 0;
#pragma unroll
            for (int x = 0; x < kWarps; ++x) {
                if (x < warp) incl += scratch[x];
                all += scratch[x];
            }
            const int64_t from = before + incl - w;
            if (w > 0 && from <= f && f < from + w) {
                scratch[kWarps] = r;
                scratch[kWarps + 1] = from;
            }
            before += all;
            if (f < before) break;               // the same for every thread
        }
        __syncthreads();
    }
    int64_t r = scratch[kWarps], line0 = scratch[kWarps + 1];
    Share rq = load_share(p, r, NC);

    const uint32_t lane4 = 4u * lane;
    uint32_t* counters = p.counters;
    float* parts = p.parts;

    while (f < f_end) {
        while (f >= line0 + weight_of(p, rq)) {      // next request that has queries
            line0 += weight_of(p, rq);
            rq = load_share(p, ++r, NC);
        }
        const int64_t seg = (f - line0) / rq.steps;
        const int64_t seg0 = line0 + seg * rq.steps, seg1 = seg0 + rq.steps;
        const int64_t end = f_end < seg1 ? f_end : seg1;
        const int head = (int)(seg / rq.blocks), block = (int)(seg % rq.blocks);
        const int sb = (int)(f - seg0), cnt = (int)(end - f);
        const int row0 = block * NC;                     // first query row (token * group + head in group)
        const int rows = rq.n * p.group - row0 < NC ? rq.n * p.group - row0 : NC;
        const int64_t first_pos = rq.kv - rq.n + row0 / p.group;
        const int64_t last_pos = rq.kv - rq.n + (row0 + rows - 1) / p.group;

        // ---------------- this warp's steps ----------------
        uint32_t qf[NT][D / 8];                          // Q^T fragments: D / 4 dimensions from (D / 4) * t
        int khi[NT][2], klo[NT][2];                      // keys columns 2t, 2t + 1 see
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = row0 + nt * 8 + g;
            const bool live = nt * 8 + g < rows;
            const uint16_t* src = p.q + (int64_t)(rq.q0 + row / p.group) * p.q_stride +
                                  (int64_t)(head * p.group + row % p.group) * D + t * (D / 4);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                uint4 x = make_uint4(0, 0, 0, 0);
                if (live) x = __ldg(reinterpret_cast<const uint4*>(src) + i);
                qf[nt][4 * i] = x.x; qf[nt][4 * i + 1] = x.y; qf[nt][4 * i + 2] = x.z; qf[nt][4 * i + 3] = x.w;
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int col = nt * 8 + 2 * t + c;
                const int64_t pos = rq.kv - rq.n + (row0 + col) / p.group;
                const bool has = col < rows;             // other columns' results are dropped
                int64_t hi = pos < rq.hi - 1 ? pos : rq.hi - 1;
                int64_t lo = p.window > 0 && pos - p.window + 1 > 0 ? pos - p.window + 1 : 0;
                khi[nt][c] = has ? (int)hi : INT_MAX;
                klo[nt][c] = has ? (int)lo : 0;
            }
        }
        // keys that every column sees: no mask needed between these
        const int64_t all_hi = first_pos < rq.hi - 1 ? first_pos : rq.hi - 1;
        const int64_t all_lo = p.window > 0 ? last_pos - p.window + 1 : 0;

        float o[NT][D / 16][4];
        float ref[NT][2], sum[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[nt][i][c] = 0.0f;
#pragma unroll
            for (int c = 0; c < 2; ++c) { ref[nt][c] = kRefInit; sum[nt][c] = 0.0f; }
        }

        const int s0 = sb + (int)((int64_t)cnt * warp / kWarps), s1 = sb + (int)((int64_t)cnt * (warp + 1) / kWarps);
        const int32_t* table = p.block_table + r * p.table_width;
        auto key_of = [&](int s) { return (int64_t)(rq.lo_step + s) * kStep; };
        auto page_of = [&](int s) {
            const int64_t kb = key_of(s < s1 ? s : s1 - 1);
            return __ldg(table + (kb >> p.page_shift));
        };
        StepData<D> next;
        int32_t page_next = 0;
        if (s0 < s1) {
            load_step<D>(next, p, head, key_of(s0), page_of(s0), g, t);
            page_next = page_of(s0 + 1);
        }
        for (int s = s0; s < s1; ++s) {
            const StepData<D> cur = next;
            if (s + 1 < s1) {
                load_step<D>(next, p, head, key_of(s + 1), page_next, g, t);
                page_next = page_of(s + 2);
            }
            const int64_t kb = key_of(s);

            // S^T = K Q^T
            float acc[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[nt][c] = 0.0f;
#pragma unroll
            for (int w = 0; w < D / 32; ++w) {
                uint32_t a[2][4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    a[h][0] = lds_tab<0>(prmt(cur.k[h][w], lane4, 0x7604u));
                    a[h][1] = lds_tab<0>(prmt(cur.k[h][w], lane4, 0x7614u));
                    a[h][2] = lds_tab<0>(prmt(cur.k[h][w], lane4, 0x7624u));
                    a[h][3] = lds_tab<0>(prmt(cur.k[h][w], lane4, 0x7634u));
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma16816<F16>(acc[nt], a[0][0], a[1][0], a[0][1], a[1][1], qf[nt][4 * w], qf[nt][4 * w + 1]);
                    mma16816<F16>(acc[nt], a[0][2], a[1][2], a[0][3], a[1][3], qf[nt][4 * w + 2], qf[nt][4 * w + 3]);
                }
            }

            // weights p = 2^(s - ref), and W = p * range_v in fp16
            const float ks[2] = {to_float<F16>(cur.kr[0]) * p.scale_log2, to_float<F16>(cur.kr[1]) * p.scale_log2};
            float vr[2] = {to_float<F16>(cur.vr[0]), to_float<F16>(cur.vr[1])};
            float ex[2] = {range_exponent(vr[0]), range_exponent(vr[1])};
            const bool masked = cur.bad || kb + kStep - 1 > all_hi || kb < all_lo;
            if (!masked) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[nt][c] *= ks[c >> 1];
            } else {
                // a hidden key's range may be anything, NaN included: its score and
                // its weight are replaced, not multiplied
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int64_t key = kb + g + 8 * (c >> 1);
                        const bool seen = !cur.bad && key <= khi[nt][c & 1] && key >= klo[nt][c & 1];
                        acc[nt][c] = seen ? acc[nt][c] * ks[c >> 1] : -INFINITY;
                    }
            }
            float high = -INFINITY;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 4; ++c) high = fmaxf(high, acc[nt][c] - ref[nt][c & 1] + ex[c >> 1]);
            if (__any_sync(0xffffffffu, high > kRaise)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float u = fmaxf(acc[nt][c] + ex[0], acc[nt][c + 2] + ex[1]);
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) u = fmaxf(u, __shfl_xor_sync(0xffffffffu, u, x));
                        const float to = fmaxf(ref[nt][c], u);
                        const float f0 = exp2_approx(ref[nt][c] - to);
                        ref[nt][c] = to;
                        sum[nt][c] *= f0;
#pragma unroll
                        for (int i = 0; i < D / 16; ++i) {
                            o[nt][i][c] *= f0;
                            o[nt][i][c + 2] *= f0;
                        }
                    }
            }
            uint32_t b[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float w[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float e = exp2_approx(acc[nt][c] - ref[nt][c & 1]);
                    sum[nt][c & 1] += e;
                    w[c] = e * vr[c >> 1];
                    if (masked && acc[nt][c] == -INFINITY) w[c] = 0.0f;
                }
                b[nt][0] = transpose8(pack2<true>(w[0], w[1]));
                b[nt][1] = transpose8(pack2<true>(w[2], w[3]));
            }

            // O^T += V^T W^T: dimensions (D / 8) g + 2i in rows g, + 1 in rows g + 8 of tile i
#pragma unroll
            for (int w = 0; w < D / 64; ++w) {
                uint32_t even[2], odd[2];                // byte j: dimension 2j (+ 1) of keys (a, a + 1)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t ka = cur.v[2 * h][w], kn = cur.v[2 * h + 1][w];
                    even[h] = (ka & 0x0f0f0f0fu) | ((kn << 4) & 0xf0f0f0f0u);
                    odd[h] = ((ka >> 4) & 0x0f0f0f0fu) | (kn & 0xf0f0f0f0u);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t sel = 0x7604u + 0x10u * j;
                    const uint32_t a0 = lds_tab<128>(prmt(even[0], lane4, sel)), a1 = lds_tab<128>(prmt(odd[0], lane4, sel));
                    const uint32_t a2 = lds_tab<128>(prmt(even[1], lane4, sel)), a3 = lds_tab<128>(prmt(odd[1], lane4, sel));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma16816<true>(o[nt][4 * w + j], a0, a1, a2, a3, b[nt][0], b[nt][1]);
                }
            }
        }

        // ---------------- join the warps ----------------
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float v = sum[nt][c];
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) v += __shfl_xor_sync(0xffffffffu, v, x);
                if (g == 0) stat[warp * NC + nt * 8 + 2 * t + c] = make_float2(ref[nt][c], v);
            }
        const bool whole = f == seg0 && end == seg1;
        // this piece's slot: the CTA's last segment when the segment starts here, else its first
        const bool starts = f == seg0;
        float* part = parts + (size_t)(2 * blockIdx.x + (starts ? 1 : 0)) * slot_floats(D);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float* dst = merge + (warp * 8 + 2 * t + c) * kOStride + g * (D / 8);
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    dst[2 * i] = o[nt][i][c];
                    dst[2 * i + 1] = o[nt][i][c + 2];
                }
            }
            __syncthreads();
            for (int i = tid; i < 8 * (D / 4); i += kThreads) {
                const int c = i / (D / 4), d = (i % (D / 4)) * 4, col = nt * 8 + c;
                float m = kRefInit;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) m = fmaxf(m, stat[w * NC + col].x);
                float l = 0.0f;
                float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const float2 st = stat[w * NC + col];
                    const float k = exp2_approx(st.x - m);
                    const float4 x = *reinterpret_cast<const float4*>(merge + (w * 8 + c) * kOStride + d);
                    l += st.y * k;
                    v.x += x.x * k; v.y += x.y * k; v.z += x.z * k; v.w += x.w * k;
                }
                if (whole) {
                    if (col < rows) {
                        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                        const int row = row0 + col;
                        uint16_t* dst = p.out + ((int64_t)(rq.q0 + row / p.group) * (p.heads * p.group) +
                                                 head * p.group + row % p.group) * D + d;
                        *reinterpret_cast<uint2*>(dst) = make_uint2(pack2<F16>(v.x * inv, v.y * inv), pack2<F16>(v.z * inv, v.w * inv));
                    }
                } else {
                    __stcg(reinterpret_cast<float4*>(part + col * D + d), v);
                    if (d == 0) {
                        __stcg(part + kMaxCols * D + 2 * col, m);
                        __stcg(part + kMaxCols * D + 2 * col + 1, l);
                    }
                }
            }
            __syncthreads();
        }
        if (!whole) {
            // the last CTA of the segment to arrive joins the parts in key order
            const int c0 = (int)(seg0 / chunk), c1 = (int)((seg1 - 1) / chunk);
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                const uint32_t n = (uint32_t)(c1 - c0);
                const bool last = atomicInc(&counters[c0], n) == n;        // wraps to 0
                scratch[kWarps + 2] = last;
            }
            __syncthreads();
            const bool last = scratch[kWarps + 2] != 0;
            if (last) {
                __threadfence();
                for (int i = tid; i < NC * (D / 4); i += kThreads) {
                    const int col = i / (D / 4), d = (i % (D / 4)) * 4;
                    if (col >= rows) continue;
                    float m = kRefInit;
                    for (int c = c0; c <= c1; ++c) {
                        const float* src = parts + (size_t)(2 * c + (c == c0 ? 1 : 0)) * slot_floats(D);
                        m = fmaxf(m, __ldcg(src + kMaxCols * D + 2 * col));
                    }
                    float l = 0.0f;
                    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    for (int c = c0; c <= c1; ++c) {
                        const float* src = parts + (size_t)(2 * c + (c == c0 ? 1 : 0)) * slot_floats(D);
                        const float k = exp2_approx(__ldcg(src + kMaxCols * D + 2 * col) - m);
                        const float4 x = __ldcg(reinterpret_cast<const float4*>(src + col * D + d));
                        l += __ldcg(src + kMaxCols * D + 2 * col + 1) * k;
                        v.x += x.x * k; v.y += x.y * k; v.z += x.z * k; v.w += x.w * k;
                    }
                    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                    const int row = row0 + col;
                    uint16_t* dst = p.out + ((int64_t)(rq.q0 + row / p.group) * (p.heads * p.group) + head * p.group +
                                             row % p.group) * D + d;
                    *reinterpret_cast<uint2*>(dst) = make_uint2(pack2<F16>(v.x * inv, v.y * inv), pack2<F16>(v.z * inv, v.w * inv));
                }
            }
            __syncthreads();
        }
        f = end;
    }
}

template <int D, int NT>
constexpr size_t smem_bytes()
{
    return kTabBytes + (size_t)kWarps * 8 * (D + 4) * 4 + (size_t)kWarps * 8 * NT * 8 + (kWarps + 4) * 8;
}

template <int D, bool F16, int NT>
cudaError_t launch_attend(const KvAttendParams& p, cudaStream_t s)
{
    static bool configured[64] = {false};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    constexpr size_t bytes = smem_bytes<D, NT>();
    if (!configured[dev]) {
        int reserved = 0;
        if ((e = cudaDeviceGetAttribute(&reserved, cudaDevAttrReservedSharedMemoryPerBlock, dev)) != cudaSuccess) return e;
        if (reserved != (int)kTabOff) return cudaErrorNotSupported;       // the table's address is fixed
        if ((e = cudaFuncSetAttribute(attend_kernel<D, F16, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes)) != cudaSuccess)
            return e;
        configured[dev] = true;
    }
    const int sms = sm_count() > 0 ? sm_count() : 148;
    int grid = sms * (NT == 1 ? kMaxCtasPerSm : 1);
    grid = grid < kMaxCtas ? grid : kMaxCtas;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = s;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attend_kernel<D, F16, NT>, p);
}

template <int D, bool F16>
cudaError_t launch_for(const KvAttendParams& p, int64_t max_rows, cudaStream_t s)
{
    return max_rows <= 8 ? launch_attend<D, F16, 1>(p, s) : launch_attend<D, F16, 2>(p, s);
}

}  // namespace

cudaError_t launch_kv_attend_small(const KvAttendParams& p, int head_dim, bool f16, int64_t max_rows, cudaStream_t s)
{
    if (head_dim == 128) return f16 ? launch_for<128, true>(p, max_rows, s) : launch_for<128, false>(p, max_rows, s);
    return f16 ? launch_for<64, true>(p, max_rows, s) : launch_for<64, false>(p, max_rows, s);
}

}  // namespace logq
