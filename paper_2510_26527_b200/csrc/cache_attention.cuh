// What the two kernels of the attention over 4-bit pages share (formulas: cache_attention.cu): the problem, how it is cut into segments and shares,
// the codes as fp16 numbers, finished outputs, the joining of partial results.
#pragma once

#include <cuda_fp16.h>

#include "kv_pages.cuh"

namespace polyspec {
namespace attend {

constexpr int kMaxCtas = 608;                   // CTAs that the workspace has room for
constexpr float kNone = -3.0e38f;               // a maximum over nothing
constexpr float kLift = 3.0f;                   // p' is 2^3 at the maximum that the reference was taken from
constexpr float kSlack = 12.0f;                 // and may rise to 2^15, near fp16's end, before sums are rescaled

struct AttendParams {
    polyspec_cache_pages s;
    polyspec_block_rows r;
    const unsigned short* q;                    // bf16 bits
    long long q_stride;
    int q_heads, kv_heads, group;
    float scale_log2;                           // scale * log2(e)
    const unsigned char* pool;
    size_t plane_bytes;
    int units_per_page;
    unsigned short* out;
    float* lse;
    float* partial;                             // [2 * CTAs][rows of a tile][head_dim + 2]
    int4* joins;                                // [CTAs]: (parts, sequence * 64 + row groups, key head, first row) of the segment that begins there and ends elsewhere
    int32_t* status;
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float lg2(float x)
{
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t half2_bits(float a, float b)
{
    const __half2 x = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&x);
}
__device__ __forceinline__ uint32_t bf16x2_bits(float a, float b)
{
    uint32_t x;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(x) : "f"(b), "f"(a));
    return x;
}
__device__ __forceinline__ float low(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float high(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }

// Pair i (0..3) of a word's codes as two fp16 numbers: elements 2i, 2i+1 for keys.  Odd pairs come 16-fold.
__device__ __forceinline__ uint32_t code_pair(uint32_t word, int i) { return (i >= 2 ? word >> 8 : word) & (i & 1 ? 0x00f000f0u : 0x000f000fu); }

// The power of two that brings numbers of up to `top` in size into [2^14, 2^15), and what their products with codes (which bring 2^-24) are to be multiplied with.
__device__ __forceinline__ float row_scale(const AttendParams& p, float top, float* factor)
{
    const int k = top > 0.0f ? max(-100, static_cast<int>(__float_as_uint(top) >> 23) - 127) : 0;          // top in [2^k, 2^(k+1))
    *factor = p.scale_log2 * __uint_as_float(static_cast<uint32_t>(min(254, 10 + k + 127)) << 23);
    return __uint_as_float(static_cast<uint32_t>(14 - k + 127) << 23);
}

// A segment, and where in the list of them a cursor stands: row tile `tile` of `tiles` with tile_rows rows each (a multiple of 8; rows times heads of the
// group are dealt out evenly), `steps` steps over the tokens.
struct Segment { int b, head, tile, tiles, tile_rows, steps; kv::SeqRows q; };

template <int ROWS, int STEP>
__device__ __forceinline__ void seq_segments(const AttendParams& p, Segment& g)
{
    const int groups = (g.q.n * p.group + 7) / 8;
    g.tiles = (groups + ROWS / 8 - 1) / (ROWS / 8);
    g.tile_rows = g.tiles ? (groups + g.tiles - 1) / g.tiles * 8 : 8;
    g.steps = max(1, (g.q.base + g.q.granted + STEP - 1) / STEP);
}

// Slots that row i of a block attends to: up to its own, none if that was not granted.
__device__ __forceinline__ int row_limit(const kv::SeqRows& q, int i) { return i < q.granted ? q.base + i + 1 : 0; }

// All sequences' steps and overheads one behind the other: the sequence that holds place `at`, the place within it; returns the total.  Every thread
// calls it.
template <class S>
__device__ __forceinline__ long long locate(const AttendParams& p, long long at, int* seq, long long* within, long long* warp_sums, int* hit, long long* hit_at)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long carry = 0;
    if (threadIdx.x == 0) *hit = -1;
    for (int b0 = 0; b0 < p.s.n_seqs; b0 += S::THREADS) {
        const int b = b0 + threadIdx.x;
        long long n = 0;
        if (b < p.s.n_seqs) {
            Segment g;
            g.q = kv::seq_rows(p.s, p.r, b);
            if (g.q.bad && blockIdx.x == 0) kv::report(p.status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE);
            seq_segments<S::ROWS, S::STEP>(p, g);
            n = static_cast<long long>(g.tiles) * (g.steps + S::OVERHEAD) * p.kv_heads;
        }
        long long inc = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, inc, d);
            if (lane >= d) inc += y;
        }
        __syncthreads();
        if (lane == 31) warp_sums[warp] = inc;
        __syncthreads();
        long long before = carry;
        for (int w = 0; w < S::WARPS; ++w) {
            if (w < warp) before += warp_sums[w];
            carry += warp_sums[w];
        }
        const long long start = before + inc - n;
        if (n > 0 && start <= at && at < start + n) { *hit = b; *hit_at = at - start; }
    }
    __syncthreads();
    *seq = *hit;
    *within = *hit_at;
    __syncthreads();
    return carry;
}

// A cursor over segments: the next (row tile, then head, then sequence with rows).
template <class S>
__device__ __forceinline__ void next_segment(const AttendParams& p, Segment& g)
{
    if (++g.tile < g.tiles) return;
    g.tile = 0;
    if (++g.head < p.kv_heads) return;
    g.head = 0;
    do {
        if (++g.b >= p.s.n_seqs) { g.tiles = 0; g.tile_rows = 8; g.steps = 0x7fffffff; g.q = kv::SeqRows{0, 0, 0, 0, 0, false}; return; }
        g.q = kv::seq_rows(p.s, p.r, g.b);
        seq_segments<S::ROWS, S::STEP>(p, g);
    } while (g.tiles == 0);
}

// Tokens that some row of the segment attends to.
__device__ __forceinline__ int visible(const AttendParams& p, const Segment& g)
{
    const int first = g.tile * g.tile_rows / p.group, last = min(g.q.n - 1, (g.tile * g.tile_rows + g.tile_rows - 1) / p.group);
    return first < g.q.granted ? row_limit(g.q, min(last, g.q.granted - 1)) : 0;
}

// Normalised outputs of eight neighbouring elements of a row.
__device__ __forceinline__ void store_out(const AttendParams& p, const kv::SeqRows& q, int kv_head, int r, int D, int d0, const float* x, float m, float l)
{
    const int i = r / p.group;
    if (i >= q.n) return;
    const size_t at = static_cast<size_t>(q.row0 + i) * p.q_heads + kv_head * p.group + r % p.group;
    const bool none = row_limit(q, i) == 0;
    const float inv = none ? 0.0f : 1.0f / l;
    uint4 y;
    y.x = bf16x2_bits(x[0] * inv, x[1] * inv);
    y.y = bf16x2_bits(x[2] * inv, x[3] * inv);
    y.z = bf16x2_bits(x[4] * inv, x[5] * inv);
    y.w = bf16x2_bits(x[6] * inv, x[7] * inv);
    if (none) y = make_uint4(0, 0, 0, 0);
    *reinterpret_cast<uint4*>(p.out + at * D + d0) = y;
    if (d0 == 0 && p.lse) p.lse[at] = none ? -INFINITY : (m + log2f(l)) * 0.69314718055994530942f;
}

// Joins the parts of the segment that begins in CTA blockIdx.x and ends in a later one, in order.
template <class S>
__global__ void __launch_bounds__(256) join_kernel(const AttendParams p)
{
    constexpr int D = S::D, kVecs = D / 8;
    wait_for_stream();
    const int4 job = p.joins[blockIdx.x];
    if (job.x == 0) return;
    const kv::SeqRows q = kv::seq_rows(p.s, p.r, job.y >> 6);
    const int job_rows = (job.y & 63) * 8;
    for (int item = threadIdx.x; item < S::ROWS * kVecs; item += 256) {
        const int r = item / kVecs, d0 = item % kVecs * 8;
        if (job.w + r >= q.n * p.group || r >= job_rows) continue;
        float x[8], m = kNone, l = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.0f;
        for (int k = 0; k < job.x; ++k) {
            const float* part = p.partial + static_cast<size_t>(k ? 2 * (blockIdx.x + k) : 2 * blockIdx.x + 1) * S::PART;
            const float2 ml = *reinterpret_cast<const float2*>(part + S::ROWS * D + 2 * r);
            const float4 a = reinterpret_cast<const float4*>(part + r * D + d0)[0], b = reinterpret_cast<const float4*>(part + r * D + d0)[1];
            const float to = fmaxf(m, ml.x), was = ex2(m - to), is = ex2(ml.x - to);
            m = to;
            l = fmaf(l, was, ml.y * is);
            x[0] = fmaf(x[0], was, a.x * is); x[1] = fmaf(x[1], was, a.y * is); x[2] = fmaf(x[2], was, a.z * is); x[3] = fmaf(x[3], was, a.w * is);
            x[4] = fmaf(x[4], was, b.x * is); x[5] = fmaf(x[5], was, b.y * is); x[6] = fmaf(x[6], was, b.z * is); x[7] = fmaf(x[7], was, b.w * is);
        }
        store_out(p, q, job.z, job.w + r, D, d0, x, m, l);
    }
}

// The tensor-core kernel (cache_attention_wide.cu): head_dim 128, row tiles of up to kWideRows.
constexpr int kWideRows = 48;
cudaError_t launch_attend_wide(const AttendParams& p, cudaStream_t stream);

}  // namespace attend
}  // namespace polyspec
