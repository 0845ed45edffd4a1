// Attention of a block's rows over a cache held in 4 bits (layout: kv_pages.cuh), and the weight that each cached token was given.
//
//   s[r, j] = scale * q[r] . K[j],  K[j] = ks[j] * ck[j] + ko[j];  out[r] = sum_j softmax_j(s)[r, j] V[j],  V[j] = vs[j] * cv[j] + vo[j]
//
// The matrix instructions multiply codes, never dequantised numbers:
//   s[r, j] = ks[j] * (q[r] . ck[j]) + ko[j] * sum(q[r])                        one product and one FMA per (row, token)
//   out[r]  = (sum_j p'[r, j] cv[j] + sum_j p[r, j] vo[j]) / sum_j p[r, j],     p' = p * vs[j]
// p' comes out of the exponential itself: 2^(s + log2 vs[j] - m), with m the running maximum of s + log2 vs, so that it is at its most
// accurate where it counts; p = p' / vs[j].
//
// A code is an fp16 number without any arithmetic: four bits under a mask are a subnormal, code * 2^-24, and the same mask four
// bits higher gives 16 * code * 2^-24.  Matrix instructions multiply subnormals exactly; the 16 goes into the query's elements
// (as 1/16) or out of the finished sums.  So eight codes cost four masks and one shift (keys), and two byte permutes more per sixteen
// where pairs of tokens have to be brought together (values).  Queries are scaled by a power of two into fp16's upper range, where their
// bf16 digits are exact down to 2^-28 of the block's largest.
//
// mma.sync on 16 rows: a block's rows times the heads that share a key head, 4 to 36 of them, fill a tile; tcgen05's tiles of 128
// rows would be mostly empty, and its operands would have to be expanded through shared or tensor memory.
//
// Work: (sequence, key head, row tile) are segments of `steps` of 16 tokens per warp; the steps of all segments, one after the other, are cut into equal
// shares, one per CTA, whatever the lengths.  Each warp streams its tiles through a ring of its own (cp.async) and keeps maximum,
// sums and the output tile in registers; a segment's warps meet once at its end.  A segment that crosses CTAs leaves partial
// results, which a second kernel joins.
#include <cuda_fp16.h>

#include "kv_pages.cuh"

namespace polyspec {
namespace {

constexpr int kMaxCtas = 304;                   // CTAs that the workspace has room for
constexpr float kNone = -3.0e38f;               // a maximum over nothing
constexpr float kLift = 7.0f;                   // p' is kept 2^7 above 1 at the maximum, out of fp16's subnormals
constexpr float kSlack = 8.0f;                  // and may rise to 2^15 before sums are rescaled

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
    int4* joins;                                // [CTAs]: (parts, sequence, key head, row tile) of the segment that begins there and ends elsewhere
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
    asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp(float x)
{
    float y;
    asm("rcp.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
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

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Pair i (0..3) of a word's codes as two fp16 numbers: elements 2i, 2i+1 for keys.  Odd pairs come 16-fold.
__device__ __forceinline__ uint32_t code_pair(uint32_t word, int i) { return (i >= 2 ? word >> 8 : word) & (i & 1 ? 0x00f000f0u : 0x000f000fu); }

__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool there)
{
    const int n = there ? 16 : 0;               // 0: the piece is filled with zeros, nothing is read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(n) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Rows of a tile as the A operand of the first product.  The element order inside a step of 16 follows the codes' (words are dealt out to lanes
// whole); elements whose codes come 16-fold are divided by 16.  Thread `item` holds eight elements of one row.
template <int D>
__device__ __forceinline__ void store_fragment(uint32_t* frag /* [tiles][D / 16][32][4] */, int r, int word, const float* x, float by)
{
    constexpr int kWords = D / 32;              // words of a token per lane
    const int t = word / kWords, w = word % kWords, lane = (r & 7) * 4 + t, reg = (r >> 3) & 1;
    uint32_t* to = frag + (((r >> 4) * (D / 16) + 2 * w) * 32 + lane) * 4 + reg;
    const float by16 = by * 0.0625f;
    to[0] = half2_bits(x[0] * by, x[1] * by);
    to[2] = half2_bits(x[2] * by16, x[3] * by16);
    to[128] = half2_bits(x[4] * by, x[5] * by);
    to[130] = half2_bits(x[6] * by16, x[7] * by16);
}

// The rows of a tile into shared memory, by all THREADS of a CTA.  Row r of a tile is row (tile * ROWS + r) / group of the block, head
// kv_head * group + (tile * ROWS + r) % group.  sums[r] = scale * log2(e) * sum of the row; *factor = what a product of fragments and codes
// is multiplied with.  Ends with the CTA in step.
template <int D, int ROWS, int THREADS>
__device__ __forceinline__ void load_rows(const AttendParams& p, const kv::SeqRows& q, int kv_head, int tile, uint32_t* frag, float* sums, float* warp_max,
                                          float* factor)
{
    constexpr int kVecs = D / 8, kItems = ROWS * kVecs, kPer = (kItems + THREADS - 1) / THREADS;
    static_assert(kItems % THREADS == 0 || (kPer == 1 && kItems % 32 == 0), "whole warps take part or none");
    uint4 raw[kPer];
    float top = 0.0f;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int item = u * THREADS + threadIdx.x, r = tile * ROWS + item / kVecs, i = r / p.group;
        raw[u] = make_uint4(0, 0, 0, 0);
        if (item < kItems && i < q.n) raw[u] = *reinterpret_cast<const uint4*>(p.q + (q.row0 + i) * p.q_stride + (kv_head * p.group + r % p.group) * D + item % kVecs * 8);
        const uint32_t* x = reinterpret_cast<const uint32_t*>(&raw[u]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = fabsf(low(x[e])), b = fabsf(high(x[e]));
            if (a <= 3.4e38f) top = fmaxf(top, a);
            if (b <= 3.4e38f) top = fmaxf(top, b);
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) top = fmaxf(top, warp_max[w]);
    // top in [2^k, 2^(k+1)): by 2^(14-k) into [2^14, 2^15); codes bring 2^-24
    const int k = top > 0.0f ? max(-100, static_cast<int>(__float_as_uint(top) >> 23) - 127) : 0;
    const float by = __uint_as_float(static_cast<uint32_t>(14 - k + 127) << 23);
    *factor = p.scale_log2 * __uint_as_float(static_cast<uint32_t>(min(254, 10 + k + 127)) << 23);
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int item = u * THREADS + threadIdx.x, r = item / kVecs;
        if (item >= kItems) break;
        const uint32_t* y = reinterpret_cast<const uint32_t*>(&raw[u]);
        float x[8], sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[2 * e] = low(y[e]); x[2 * e + 1] = high(y[e]); sum += x[2 * e] + x[2 * e + 1]; }
        store_fragment<D>(frag, r, item % kVecs, x, by);
#pragma unroll
        for (int d = 1; d < kVecs; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (item % kVecs == 0) sums[r] = sum * p.scale_log2;
    }
    __syncthreads();
}

// What a CTA's share of the steps is, and where in it a cursor stands.
struct Segment { int b, head, tile, tiles, steps; kv::SeqRows q; };

template <int ROWS, int STEP>
__device__ __forceinline__ void seq_segments(const AttendParams& p, Segment& g)
{
    g.tiles = (g.q.n * p.group + ROWS - 1) / ROWS;
    g.steps = max(1, (g.q.base + g.q.granted + STEP - 1) / STEP);
}

// Slots that row i of a block attends to: up to its own, none if that was not granted.
__device__ __forceinline__ int row_limit(const kv::SeqRows& q, int i) { return i < q.granted ? q.base + i + 1 : 0; }

template <int D_, int MT_, int WARPS_, int STAGES_, int CTAS_>
struct Shape {
    static constexpr int D = D_, MT = MT_, WARPS = WARPS_, STAGES = STAGES_, CTAS = CTAS_;
    static constexpr int THREADS = WARPS * 32, ROWS = MT * 16, STEP = WARPS * 16;       // STEP: tokens
    static constexpr int UB = kv::unit_bytes(D), STAGE = 4 * UB;
    static constexpr int FRAG = MT * (D / 16) * 512;                                    // bytes
    static constexpr int RING = WARPS * STAGES * STAGE;
    static constexpr int MERGE = WARPS / 2 * MT * (D / 8) * 512;
    static constexpr size_t SMEM = FRAG + RING + MERGE;
    static constexpr int PART = ROWS * (D + 2);                                         // floats of a partial result
    static_assert(SMEM * CTAS <= 220 * 1024, "shared memory");
};

// Where the steps of sequence b begin among all sequences' steps: the sequence that holds step `at`, or the total.  Every thread calls it.
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
            n = static_cast<long long>(g.tiles) * g.steps * p.kv_heads;
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
        if (++g.b >= p.s.n_seqs) { g.tiles = 0; g.steps = 0x7fffffff; g.q = kv::SeqRows{0, 0, 0, 0, 0, false}; return; }
        g.q = kv::seq_rows(p.s, p.r, g.b);
        seq_segments<S::ROWS, S::STEP>(p, g);
    } while (g.tiles == 0);
}

// Tokens that some row of the segment attends to.
template <class S>
__device__ __forceinline__ int visible(const AttendParams& p, const Segment& g)
{
    const int first = g.tile * S::ROWS / p.group, last = min(g.q.n - 1, (g.tile * S::ROWS + S::ROWS - 1) / p.group);
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

template <class S>
__global__ void __launch_bounds__(S::THREADS, S::CTAS) attend_kernel(const AttendParams p)
{
    constexpr int D = S::D, MT = S::MT, W = S::WARPS, NS = S::STAGES, KS = D / 16, NT = D / 8, UB = S::UB, WORDS = D / 32, H = D / 64;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ long long warp_sums[W], hit_at;
    __shared__ int hit;
    __shared__ float warp_max[W], sums[S::ROWS], sm_m[W][S::ROWS], sm_l[W][S::ROWS], sm_o[W][S::ROWS];
    uint32_t* frag = reinterpret_cast<uint32_t*>(smem);
    float4* merge = reinterpret_cast<float4*>(smem + S::FRAG + S::RING);
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, g8 = lane >> 2, t4 = lane & 3;
    unsigned char* ring = smem + S::FRAG + warp * NS * S::STAGE;
    const uint32_t ring_at = static_cast<uint32_t>(__cvta_generic_to_shared(ring));
    wait_for_stream();

    // this CTA's share [s0, s1) of all steps
    int seq;
    long long within;
    const long long total = locate<S>(p, -1, &seq, &within, warp_sums, &hit, &hit_at);
    const long long ctas = min(total, static_cast<long long>(gridDim.x));         // that have a step to do
    if (threadIdx.x == 0) p.joins[blockIdx.x] = make_int4(0, 0, 0, 0);
    if (blockIdx.x >= ctas) return;
    const long long s0 = total * blockIdx.x / ctas, s1 = total * (blockIdx.x + 1) / ctas;
    locate<S>(p, s0, &seq, &within, warp_sums, &hit, &hit_at);
    Segment mine;                                // the consumer's
    mine.b = seq;
    mine.q = kv::seq_rows(p.s, p.r, seq);
    seq_segments<S::ROWS, S::STEP>(p, mine);
    int step = static_cast<int>(within % mine.steps);
    {
        const int n = static_cast<int>(within / mine.steps);
        mine.head = n / mine.tiles;
        mine.tile = n % mine.tiles;
    }
    Segment ahead = mine;                       // the producer's
    int ahead_step = step, ahead_visible = visible<S>(p, ahead);
    const int n_steps = static_cast<int>(s1 - s0);

    // lane 2k + u: unit u of the warp's k-th tile from here on, as a number of units in a plane, or ~0
    uint32_t unit_numbers = 0;
    int unit_k = 16;                            // tiles of `unit_numbers` that are used up
    uint32_t bad_units = 0;                     // bit 2 stage + u: nothing could be read there

    auto issue = [&](int stage) {
        if (unit_k == 16) {
            const long long slot = (static_cast<long long>(ahead_step + (lane >> 1)) * W + warp) * 16 + (lane & 1) * 8;
            unit_numbers = 0xffffffffu;
            if (slot < ahead_visible) {
                const int unit = static_cast<int>(slot >> 3), at = unit / p.units_per_page;
                const int page = p.s.table[static_cast<size_t>(ahead.b) * p.s.max_pages + at];
                if (page >= 0 && page < p.s.n_pages)
                    unit_numbers = (static_cast<uint32_t>(page) * p.kv_heads + ahead.head) * p.units_per_page + (unit - at * p.units_per_page);
                else
                    kv::report(p.status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE);
            }
            unit_k = 0;
        }
        const uint32_t to = ring_at + stage * S::STAGE;
        const uint32_t u0 = __shfl_sync(0xffffffffu, unit_numbers, 2 * unit_k), u1 = __shfl_sync(0xffffffffu, unit_numbers, 2 * unit_k + 1);
        const bool there0 = u0 != 0xffffffffu, there1 = u1 != 0xffffffffu;
        const unsigned char* k0 = p.pool + static_cast<size_t>(there0 ? u0 : 0) * UB;
        const unsigned char* k1 = p.pool + static_cast<size_t>(there1 ? u1 : 0) * UB;
        bad_units = (bad_units & ~(3u << (2 * stage))) | ((there0 ? 0u : 1u) | (there1 ? 0u : 2u)) << (2 * stage);
        if (D == 128) {
            copy16(to + lane * 16, k0 + lane * 16, there0);
            copy16(to + UB + lane * 16, k1 + lane * 16, there1);
            copy16(to + 2 * UB + lane * 16, k0 + p.plane_bytes + lane * 16, there0);
            copy16(to + 3 * UB + lane * 16, k1 + p.plane_bytes + lane * 16, there1);
        } else {
            const int o = (lane & 15) * 16;
            const unsigned char* k = lane < 16 ? k0 : k1;
            const bool there = lane < 16 ? there0 : there1;
            copy16(to + (lane >> 4) * UB + o, k + o, there);
            copy16(to + (2 + (lane >> 4)) * UB + o, k + p.plane_bytes + o, there);
        }
        if (lane < 8) {                         // scales and offsets: two pieces of each unit
            const int n = lane >> 1, o = 4 * D + (lane & 1) * 16;
            copy16(to + n * UB + o, (n & 1 ? k1 : k0) + (n >> 1 ? p.plane_bytes : 0) + o, n & 1 ? there1 : there0);
        }
        ++unit_k;
        if (++ahead_step == ahead.steps) {
            next_segment<S>(p, ahead);
            ahead_step = 0;
            ahead_visible = visible<S>(p, ahead);
            unit_k = 16;
        }
    };

    int issued = 0;
    for (; issued < NS - 1; ++issued) {
        if (issued < n_steps) issue(issued);
        copies_end();
    }

    float o[MT][NT][4], m[MT][2], l[MT][2], lo[MT][2];
    int limit[MT][2];
    int seen = 0, done = 0, stage = 0;          // done: steps
    bool from_start = step == 0;
    float factor = 0.0f;
    bool fresh = true;
    while (done < n_steps) {
        if (fresh) {
            load_rows<D, S::ROWS, S::THREADS>(p, mine.q, mine.head, mine.tile, frag, sums, warp_max, &factor);
            seen = visible<S>(p, mine);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int r = mine.tile * S::ROWS + i * 16 + j * 8 + g8;
                    limit[i][j] = row_limit(mine.q, r / p.group);
                    m[i][j] = kNone;
                    l[i][j] = lo[i][j] = 0.0f;
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) o[i][n][0] = o[i][n][1] = o[i][n][2] = o[i][n][3] = 0.0f;
            }
            fresh = false;
        }
        copies_wait<NS - 2>();
        __syncwarp();
        const int key0 = (step * W + warp) * 16;
        if (key0 < seen) {
            const unsigned char* at = ring + stage * S::STAGE;
            // codes of keys, and the first product
            uint32_t kw[2][WORDS];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (D == 128) {
                    const uint4 x = *reinterpret_cast<const uint4*>(at + u * UB + lane * 16);
                    kw[u][0] = x.x; kw[u][1] = x.y; kw[u][WORDS - 2] = x.z; kw[u][WORDS - 1] = x.w;
                } else {
                    const uint2 x = *reinterpret_cast<const uint2*>(at + u * UB + lane * 8);
                    kw[u][0] = x.x; kw[u][1] = x.y;
                }
            }
            float sc[MT][2][4];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int u = 0; u < 2; ++u) sc[i][u][0] = sc[i][u][1] = sc[i][u][2] = sc[i][u][3] = 0.0f;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                uint32_t b[2][2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    b[u][0] = code_pair(kw[u][s >> 1], 2 * (s & 1));
                    b[u][1] = code_pair(kw[u][s >> 1], 2 * (s & 1) + 1);
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const uint4 a = *reinterpret_cast<const uint4*>(frag + ((i * KS + s) * 32 + lane) * 4);
                    mma(sc[i][0], a.x, a.y, a.z, a.w, b[0][0], b[0][1]);
                    mma(sc[i][1], a.x, a.y, a.z, a.w, b[1][0], b[1][1]);
                }
            }
            // scales and offsets of the lane's four tokens: 8u + 2 t4 + j
            float ks[2][2], ko[2][2], lv[2][2], iv[2][2], ov[2][2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint2 kp = *reinterpret_cast<const uint2*>(at + u * UB + 4 * D + t4 * 8);
                const uint2 vp = *reinterpret_cast<const uint2*>(at + (2 + u) * UB + 4 * D + t4 * 8);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    ks[u][j] = low(j ? kp.y : kp.x) * factor;
                    ko[u][j] = high(j ? kp.y : kp.x);
                    const float vs = low(j ? vp.y : vp.x);
                    lv[u][j] = lg2(vs);
                    iv[u][j] = rcp(vs);
                    ov[u][j] = high(j ? vp.y : vp.x) * iv[u][j];
                }
            }
            // masked: some row does not see some token of the tile, or a page could not be read
            const uint32_t bad = bad_units >> (2 * stage) & 3u;
            const bool masked = key0 + 16 > mine.q.base + 1 || bad;
            uint32_t pr[MT][4];
#pragma unroll
            for (int i = 0; i < MT; ++i) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {                           // rows g8 and g8 + 8
                    const float sq = sums[i * 16 + j * 8 + g8];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
#pragma unroll
                        for (int c = 0; c < 2; ++c)
                            sc[i][u][2 * j + c] = fmaf(sc[i][u][2 * j + c], ks[u][c], fmaf(sq, ko[u][c], lv[u][c]));
                    }
                }
                uint32_t hidden = 0;                                    // bit 4 u + 2 j + c
                if (masked) {
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int c = 0; c < 2; ++c)
                                if (key0 + 8 * u + 2 * t4 + c >= limit[i][j] || (bad >> u & 1u)) {
                                    hidden |= 1u << (4 * u + 2 * j + c);
                                    sc[i][u][2 * j + c] = -INFINITY;
                                }
                }
                const float top0 = fmaxf(fmaxf(sc[i][0][0], sc[i][0][1]), fmaxf(sc[i][1][0], sc[i][1][1]));
                const float top1 = fmaxf(fmaxf(sc[i][0][2], sc[i][0][3]), fmaxf(sc[i][1][2], sc[i][1][3]));
                // sums are rescaled only when the maximum has risen by 2^8 since the last time
                if (__any_sync(0xffffffffu, top0 > m[i][0] + kSlack || top1 > m[i][1] + kSlack)) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float top = j ? top1 : top0;
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                        const float to = fmaxf(m[i][j], top), by = ex2(m[i][j] - to);
                        m[i][j] = to;
                        l[i][j] *= by;
                        lo[i][j] *= by;
#pragma unroll
                        for (int n = 0; n < NT; ++n) { o[i][n][2 * j] *= by; o[i][n][2 * j + 1] *= by; }
                    }
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float ref = m[i][j] - kLift;
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int c = 0; c < 2; ++c) sc[i][u][2 * j + c] = ex2(sc[i][u][2 * j + c] - ref);
                    if (!masked) {
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                l[i][j] = fmaf(sc[i][u][2 * j + c], iv[u][c], l[i][j]);
                                lo[i][j] = fmaf(sc[i][u][2 * j + c], ov[u][c], lo[i][j]);
                            }
                    } else {                    // scales behind what a row sees may be anything
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int c = 0; c < 2; ++c)
                                if (!(hidden >> (4 * u + 2 * j + c) & 1u)) {
                                    l[i][j] = fmaf(sc[i][u][2 * j + c], iv[u][c], l[i][j]);
                                    lo[i][j] = fmaf(sc[i][u][2 * j + c], ov[u][c], lo[i][j]);
                                }
                    }
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    pr[i][2 * u] = half2_bits(sc[i][u][0], sc[i][u][1]);
                    pr[i][2 * u + 1] = half2_bits(sc[i][u][2], sc[i][u][3]);
                }
            }
            // codes of values: words of the lane's two tokens, paired by token, and the second product
            uint32_t vw[2][2][H];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (D == 128) {
                    const uint4 x = *reinterpret_cast<const uint4*>(at + (2 + u) * UB + lane * 16);
                    vw[u][0][0] = x.x; vw[u][0][H - 1] = x.y; vw[u][1][0] = x.z; vw[u][1][H - 1] = x.w;
                } else {
                    const uint2 x = *reinterpret_cast<const uint2*>(at + (2 + u) * UB + lane * 8);
                    vw[u][0][0] = x.x; vw[u][1][0] = x.y;
                }
            }
#pragma unroll
            for (int h = 0; h < H; ++h) {
                uint32_t even[2], odd[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    even[u] = __byte_perm(vw[u][0][h], vw[u][1][h], 0x5410);
                    odd[u] = __byte_perm(vw[u][0][h], vw[u][1][h], 0x7632);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t b0 = code_pair(e & 1 ? odd[0] : even[0], e >> 1), b1 = code_pair(e & 1 ? odd[1] : even[1], e >> 1);
#pragma unroll
                    for (int i = 0; i < MT; ++i) mma(o[i][h * 8 + e], pr[i][0], pr[i][1], pr[i][2], pr[i][3], b0, b1);
                }
            }
        }
        __syncwarp();
        // the stage that was read before this one is free again
        {
            const int to = stage == 0 ? NS - 1 : stage - 1;
            if (issued < n_steps) issue(to);
            ++issued;
            copies_end();
        }
        stage = stage + 1 == NS ? 0 : stage + 1;
        ++done;
        ++step;
        if (step < mine.steps && done < n_steps) continue;

        // the segment, or this CTA's part of it, is done: its warps meet
        const bool whole = from_start && step == mine.steps;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int d = 1; d < 4; d <<= 1) {
                    l[i][j] += __shfl_xor_sync(0xffffffffu, l[i][j], d);
                    lo[i][j] += __shfl_xor_sync(0xffffffffu, lo[i][j], d);
                }
                if (t4 == 0) sm_m[warp][i * 16 + j * 8 + g8] = m[i][j];
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = i * 16 + j * 8 + g8;
                float top = kNone;
#pragma unroll
                for (int w = 0; w < W; ++w) top = fmaxf(top, sm_m[w][r]);
                const float by = ex2(m[i][j] - top);
                if (t4 == 0) { sm_l[warp][r] = l[i][j] * by; sm_o[warp][r] = lo[i][j] * by; }
                m[i][j] = top;
#pragma unroll
                for (int n = 0; n < NT; ++n) { o[i][n][2 * j] *= by; o[i][n][2 * j + 1] *= by; }
            }
        if (warp >= W / 2) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    merge[(((warp - W / 2) * MT + i) * NT + n) * 32 + lane] = make_float4(o[i][n][0], o[i][n][1], o[i][n][2], o[i][n][3]);
        }
        __syncthreads();
        if (warp < W / 2) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float4* at = &merge[((warp * MT + i) * NT + n) * 32 + lane];
                    const float4 x = *at;
                    *at = make_float4(o[i][n][0] + x.x, o[i][n][1] + x.y, o[i][n][2] + x.z, o[i][n][3] + x.w);
                }
        }
        __syncthreads();
        // lane and half of the head: elements 64 h + 16 t4 .. + 15 of rows g8 and g8 + 8
        for (int item = threadIdx.x; item < MT * H * 32; item += S::THREADS) {
            const int ln = item & 31, h = item >> 5 & (H - 1), i = item / (32 * H), g = ln >> 2, t = ln & 3;
            float x[4][8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int w = 0; w < W / 2; ++w) {
                    const float4 y = merge[((w * MT + i) * NT + h * 8 + e) * 32 + ln];
                    sum.x += y.x; sum.y += y.y; sum.z += y.z; sum.w += y.w;
                }
                const float by = e & 2 ? 1048576.0f : 16777216.0f;      // 2^20, 2^24: what the codes' form left out
                x[0][e] = sum.x * by; x[1][e] = sum.y * by; x[2][e] = sum.z * by; x[3][e] = sum.w * by;
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = i * 16 + j * 8 + g;
                float top = kNone, lt = 0.0f, ot = 0.0f;
#pragma unroll
                for (int w = 0; w < W; ++w) { top = fmaxf(top, sm_m[w][r]); lt += sm_l[w][r]; ot += sm_o[w][r]; }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float* y = x[2 * j + c];
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] += ot;
                    const int d0 = 64 * h + 16 * t + 8 * c;
                    if (whole) {
                        store_out(p, mine.q, mine.head, mine.tile * S::ROWS + r, D, d0, y, top - kLift, lt);
                    } else if ((mine.tile * S::ROWS + r) / p.group < mine.q.n) {
                        float* part = p.partial + static_cast<size_t>(2 * blockIdx.x + (from_start ? 1 : 0)) * S::PART;
                        reinterpret_cast<float4*>(part + r * D + d0)[0] = make_float4(y[0], y[1], y[2], y[3]);
                        reinterpret_cast<float4*>(part + r * D + d0)[1] = make_float4(y[4], y[5], y[6], y[7]);
                        if (d0 == 0) { part[S::ROWS * D + 2 * r] = top - kLift; part[S::ROWS * D + 2 * r + 1] = lt; }
                    }
                }
            }
        }
        if (!whole && from_start && threadIdx.x == 0) {
            // the CTAs that the rest of the segment falls to
            const long long last = s1 - step + mine.steps - 1;          // its last step
            const int end = static_cast<int>(((last + 1) * ctas - 1) / total);
            p.joins[blockIdx.x] = make_int4(end - static_cast<int>(blockIdx.x) + 1, mine.b, mine.head, mine.tile);
        }
        if (step == mine.steps) {
            next_segment<S>(p, mine);
            step = 0;
        }
        from_start = true;
        fresh = true;
    }
    copies_wait<0>();
}

// Joins the parts of the segment that begins in CTA blockIdx.x and ends in a later one, in order.
template <class S>
__global__ void __launch_bounds__(256) join_kernel(const AttendParams p)
{
    constexpr int D = S::D, kVecs = D / 8;
    wait_for_stream();
    const int4 job = p.joins[blockIdx.x];
    if (job.x == 0) return;
    const kv::SeqRows q = kv::seq_rows(p.s, p.r, job.y);
    for (int item = threadIdx.x; item < S::ROWS * kVecs; item += 256) {
        const int r = item / kVecs, d0 = item % kVecs * 8;
        if ((job.w * S::ROWS + r) / p.group >= q.n) continue;
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
        store_out(p, q, job.z, job.w * S::ROWS + r, D, d0, x, m, l);
    }
}

template <class S>
cudaError_t launch_attend(const AttendParams& p, cudaStream_t stream)
{
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(attend_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(S::SMEM));
    if (e != cudaSuccess) return e;
    const int ctas = sms * S::CTAS < kMaxCtas ? sms * S::CTAS : kMaxCtas;
    e = launch_early(attend_kernel<S>, dim3(static_cast<unsigned>(ctas)), S::THREADS, S::SMEM, stream, p);
    if (e == cudaSuccess) e = launch_early(join_kernel<S>, dim3(static_cast<unsigned>(ctas)), 256, 0, stream, p);
    return e;
}

constexpr int kMaxRows = 32;                    // rows of the largest tile
inline size_t align256(size_t x) { return (x + 255) / 256 * 256; }
inline size_t attend_bytes(int head_dim) { return align256(kMaxCtas * sizeof(int4)) + static_cast<size_t>(2 * kMaxCtas) * kMaxRows * (head_dim + 2) * 4; }

// ---- accumulated weights: w[j] = keep * w[j] + sum over heads and rows of 2^(s2[r, j] - lse2[r])
struct WeighParams {
    AttendParams a;
    const float* lse;
    float keep;
    float* weights;
};

constexpr int kWeighWarps = 8, kWeighTokens = kWeighWarps * 16;

// A CTA has 128 tokens of a sequence, a warp 16 of them: keys only, once per head and row tile, the products as in attend_kernel.  Sums stay in a
// lane's registers over all heads and rows; the lanes of one token meet at the end.  So every sum has one order.
template <int D>
__global__ void __launch_bounds__(kWeighWarps * 32) weigh_kernel(const WeighParams w)
{
    constexpr int KS = D / 16, UB = kv::unit_bytes(D), WORDS = D / 32, ROWS = 32, MT = 2, THREADS = kWeighWarps * 32;
    __shared__ __align__(16) uint32_t frag[MT * KS * 128];
    __shared__ float warp_max[kWeighWarps], sums[ROWS];
    const AttendParams& p = w.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g8 = lane >> 2, t4 = lane & 3, b = blockIdx.y;
    wait_for_stream();
    const kv::SeqRows q = kv::seq_rows(p.s, p.r, b);
    if (q.bad && blockIdx.x == 0 && threadIdx.x == 0) kv::report(p.status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE);
    if (static_cast<long long>(blockIdx.x) * kWeighTokens >= q.len) return;
    const int key0 = blockIdx.x * kWeighTokens + warp * 16;
    uint32_t unit[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        unit[u] = 0xffffffffu;
        if (key0 + 8 * u < q.base + q.granted) {
            const int n = (key0 >> 3) + u, at = n / p.units_per_page;
            const int page = p.s.table[static_cast<size_t>(b) * p.s.max_pages + at];
            if (page >= 0 && page < p.s.n_pages) unit[u] = static_cast<uint32_t>(page) * p.kv_heads * p.units_per_page + (n - at * p.units_per_page);
            else if (lane == 0) kv::report(p.status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE);
        }
    }
    float acc[2][2] = {{0.0f, 0.0f}, {0.0f, 0.0f}};
    const int tiles = (q.n * p.group + ROWS - 1) / ROWS;
    for (int head = 0; head < p.kv_heads; ++head) {
        // the head's keys stay in registers over its row tiles
        uint32_t kw[2][WORDS];
        uint2 kp[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            kp[u] = make_uint2(0, 0);
#pragma unroll
            for (int i = 0; i < WORDS; ++i) kw[u][i] = 0;
            if (unit[u] != 0xffffffffu) {
                const unsigned char* at = p.pool + (static_cast<size_t>(unit[u]) + static_cast<size_t>(head) * p.units_per_page) * UB;
#pragma unroll
                for (int i = 0; i < WORDS; i += 2) {
                    const uint2 x = *reinterpret_cast<const uint2*>(at + lane * (WORDS * 4) + i * 4);
                    kw[u][i] = x.x; kw[u][i + 1] = x.y;
                }
                kp[u] = *reinterpret_cast<const uint2*>(at + 4 * D + t4 * 8);
            }
        }
        for (int tile = 0; tile < tiles; ++tile) {
            float factor;
            __syncthreads();                    // the rows of the tile before have been read
            load_rows<D, ROWS, THREADS>(p, q, head, tile, frag, sums, warp_max, &factor);
            float sc[MT][2][4];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int u = 0; u < 2; ++u) sc[i][u][0] = sc[i][u][1] = sc[i][u][2] = sc[i][u][3] = 0.0f;
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const uint4 a = *reinterpret_cast<const uint4*>(frag + ((i * KS + s) * 32 + lane) * 4);
#pragma unroll
                    for (int u = 0; u < 2; ++u)
                        mma(sc[i][u], a.x, a.y, a.z, a.w, code_pair(kw[u][s >> 1], 2 * (s & 1)), code_pair(kw[u][s >> 1], 2 * (s & 1) + 1));
                }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int r = tile * ROWS + i * 16 + j * 8 + g8, row = r / p.group;
                    const int limit = row < q.n ? row_limit(q, row) : 0;
                    if (limit == 0) continue;
                    const float lse = w.lse[static_cast<size_t>(q.row0 + row) * p.q_heads + head * p.group + r % p.group] * 1.44269504088896340736f;
                    const float sq = sums[i * 16 + j * 8 + g8];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        if (unit[u] == 0xffffffffu) continue;
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const uint32_t pair = c ? kp[u].y : kp[u].x;
                            const float x = fmaf(sc[i][u][2 * j + c], low(pair) * factor, sq * high(pair));
                            if (key0 + 8 * u + 2 * t4 + c < limit) acc[u][c] += ex2(x - lse);
                        }
                    }
                }
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) acc[u][c] += __shfl_xor_sync(0xffffffffu, acc[u][c], d);
            const int slot = key0 + 8 * u + 2 * t4 + c;
            if (g8 == 0 && slot < q.len) {
                float* to = w.weights + static_cast<size_t>(b) * p.s.max_pages * p.s.page_tokens + slot;
                *to = fmaf(w.keep, *to, acc[u][c]);
            }
        }
}

polyspec_status fill(AttendParams* p, const polyspec_cache_pages* s, const polyspec_block_rows* r, const void* q, long long q_stride, int q_heads,
                     int kv_heads, int head_dim, float scale, const void* pool, int32_t* device_status)
{
    polyspec_status st = kv::check_state(s);
    if (st == POLYSPEC_OK) st = kv::check_rows(r);
    if (st == POLYSPEC_OK) st = kv::check_heads(q_heads, kv_heads, head_dim);
    if (st != POLYSPEC_OK) return st;
    if (!kv::rows_ok(q, q_stride, q_heads, head_dim) || !pool || !kv::aligned16(pool) || !aligned4(device_status)) return POLYSPEC_ERR_INVALID_ARG;
    if (!(scale >= -3.0e38f && scale <= 3.0e38f)) return POLYSPEC_ERR_INVALID_ARG;
    const size_t bytes = kv::page_bytes(*s, kv_heads, head_dim);
    if (s->n_pages * (bytes / kv::unit_bytes(head_dim)) >= 0xffffffffull) return POLYSPEC_ERR_UNSUPPORTED;      // units of a plane are counted in 32 bits
    p->s = *s;
    p->r = *r;
    p->q = static_cast<const unsigned short*>(q);
    p->q_stride = q_stride;
    p->q_heads = q_heads; p->kv_heads = kv_heads; p->group = q_heads / kv_heads;
    p->scale_log2 = scale * 1.44269504088896340736f;
    p->pool = static_cast<const unsigned char*>(pool);
    p->plane_bytes = bytes * s->n_pages;
    p->units_per_page = s->page_tokens / kv::kUnit;
    p->status = device_status;
    p->out = nullptr; p->lse = nullptr; p->partial = nullptr; p->joins = nullptr;
    return POLYSPEC_OK;
}

}  // namespace
}  // namespace polyspec

using namespace polyspec;

extern "C" {

polyspec_status polyspec_cache_attention_workspace(int q_heads, int kv_heads, int head_dim, size_t* bytes)
{
    if (!bytes) return POLYSPEC_ERR_INVALID_ARG;
    const polyspec_status st = kv::check_heads(q_heads, kv_heads, head_dim);
    if (st == POLYSPEC_OK) *bytes = align256(attend_bytes(head_dim));
    return st;
}

polyspec_status polyspec_cache_attention(const polyspec_cache_pages* s, const polyspec_block_rows* r, const void* q, long long q_stride, int q_heads,
                                         int kv_heads, int head_dim, float scale, const void* pool, void* out, float* lse, int32_t* device_status,
                                         void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    AttendParams p;
    const polyspec_status st = fill(&p, s, r, q, q_stride, q_heads, kv_heads, head_dim, scale, pool, device_status);
    if (st != POLYSPEC_OK) return st;
    if (!out || !kv::aligned16(out) || !aligned4(lse)) return POLYSPEC_ERR_INVALID_ARG;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return POLYSPEC_ERR_INVALID_ARG;
    if (workspace_bytes < attend_bytes(head_dim)) return POLYSPEC_ERR_WORKSPACE;
    p.out = static_cast<unsigned short*>(out);
    p.lse = lse;
    p.joins = static_cast<int4*>(workspace);
    p.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + align256(kMaxCtas * sizeof(int4)));
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    // rows of a sequence times the heads that share a key head, on average: more than one tile of 16, and two tiles share the codes' expansion
    const bool wide = static_cast<long long>(r->rows) * p.group > 16LL * s->n_seqs;
    cudaError_t e;
    if (head_dim == 128) e = wide ? launch_attend<Shape<128, 2, 4, 5, 2>>(p, stream) : launch_attend<Shape<128, 1, 8, 4, 2>>(p, stream);
    else e = wide ? launch_attend<Shape<64, 2, 8, 4, 2>>(p, stream) : launch_attend<Shape<64, 1, 8, 5, 2>>(p, stream);
    return cuda_failed(e) ? POLYSPEC_ERR_CUDA : POLYSPEC_OK;
}

polyspec_status polyspec_cache_weigh(const polyspec_cache_pages* s, const polyspec_block_rows* r, const void* q, long long q_stride, int q_heads,
                                     int kv_heads, int head_dim, float scale, const void* pool, const float* lse, float keep, float* weights,
                                     int32_t* device_status, void* cuda_stream)
{
    WeighParams w;
    const polyspec_status st = fill(&w.a, s, r, q, q_stride, q_heads, kv_heads, head_dim, scale, pool, device_status);
    if (st != POLYSPEC_OK) return st;
    if (!lse || !weights || !aligned4(lse, weights) || !(keep >= 0.0f && keep <= 1.0f)) return POLYSPEC_ERR_INVALID_ARG;
    const long long chunks = (static_cast<long long>(s->max_pages) * s->page_tokens + kWeighTokens - 1) / kWeighTokens;
    if (s->n_seqs > 65535) return POLYSPEC_ERR_UNSUPPORTED;
    w.lse = lse;
    w.keep = keep;
    w.weights = weights;
    const dim3 grid(static_cast<unsigned>(chunks), static_cast<unsigned>(s->n_seqs));
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = head_dim == 128 ? launch_early(weigh_kernel<128>, grid, kWeighWarps * 32, 0, stream, w)
                                          : launch_early(weigh_kernel<64>, grid, kWeighWarps * 32, 0, stream, w);
    return cuda_failed(e) ? POLYSPEC_ERR_CUDA : POLYSPEC_OK;
}

}  // extern "C"
