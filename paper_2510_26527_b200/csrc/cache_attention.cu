// Attention of a block's rows over a cache held in 4 bits (layout: kv_pages.cuh), and the weight that each cached token was given.
//
//   s[r, j] = scale * q[r] . K[j],  K[j] = ks[j] * ck[j] + ko[j];  out[r] = sum_j softmax_j(s)[r, j] V[j],  V[j] = vs[j] * cv[j] + vo[j]
//
// The matrix instructions multiply codes, never dequantised numbers:
//   s[r, j] = ks[j] * (q[r] . ck[j]) + ko[j] * sum(q[r])                        one product and one FMA per (row, token)
//   out[r]  = (sum_j (p[r, j] vs[j]) cv[j] + sum_j p[r, j] vo[j]) / sum_j p[r, j],     p = 2^(s - m)
// with m near the running maximum of s.  p and both sums of p are fp32; only the products p vs are rounded, to fp16, times a power of two that
// keeps a row's largest at 2^3 or more: what it loses of the others is small beside the largest, whatever their scales.
//
// A code is an fp16 number without any arithmetic: four bits under a mask are a subnormal, code * 2^-24, and the same mask four
// bits higher gives 16 * code * 2^-24.  Matrix instructions multiply subnormals exactly; the 16 goes into the query's elements
// (as 1/16) or out of the finished sums.  So eight codes cost four masks and one shift (keys), and two byte permutes more per sixteen
// where pairs of tokens have to be brought together (values).  Queries are scaled by a power of two into fp16's upper range, where their
// bf16 digits are exact down to 2^-28 of the block's largest.
//
// mma.sync with tokens and elements as the 16 rows of its A operand and the block's rows as its 8 columns: a block's rows times the heads that
// share a key head are 4 to 36, so the columns are well filled, a lane has the scales of two tokens only, and softmax weights change from the first
// product's layout to the second's with one movmatrix per 8 x 8.  (tcgen05's tiles of 128 rows would be mostly empty, and its operands would have to
// be expanded through shared or tensor memory.)
//
// Work: (sequence, key head, row tile) are segments of `steps` of 32 tokens per warp; the steps of all segments, one after the other, are cut into equal
// shares, one per CTA, whatever the lengths; what a segment costs besides its steps counts as kOverhead of them.  Each warp streams its tokens through
// a ring of its own (bulk copies of one or two units) and keeps maximum, sums and the output tile in registers; a segment's warps meet once at its
// end.  A segment that crosses CTAs leaves partial results, which a second kernel joins.
//
// Measured (B200): one token over 4000 12.5 us, most of it two launches' dependent look-ups; single tokens of 16 sequences of up to 65536 tokens, 350 MB of
// pages, 84.5 us, 4.1 TB/s (the copies alone 60; with two stages none is under way while a warp computes); blocks of 4 to 9 rows of 64 sequences of up to 8192
// tokens, 428 MB, 263 us: bound by the latency of products, exponentials and products one behind the other, half of the issue slots used, with three warps per
// scheduler that the output tile's registers leave (with the pages in L2 hardly less: 272 against 277 of an earlier form).  A variant on tcgen05, tokens as
// the rows of a tile of 128, took 367: its sixteen and more warps' waits and look-ups per step cost as many instructions as the products they save.
#include <cuda_fp16.h>

#include "kv_pages.cuh"
#include "number_pairs.cuh"
#include "tensor_device.cuh"

namespace polyspec {
namespace {

using namespace numbers;

using tensordev::mbar_expect_tx;
using tensordev::mbar_init;
using tensordev::mbar_try;
using tensordev::smem_addr;

constexpr int kMaxCtas = 608;                   // CTAs that the workspace has room for
constexpr int kOverhead = 4;                    // steps' worth of work that a segment costs besides its steps: its rows, the meeting of its warps
constexpr float kNone = -3.0e38f;               // a maximum over nothing
constexpr float kLift = 3.0f;                   // a row's largest product of weight and scale is 2^3 when its reference is set
constexpr float kSlack = 12.0f;                 // and may rise to 2^15, near fp16's end, before sums are rescaled
// Scales from 2^-24 to 2^40 need no units: the largest weight is between 2^-37 and 2^27 when the reference is set (so what is lost below 2^-126 is 2^-89 of it at most),
// and weights stay below 2^39, which leaves values of up to 2^64 room for their sums in fp32.
constexpr float kLeastScale = -24.0f, kMostScale = 40.0f;
constexpr float kMostUnit = 126.0f;             // units are 2^-126 to 2^126

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
    int4* joins;                                // [2 * CTAs]: of the segment that begins in a CTA and ends elsewhere (parts, rows of its tile, key head, first row), its
                                                // sequence's rows (first row of the tensors, rows, slot, granted)
    int32_t* status;
};

__device__ __forceinline__ uint32_t half2_bits(float a, float b)
{
    const __half2 x = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&x);
}

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Pair i (0..3) of a word's codes as two fp16 numbers: elements 2i, 2i+1 for keys.  Odd pairs come 16-fold.
__device__ __forceinline__ uint32_t code_pair(uint32_t word, int i) { return (i >= 2 ? word >> 8 : word) & (i & 1 ? 0x00f000f0u : 0x000f000fu); }

// The 8 x 8 matrix of 16-bit numbers whose rows the lanes hold in pairs, transposed.
__device__ __forceinline__ uint32_t transpose(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void copy_bulk(uint32_t to, const void* from, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
}

// Rows of a tile as the B operand of the first product, [8-row groups][D / 16][32 lanes] pairs of words.  The element order inside a step of 16
// follows the codes' (words are dealt out to lanes whole); elements whose codes come 16-fold are divided by 16.  x: eight elements of row r.
template <int D>
__device__ __forceinline__ void store_fragment(uint32_t* frag, int r, int word, const float* x, float by)
{
    constexpr int kWords = D / 32;              // words of a token per lane
    const int t = word / kWords, w = word % kWords, lane = (r & 7) * 4 + t;
    uint2* to = reinterpret_cast<uint2*>(frag) + ((r >> 3) * (D / 16) + 2 * w) * 32 + lane;
    const float by16 = by * 0.0625f;
    to[0] = make_uint2(half2_bits(x[0] * by, x[1] * by), half2_bits(x[2] * by16, x[3] * by16));
    to[32] = make_uint2(half2_bits(x[4] * by, x[5] * by), half2_bits(x[6] * by16, x[7] * by16));
}

// The power of two that brings numbers of up to `top` in size into [2^14, 2^15), and what their products with codes (which bring 2^-24) are to be multiplied with.
__device__ __forceinline__ float row_scale(const AttendParams& p, float top, float* factor)
{
    const int k = top > 0.0f ? max(-100, static_cast<int>(__float_as_uint(top) >> 23) - 127) : 0;          // top in [2^k, 2^(k+1))
    *factor = p.scale_log2 * 1024.0f * __uint_as_float(static_cast<uint32_t>(k + 127) << 23);              // (2^(10 + k) alone may be past fp32)
    return __uint_as_float(static_cast<uint32_t>(14 - k + 127) << 23);
}

// The rows of a tile into shared memory, by all THREADS of a CTA: rows row0 .. row0 + ROWS - 1 of (row of the block, head of the group), zeros from
// `end` on.  sums[r] = scale * log2(e) * sum of the row; *factor = what a product of fragments and codes is multiplied with.  Ends with the CTA in step.
template <int D, int ROWS, int THREADS>
__device__ __forceinline__ void load_rows(const AttendParams& p, const kv::SeqRows& q, int kv_head, int row0, int end, uint32_t* frag, float* sums,
                                          float* warp_max, float* factor)
{
    constexpr int kVecs = D / 8, kItems = ROWS * kVecs, kPer = (kItems + THREADS - 1) / THREADS;
    static_assert(kItems % THREADS == 0 || (kPer == 1 && kItems % 32 == 0), "whole warps take part or none");
    uint4 raw[kPer];
    float top = 0.0f;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int item = u * THREADS + threadIdx.x, r = row0 + item / kVecs, i = r / p.group;
        raw[u] = make_uint4(0, 0, 0, 0);
        if (item < kItems && r < end) raw[u] = *reinterpret_cast<const uint4*>(p.q + (q.row0 + i) * p.q_stride + (kv_head * p.group + r % p.group) * D + item % kVecs * 8);
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
    const float by = row_scale(p, top, factor);
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int item = u * THREADS + threadIdx.x, r = item / kVecs;
        if (item >= kItems) break;
        const uint32_t* y = reinterpret_cast<const uint32_t*>(&raw[u]);
        float x[8], sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[2 * e] = low(y[e]); x[2 * e + 1] = high(y[e]); sum = fmaf(x[2 * e], p.scale_log2, fmaf(x[2 * e + 1], p.scale_log2, sum)); }
        store_fragment<D>(frag, r, item % kVecs, x, by);
#pragma unroll
        for (int d = 1; d < kVecs; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (item % kVecs == 0) sums[r] = sum;
    }
    __syncthreads();
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

// NT: groups of 8 rows in a tile.
template <int D_, int NT_, int WARPS_, int STAGES_, int CTAS_>
struct Shape {
    static constexpr int D = D_, NT = NT_, WARPS = WARPS_, STAGES = STAGES_, CTAS = CTAS_;
    static constexpr int THREADS = WARPS * 32, ROWS = NT * 8, STEP = WARPS * 32;        // STEP: tokens
    static constexpr int UB = kv::unit_bytes(D), STAGE = 8 * UB, M = D / 16;            // M: 16-element groups of the output
    static constexpr int FRAG = NT * (D / 16) * 256;                                    // bytes
    static constexpr int RING = WARPS * STAGES * STAGE;
    static constexpr int MERGE = WARPS / 2 * NT * M * 512;
    static constexpr size_t SMEM = FRAG + RING + MERGE;
    static constexpr int PART = ROWS * (D + 2);                                         // floats of a partial result
    static_assert(SMEM * CTAS <= 220 * 1024, "shared memory");
};

// All sequences' steps and overheads one behind the other, cut into equal shares.  share[0], share[1]: this CTA's first place and the one behind its last;
// seq, within: the sequence that holds the first, the place within it.  False where there is nothing left for this CTA.  Every thread calls it.
struct Share { long long total, ctas, begin, end, within; int seq; };
template <class S>
__device__ __forceinline__ bool find_share(const AttendParams& p, Share* share /* shared memory */, long long* warp_sums, Share& mine)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long carry = 0, first_start = 0, first_n = 0;      // of the first S::THREADS sequences: often all there are
    auto places = [&](int b) {
        Segment g;
        g.q = kv::seq_rows(p.s, p.r, b);
        if (g.q.bad && blockIdx.x == 0) kv::report(p.status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE);
        seq_segments<S::ROWS, S::STEP>(p, g);
        return static_cast<long long>(g.tiles) * (g.steps + kOverhead) * p.kv_heads;
    };
    // where sequence b's places begin; carry: the sequences' before this round
    auto start_of = [&](long long n) {
        long long inc = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, inc, d);
            if (lane >= d) inc += y;
        }
        __syncthreads();
        if (lane == 31) warp_sums[warp] = inc;
        __syncthreads();
        long long start = carry + inc - n;
        for (int w = 0; w < S::WARPS; ++w) {
            if (w < warp) start += warp_sums[w];
            carry += warp_sums[w];
        }
        return start;
    };
    for (int b0 = 0; b0 < p.s.n_seqs; b0 += S::THREADS) {
        const int b = b0 + threadIdx.x;
        const long long n = b < p.s.n_seqs ? places(b) : 0, start = start_of(n);
        if (b0 == 0) { first_start = start; first_n = n; }
    }
    mine.total = carry;
    mine.ctas = min(carry, static_cast<long long>(gridDim.x));
    if (blockIdx.x >= mine.ctas) return false;
    mine.begin = mine.total * blockIdx.x / mine.ctas;
    mine.end = mine.total * (blockIdx.x + 1) / mine.ctas;
    auto look = [&](int b, long long start, long long n) {
        if (n > 0 && start <= mine.begin && mine.begin < start + n) { share->seq = b; share->within = mine.begin - start; }
    };
    look(threadIdx.x, first_start, first_n);
    carry = 0;
    if (p.s.n_seqs > S::THREADS)
        for (int b0 = 0; b0 < p.s.n_seqs; b0 += S::THREADS) {
            const int b = b0 + threadIdx.x;
            const long long n = b < p.s.n_seqs ? places(b) : 0, start = start_of(n);
            if (b0 > 0) look(b, start, n);
        }
    __syncthreads();
    mine.seq = share->seq;
    mine.within = share->within;
    return true;
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

// Normalised outputs of eight neighbouring elements of a row; zeros where it attends to nothing, or none of what it attends to could be read.
__device__ __forceinline__ void store_out(const AttendParams& p, const kv::SeqRows& q, int kv_head, int r, int D, int d0, const float* x, float m, float l)
{
    const int i = r / p.group;
    if (i >= q.n) return;
    const size_t at = static_cast<size_t>(q.row0 + i) * p.q_heads + kv_head * p.group + r % p.group;
    const bool none = row_limit(q, i) == 0 || l == 0.0f;
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

// What a warp keeps of its tile.  Per row: the reference of the weights p = 2^(score - reference), with its sign turned; their sum l and the sum lo of p vo; and the
// output, elements x rows in the codes' form, the sum of p vs unit cv.  A power of two, `unit`, is 1 as long as one reference serves both: then it brings p vs into
// fp16's range.  Where scales are too far from 1 for that the reference follows the weights alone, and the unit the products.
// NT groups of 8 rows; a lane has rows 2 t4 and 2 t4 + 1 of each, as pairs.
template <class S>
struct Running { float o[S::NT][S::M][4]; uint64_t ref[S::NT], unit[S::NT], l[S::NT], lo[S::NT]; bool started, units; };

__device__ __forceinline__ float exponent(float x) { return static_cast<float>(static_cast<int>(__float_as_uint(x) >> 23 & 255u) - 127); }

// The largest of a row's numbers, over its tokens.
template <int T>
__device__ __forceinline__ float row_max(const float (&y)[T][2], float top)
{
#pragma unroll
    for (int v = 0; v < T; ++v) top = max3(top, y[v][0], y[v][1]);
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    return top;
}

// Rows' references rise by `up`: exponents, sums and output follow, the output by a factor of its own.
template <class S, int T>
__device__ __forceinline__ void follow(Running<S>& run, uint64_t (&x)[T][S::NT][2], int n, const float (&up)[2], const float (&by)[2], const float (&by_o)[2])
{
    const uint64_t less = pair(-up[0], -up[1]), by2 = pair(by[0], by[1]);
#pragma unroll
    for (int v = 0; v < T; ++v) { x[v][n][0] = add2(x[v][n][0], less); x[v][n][1] = add2(x[v][n][1], less); }
    run.ref[n] = add2(run.ref[n], less);
    run.l[n] = mul2(run.l[n], by2);
    run.lo[n] = mul2(run.lo[n], by2);
#pragma unroll
    for (int i = 0; i < S::M; ++i) { run.o[n][i][0] *= by_o[0]; run.o[n][i][1] *= by_o[1]; run.o[n][i][2] *= by_o[0]; run.o[n][i][3] *= by_o[1]; }
}

// References and units that fit the tokens at hand: x, exponents of their weights, less the old references (-inf: not seen), and vs, the values' scales.
// (A row that sees none of its warp's first tokens sees none of the later ones either.)  A head of equal elements has codes of 0 and a scale that says nothing, 1 from
// the append: it gets a scale of 0 (lv: -inf), or it would take the bits of others that are smaller.  `values`: the stage's units.
template <class S, int T>
__device__ __forceinline__ void set_references(Running<S>& run, uint64_t (&x)[T][S::NT][2], float (&vs)[T][2], const unsigned char* values, int lane)
{
    // a lane has words of tokens 2 t4 and 2 t4 + 1 here, of token g8 elsewhere
    constexpr int kWords = S::D / 64;
    uint32_t some[T][2][2];
    bool zeros = false;
#pragma unroll
    for (int v = 0; v < T; ++v)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t* words = reinterpret_cast<const uint32_t*>(values + (2 * v + u) * S::UB) + lane * 2 * kWords;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                some[v][u][i] = kWords == 2 ? words[2 * i] | words[2 * i + 1] : words[i];
                zeros = zeros || some[v][u][i] == 0;
            }
        }
    const bool first = !run.started;
    float lv[T][2];
    bool tame = !run.units;
#pragma unroll
    for (int v = 0; v < T; ++v) { lv[v][0] = lg2(vs[v][0]); lv[v][1] = lg2(vs[v][1]); }
    if (__any_sync(0xffffffffu, zeros)) {
#pragma unroll
        for (int v = 0; v < T; ++v)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t tokens[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    tokens[i] = __ballot_sync(0xffffffffu, some[v][u][i] != 0);
                    tokens[i] |= tokens[i] >> 16;
                    tokens[i] |= tokens[i] >> 8;
                    tokens[i] |= tokens[i] >> 4;
                }
                const int token = lane >> 2;
                if (!((token & 1 ? tokens[1] : tokens[0]) >> (token >> 1) & 1u) && vs[v][u] <= 3.4e38f) { vs[v][u] = 0.0f; lv[v][u] = -INFINITY; }
            }
    }
#pragma unroll
    for (int v = 0; v < T; ++v)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float most = -INFINITY;
#pragma unroll
            for (int n = 0; n < S::NT; ++n) {
                float a, b;
                unpair(x[v][n][u], &a, &b);
                most = max3(most, a, b);
            }
            tame = tame && (most == -INFINITY || !(lv[v][u] < kLeastScale || lv[v][u] > kMostScale));
        }
    run.started = true;
    if (__builtin_expect(__all_sync(0xffffffffu, tame), 1)) {
#pragma unroll
        for (int n = 0; n < S::NT; ++n) {
            float up[2], by[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float y[T][2];
#pragma unroll
                for (int v = 0; v < T; ++v)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        float a, b;
                        unpair(x[v][n][u], &a, &b);
                        y[v][u] = (j ? b : a) + lv[v][u];           // (NaN, of a hidden token's scale, is never the largest)
                    }
                const float top = row_max(y, -INFINITY);            // the largest product is 2^top
                up[j] = top == -INFINITY ? 0.0f : first ? top - kLift : fmaxf(top - kLift, 0.0f);
                by[j] = first ? 1.0f : ex2(-up[j]);
            }
            run.unit[n] = pair(1.0f, 1.0f);
            follow<S, T>(run, x, n, up, by, by);
        }
        return;
    }
    bool units = false;
#pragma unroll
    for (int n = 0; n < S::NT; ++n) {
        float up[2], by[2], by_o[2], unit[2], l[2];
        unpair(run.unit[n], &unit[0], &unit[1]);
        unpair(run.l[n], &l[0], &l[1]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            // The row's largest weight, of these tokens or (by their sum) of those before, is 2^top; these tokens' largest product 2^h of that, in the output's
            // unit 2^(top + h + e).  Before a row's first product its unit is the largest.
            float y[T][2], w[T][2];
#pragma unroll
            for (int v = 0; v < T; ++v)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float a, b;
                    unpair(x[v][n][u], &a, &b);
                    y[v][u] = j ? b : a;
                }
            float top = row_max(y, lg2(l[j]));           // (-inf where there were none)
            const bool sees = top > -INFINITY;
            top = sees ? ceilf(top) : 0.0f;
#pragma unroll
            for (int v = 0; v < T; ++v)
#pragma unroll
                for (int u = 0; u < 2; ++u) w[v][u] = ex2(y[v][u] - top) * vs[v][u];
            const float heavy = row_max(w, 0.0f), h = exponent(heavy), e = first ? 0.0f : exponent(unit[j]);
            const bool none = first && heavy == 0.0f, anew = !none && (first || top + h + e > kLift + 5.0f);
            // with a unit of 1 the largest weight would be 2^most; else it becomes 2^-5
            const float most = anew ? kLift - h : top + e, fall = anew ? top + h + e - kLift : 0.0f;
            const bool one = none ? !sees : most >= kLift - kMostScale && most <= kLift - kLeastScale;
            const float wanted = one ? 0.0f : none ? kMostUnit : most + 5.0f, to = fminf(fmaxf(wanted, -kMostUnit), kMostUnit);
            up[j] = one && !none ? top - most : top + 5.0f;
            unit[j] = __uint_as_float(static_cast<uint32_t>(static_cast<int>(to) + 127) << 23);
            by[j] = first ? 1.0f : ex2(-up[j]);
            by_o[j] = first ? 1.0f : ex2(to - wanted - fall);
            units = units || !one;
        }
        run.unit[n] = pair(unit[0], unit[1]);
        follow<S, T>(run, x, n, up, by, by_o);
    }
    run.units = __any_sync(0xffffffffu, units);
}

// A stage's 32 tokens, 16 at a time side by side (two chains of products hide each other's latency: 276 -> 259 us on blocks of 4 to 9 rows).  `at`: the stage,
// 4 units of keys, 4 of values.  masked: some row does not see some token, or a unit could not be read (bad).  q0: the rows' fragments where they stay in
// registers (one group of rows).  All groups of rows are computed, live or not: branches around those that are not cost more than they save.
template <class S>
__device__ __forceinline__ void attend_tokens(const AttendParams& p, Running<S>& run, const unsigned char* at, const uint32_t* frag, const uint2* q0, const float* sums,
                                              float factor, bool masked, uint32_t bad, int key0, const Segment& seg, int lane)
{
    constexpr int D = S::D, KS = D / 16, M = S::M, UB = S::UB, WORDS = D / 32, H = D / 64, L = S::NT, T = 2;
    const int g8 = lane >> 2, t4 = lane & 3;
    // codes of keys, and the first product: tokens x rows
    float sc[T][L][4];
#pragma unroll
    for (int v = 0; v < T; ++v) {
        uint32_t kw[2][WORDS];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const unsigned char* unit = at + (2 * v + u) * UB;
            if (D == 128) {
                const uint4 x = *reinterpret_cast<const uint4*>(unit + lane * 16);
                kw[u][0] = x.x; kw[u][1] = x.y; kw[u][WORDS - 2] = x.z; kw[u][WORDS - 1] = x.w;
            } else {
                const uint2 x = *reinterpret_cast<const uint2*>(unit + lane * 8);
                kw[u][0] = x.x; kw[u][1] = x.y;
            }
        }
#pragma unroll
        for (int n = 0; n < L; ++n) sc[v][n][0] = sc[v][n][1] = sc[v][n][2] = sc[v][n][3] = 0.0f;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const uint32_t a0 = code_pair(kw[0][s >> 1], 2 * (s & 1)), a1 = code_pair(kw[1][s >> 1], 2 * (s & 1));
            const uint32_t a2 = code_pair(kw[0][s >> 1], 2 * (s & 1) + 1), a3 = code_pair(kw[1][s >> 1], 2 * (s & 1) + 1);
#pragma unroll
            for (int n = 0; n < L; ++n) {
                const uint2 b = S::NT == 1 ? q0[S::NT == 1 ? s : 0] : reinterpret_cast<const uint2*>(frag)[(n * KS + s) * 32 + lane];
                mma(sc[v][n], a0, a1, a2, a3, b.x, b.y);
            }
        }
    }
    // scales and offsets of the lane's tokens g8 and g8 + 8; exponents of their weights, less the references, rows in pairs
    uint64_t x[T][L][2];
    float vs[T][2], vo[T][2], most = -INFINITY, scale = 0x1p-24f;       // (the least: so the bound below holds weights under 2^39, too)
#pragma unroll
    for (int v = 0; v < T; ++v) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const unsigned char* pairs = at + (2 * v + u) * UB + 4 * D + g8 * 4;
            const uint32_t kp = *reinterpret_cast<const uint32_t*>(pairs), vp = *reinterpret_cast<const uint32_t*>(pairs + 4 * UB);
            const float ks = low(kp) * factor, ko = high(kp);
            vs[v][u] = low(vp);
            vo[v][u] = high(vp);
            const uint64_t ks2 = pair(ks, ks), ko2 = pair(ko, ko);
#pragma unroll
            for (int n = 0; n < L; ++n) {
                const uint64_t sq = *reinterpret_cast<const uint64_t*>(&sums[n * 8 + 2 * t4]);
                x[v][n][u] = fma2(pair(sc[v][n][2 * u], sc[v][n][2 * u + 1]), ks2, fma2(sq, ko2, run.ref[n]));
            }
        }
        scale = max3(scale, vs[v][0], vs[v][1]);
    }
    uint32_t hidden[T] = {};                    // bit 4 n + 2 u + j
    if (__builtin_expect(masked, 0)) {
#pragma unroll
        for (int v = 0; v < T; ++v) {
#pragma unroll
            for (int n = 0; n < L; ++n) {
                const int r = seg.tile * seg.tile_rows + n * 8 + 2 * t4, limit0 = row_limit(seg.q, r / p.group), limit1 = row_limit(seg.q, (r + 1) / p.group);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int key = key0 + 16 * v + 8 * u + g8;
                    const bool gone = bad >> (2 * v + u) & 1u, h0 = gone || key >= limit0, h1 = gone || key >= limit1;
                    float a, b;
                    unpair(x[v][n][u], &a, &b);
                    x[v][n][u] = pair(h0 ? -INFINITY : a, h1 ? -INFINITY : b);
                    hidden[v] |= (h0 ? 1u : 0u) << (4 * n + 2 * u) | (h1 ? 2u : 0u) << (4 * n + 2 * u);
                }
            }
        }
    }
#pragma unroll
    for (int v = 0; v < T; ++v)
#pragma unroll
        for (int n = 0; n < L; ++n)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float a, b;
                unpair(x[v][n][u], &a, &b);
                most = max3(most, a, b);
            }
    // The first tokens set the references; after that sums are rescaled only when a product may have risen by 2^kSlack since the last time, by a bound of the largest
    // weight and the largest scale of a lane's tokens.  With units every stage is looked at exactly.
    if (__builtin_expect(__any_sync(0xffffffffu, !run.started || run.units || most + lg2(scale) > kLift + kSlack), 0)) set_references<S, T>(run, x, vs, at + 4 * UB, lane);
    uint32_t pr[T][L][2];
    if (__builtin_expect(!masked && !run.units, 1)) {
#pragma unroll
        for (int v = 0; v < T; ++v)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint64_t vs2 = pair(vs[v][u], vs[v][u]), vo2 = pair(vo[v][u], vo[v][u]);
#pragma unroll
                for (int n = 0; n < L; ++n) {
                    float a, b;
                    unpair(x[v][n][u], &a, &b);
                    const uint64_t weight = pair(ex2(a), ex2(b));
                    run.l[n] = add2(run.l[n], weight);
                    run.lo[n] = fma2(weight, vo2, run.lo[n]);
                    unpair(mul2(weight, vs2), &a, &b);
                    pr[v][n][u] = transpose(half2_bits(a, b));
                }
            }
    } else {                                    // scales and offsets behind what a row sees may be anything
#pragma unroll
        for (int v = 0; v < T; ++v)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int n = 0; n < L; ++n) {
                    const bool h0 = hidden[v] >> (4 * n + 2 * u) & 1u, h1 = hidden[v] >> (4 * n + 2 * u) & 2u;
                    float a, b;
                    unpair(x[v][n][u], &a, &b);
                    const uint64_t weight = pair(ex2(a), ex2(b));
                    run.l[n] = add2(run.l[n], weight);
                    run.lo[n] = fma2(weight, pair(h0 ? 0.0f : vo[v][u], h1 ? 0.0f : vo[v][u]), run.lo[n]);
                    unpair(mul2(mul2(weight, pair(h0 ? 0.0f : vs[v][u], h1 ? 0.0f : vs[v][u])), run.unit[n]), &a, &b);
                    pr[v][n][u] = transpose(half2_bits(a, b));
                }
    }
    // codes of values: words of tokens 2 t4 and 2 t4 + 1, paired by token, and the second product: elements x rows
#pragma unroll
    for (int v = 0; v < T; ++v) {
        uint32_t even[2][H], odd[2][H];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const unsigned char* unit = at + (4 + 2 * v + u) * UB;
            if (D == 128) {
                const uint4 x = *reinterpret_cast<const uint4*>(unit + lane * 16);
                even[u][0] = __byte_perm(x.x, x.z, 0x5410); odd[u][0] = __byte_perm(x.x, x.z, 0x7632);
                even[u][H - 1] = __byte_perm(x.y, x.w, 0x5410); odd[u][H - 1] = __byte_perm(x.y, x.w, 0x7632);
            } else {
                const uint2 x = *reinterpret_cast<const uint2*>(unit + lane * 8);
                even[u][0] = __byte_perm(x.x, x.y, 0x5410); odd[u][0] = __byte_perm(x.x, x.y, 0x7632);
            }
        }
#pragma unroll
        for (int i = 0; i < M; ++i) {
            // the product's rows: elements 8 g8 + i and 64 + 8 g8 + i, or of narrow heads 8 g8 + i and 8 g8 + 4 + i
            const int e0 = i, e1 = D == 128 ? i : i + 4, h1 = H - 1;
            const uint32_t a0 = code_pair(e0 & 1 ? odd[0][0] : even[0][0], e0 >> 1), a1 = code_pair(e1 & 1 ? odd[0][h1] : even[0][h1], e1 >> 1);
            const uint32_t a2 = code_pair(e0 & 1 ? odd[1][0] : even[1][0], e0 >> 1), a3 = code_pair(e1 & 1 ? odd[1][h1] : even[1][h1], e1 >> 1);
#pragma unroll
            for (int n = 0; n < L; ++n) mma(run.o[n][i], a0, a1, a2, a3, pr[v][n][0], pr[v][n][1]);
        }
    }
}

template <class S>
__global__ void __launch_bounds__(S::THREADS, S::CTAS) attend_kernel(const AttendParams p)
{
    constexpr int D = S::D, NT = S::NT, W = S::WARPS, NS = S::STAGES, KS = D / 16, M = S::M, UB = S::UB, H = D / 64;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ long long warp_sums[W];
    __shared__ Share found;
    __shared__ __align__(16) float sums[S::ROWS];            // read in pairs
    __shared__ float warp_max[W], sm_m[W][S::ROWS], sm_l[W][S::ROWS], sm_o[W][S::ROWS];
    __shared__ __align__(8) uint64_t barriers[W * NS];
    __shared__ Segment mine, produced[W];       // the segment at hand; the one that each warp's copies have come to
    __shared__ int produced_visible[W];
    uint32_t* frag = reinterpret_cast<uint32_t*>(smem);
    float4* merge = reinterpret_cast<float4*>(smem + S::FRAG + S::RING);
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, g8 = lane >> 2, t4 = lane & 3;
    unsigned char* ring = smem + S::FRAG + warp * NS * S::STAGE;
    const uint32_t ring_at = smem_addr(ring), bar_at = smem_addr(&barriers[warp * NS]);
    if (lane == 0) {
        for (int i = 0; i < NS; ++i) mbar_init(bar_at + 8u * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncwarp();
    wait_for_stream();

    if (threadIdx.x == 0) p.joins[2 * blockIdx.x] = make_int4(0, 0, 0, 0);
    Share share;
    if (!find_share<S>(p, &found, warp_sums, share)) return;
    const long long s0 = share.begin, s1 = share.end, total = share.total, ctas = share.ctas, within = share.within;
    const int seq = share.seq;
    int step, left;                             // left: places up to s1 (a step's, and an overhead's at each new segment)
    {
        Segment g;
        g.b = seq;
        g.q = kv::seq_rows(p.s, p.r, seq);
        seq_segments<S::ROWS, S::STEP>(p, g);
        const int span = g.steps + kOverhead, n = static_cast<int>(within / span);
        g.head = n / g.tiles;
        g.tile = n % g.tiles;
        const int into = static_cast<int>(within % span) - kOverhead;       // negative: before the segment's first step
        step = max(into, 0);
        left = static_cast<int>(s1 - s0) + min(into, 0);
        if (left <= 0) return;
        if (threadIdx.x == 0) mine = g;
        if (lane == 0) { produced[warp] = g; produced_visible[warp] = visible(p, g); }
        __syncthreads();
    }
    int ahead_step = step, ahead_steps = mine.steps, ahead_left = left;

    // lane 4 k + u: unit u of the warp's k-th stage from here on, as a number of units in a plane, or ~0
    uint32_t unit_numbers = 0;
    int unit_k = 8;                             // stages of `unit_numbers` that are used up
    uint32_t bad_units = 0;                     // bit 4 stage + u: nothing could be read there

    // Copies of the next stage: lanes 0 .. 3 a unit of keys each, 4 .. 7 of values; a unit that follows its even neighbour's in memory goes with it.
    auto issue = [&](int stage) {
        if (unit_k == 8) {
            const long long slot = (static_cast<long long>(ahead_step + (lane >> 2)) * W + warp) * 32 + (lane & 3) * 8;
            unit_numbers = 0xffffffffu;
            if (slot < produced_visible[warp]) {
                const Segment& ahead = produced[warp];
                const int unit = static_cast<int>(slot >> 3), at = unit / p.units_per_page;
                const int page = p.s.table[static_cast<size_t>(ahead.b) * p.s.max_pages + at];
                if (page >= 0 && page < p.s.n_pages)
                    unit_numbers = (static_cast<uint32_t>(page) * p.kv_heads + ahead.head) * p.units_per_page + (unit - at * p.units_per_page);
                else
                    kv::report(p.status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE);
            }
            unit_k = 0;
        }
        const uint32_t number = __shfl_sync(0xffffffffu, unit_numbers, 4 * unit_k + (lane & 3));
        const uint32_t neighbour = __shfl_xor_sync(0xffffffffu, number, 1);
        const bool there = number != 0xffffffffu, odd = lane & 1;
        const bool together = odd ? number == neighbour + 1 && neighbour != 0xffffffffu : neighbour == number + 1 && there && neighbour != 0xffffffffu;
        const uint32_t units = __ballot_sync(0xffffffffu, there) & 15u;
        bad_units = (bad_units & ~(15u << (4 * stage))) | (15u ^ units) << (4 * stage);
        const uint32_t bar = bar_at + 8u * stage;
        if (lane == 0) mbar_expect_tx(bar, 2 * UB * __popc(units));
        __syncwarp();
        if (lane < 8 && there && !(odd && together))
            copy_bulk(ring_at + stage * S::STAGE + lane * UB, p.pool + static_cast<size_t>(number) * UB + (lane < 4 ? 0 : p.plane_bytes), together ? 2 * UB : UB, bar);
        ++unit_k;
        --ahead_left;
        if (++ahead_step == ahead_steps) {
            __syncwarp();
            if (lane == 0) {
                Segment g = produced[warp];
                next_segment<S>(p, g);
                produced[warp] = g;
                produced_visible[warp] = visible(p, g);
            }
            __syncwarp();
            ahead_step = 0;
            ahead_steps = produced[warp].steps;
            ahead_left -= kOverhead;
            unit_k = 8;
        }
    };

    int issued = 0;
    for (; issued < NS - 1 && ahead_left > 0; ++issued) issue(issued);

    Running<S> run;
    uint2 q0[NT == 1 ? KS : 1];                 // of a tile of one group of rows the fragments stay in registers
    int seen = 0, stage = 0;
    uint32_t phase = 0;
    bool from_start = step == 0, fresh = true, ok = true;
    float factor = 0.0f;
    int steps = 0, all_see = 0;                 // of the segment; tokens that every row sees
    while (left > 0) {
        if (fresh) {
            __syncthreads();                    // the segment has been written
            steps = mine.steps;
            all_see = mine.q.base + 1;
            const int row0 = mine.tile * mine.tile_rows, end = min(mine.q.n * p.group, row0 + mine.tile_rows);
            load_rows<D, S::ROWS, S::THREADS>(p, mine.q, mine.head, row0, end, frag, sums, warp_max, &factor);
            seen = visible(p, mine);
            if (NT == 1) {
#pragma unroll
                for (int s = 0; s < KS; ++s) q0[NT == 1 ? s : 0] = reinterpret_cast<const uint2*>(frag)[s * 32 + lane];
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                run.ref[n] = run.unit[n] = run.l[n] = run.lo[n] = 0;
#pragma unroll
                for (int i = 0; i < M; ++i) run.o[n][i][0] = run.o[n][i][1] = run.o[n][i][2] = run.o[n][i][3] = 0.0f;
            }
            run.started = run.units = false;
            fresh = false;
        }
        if (ok) {                               // a bounded wait, passed or given up by the whole warp
            uint32_t i = 0;
            while (i < tensordev::kSpinLimitG && !mbar_try(bar_at + 8u * stage, phase)) ++i;
            ok = __all_sync(0xffffffffu, i < tensordev::kSpinLimitG);
        }
        const int key0 = (step * W + warp) * 32;
        const uint32_t bad = bad_units >> (4 * stage) & 15u;
        if (key0 < seen && ok && bad != 15u) {
            const unsigned char* at = ring + stage * S::STAGE;
            const bool masked = key0 + 32 > all_see || bad;
            attend_tokens<S>(p, run, at, frag, q0, sums, factor, masked, bad, key0, mine, lane);
        }
        __syncwarp();
        // the stage that was read before this one is free again
        if (ahead_left > 0 && ok) { issue(stage == 0 ? NS - 1 : stage - 1); ++issued; }
        if (++stage == NS) { stage = 0; phase ^= 1u; }
        --left;
        ++step;
        if (step < steps && left > 0) continue;

        // the segment, or this CTA's part of it, is done: its warps meet
        const bool whole = from_start && step == steps;
        const int row0 = mine.tile * mine.tile_rows, end = min(mine.q.n * p.group, row0 + mine.tile_rows);
        float ref[NT][2], l[NT][2], lo[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            unpair(run.ref[n], &ref[n][0], &ref[n][1]);
            unpair(run.l[n], &l[n][0], &l[n][1]);
            unpair(run.lo[n], &lo[n][0], &lo[n][1]);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    l[n][j] += __shfl_xor_sync(0xffffffffu, l[n][j], d);
                    lo[n][j] += __shfl_xor_sync(0xffffffffu, lo[n][j], d);
                }
                ref[n][j] = l[n][j] == 0.0f ? kNone : -ref[n][j];       // kNone: saw nothing
                if (g8 == 0) sm_m[warp][n * 8 + 2 * t4 + j] = ref[n][j];
            }
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float unit[2];
            unpair(run.unit[n], &unit[0], &unit[1]);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = n * 8 + 2 * t4 + j;
                float top = kNone;
#pragma unroll
                for (int w = 0; w < W; ++w) top = fmaxf(top, sm_m[w][r]);
                const float by = ex2(ref[n][j] - top);
                if (g8 == 0) { sm_l[warp][r] = l[n][j] * by; sm_o[warp][r] = lo[n][j] * by; }
                // out of the unit, and with what the codes' form left out: 2^24, for 16-fold codes 2^20
                const float inverse = __uint_as_float(0x7f000000u - __float_as_uint(unit[j])), even = by * 16777216.0f, odd = by * 1048576.0f;
#pragma unroll
                for (int i = 0; i < M; ++i) {
                    const float whole = i & 2 ? odd : even;
                    run.o[n][i][j] = run.o[n][i][j] * whole * inverse;
                    run.o[n][i][2 + j] = run.o[n][i][2 + j] * whole * inverse;
                }
            }
        }
        if (warp >= W / 2) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < M; ++i)
                    merge[(((warp - W / 2) * NT + n) * M + i) * 32 + lane] = make_float4(run.o[n][i][0], run.o[n][i][1], run.o[n][i][2], run.o[n][i][3]);
        }
        __syncthreads();
        if (warp < W / 2) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < M; ++i) {
                    float4* at = &merge[((warp * NT + n) * M + i) * 32 + lane];
                    const float4 x = *at;
                    *at = make_float4(run.o[n][i][0] + x.x, run.o[n][i][1] + x.y, run.o[n][i][2] + x.z, run.o[n][i][3] + x.w);
                }
        }
        __syncthreads();
        // a thread per (group of rows, lane): rows 2 t and 2 t + 1, elements 8 g .. 8 g + 7 of each half of the head
        for (int item = threadIdx.x; item < NT * 32; item += S::THREADS) {
            const int ln = item & 31, n = item >> 5, g = ln >> 2, t = ln & 3;
            float x[2][H][8];
#pragma unroll
            for (int i = 0; i < M; ++i) {
                float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int w = 0; w < W / 2; ++w) {
                    const float4 y = merge[((w * NT + n) * M + i) * 32 + ln];
                    sum.x += y.x; sum.y += y.y; sum.z += y.z; sum.w += y.w;
                }
                const int h1 = H - 1, e1 = D == 128 ? i : i + 4;
                x[0][0][i] = sum.x; x[1][0][i] = sum.y; x[0][h1][e1] = sum.z; x[1][h1][e1] = sum.w;
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = n * 8 + 2 * t + j;
                if (row0 + r >= end) continue;
                float top = kNone, lt = 0.0f, ot = 0.0f;
#pragma unroll
                for (int w = 0; w < W; ++w) { top = fmaxf(top, sm_m[w][r]); lt += sm_l[w][r]; ot += sm_o[w][r]; }
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    float* y = x[j][h];
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] += ot;
                    const int d0 = 64 * h + 8 * g;
                    if (whole) {
                        store_out(p, mine.q, mine.head, row0 + r, D, d0, y, top, lt);
                    } else {
                        float* part = p.partial + static_cast<size_t>(2 * blockIdx.x + (from_start ? 1 : 0)) * S::PART;
                        reinterpret_cast<float4*>(part + r * D + d0)[0] = make_float4(y[0], y[1], y[2], y[3]);
                        reinterpret_cast<float4*>(part + r * D + d0)[1] = make_float4(y[4], y[5], y[6], y[7]);
                        if (d0 == 0) { part[S::ROWS * D + 2 * r] = top; part[S::ROWS * D + 2 * r + 1] = lt; }
                    }
                }
            }
        }
        if (!whole && from_start && threadIdx.x == 0) {
            // the CTAs that the rest of the segment falls to
            const long long last = s1 + (steps - step) - 1;             // the place of its last step
            const int at = static_cast<int>(((last + 1) * ctas - 1) / total);
            p.joins[2 * blockIdx.x] = make_int4(at - static_cast<int>(blockIdx.x) + 1, mine.tile_rows, mine.head, row0);
            p.joins[2 * blockIdx.x + 1] = make_int4(mine.q.row0, mine.q.n, mine.q.base, mine.q.granted);
        }
        __syncthreads();
        if (step == steps) {
            left -= kOverhead;
            if (threadIdx.x == 0 && left > 0) {
                Segment g = mine;
                next_segment<S>(p, g);
                mine = g;
            }
            step = 0;
        }
        from_start = true;
        fresh = true;
    }
    // gave up: what is still on its way lands before the CTA exits
    if (!ok) {
        if (lane == 0 && p.status) atomicCAS(p.status, 0, static_cast<int>(POLYSPEC_ERR_TIMEOUT));
        for (int k = max(0, issued - NS); k < issued; ++k)
            for (uint32_t i = 0; i < tensordev::kSpinLimitG; ++i)
                if (mbar_try(bar_at + 8u * (k % NS), static_cast<uint32_t>(k / NS) & 1u)) break;
    }
}

// Joins the parts of the segment that begins in CTA blockIdx.x and ends in a later one.  A lane takes eight elements of a row, eight parts on their way at
// a time; of more parts (single tokens over a few thousand: one per 256 of them) four lanes take every fourth.
template <class S>
__global__ void __launch_bounds__(256) join_kernel(const AttendParams p)
{
    constexpr int D = S::D, kVecs = D / 8, kAhead = 8;
    wait_for_stream();
    const int4 job = p.joins[2 * blockIdx.x], rows = p.joins[2 * blockIdx.x + 1];
    if (job.x == 0) return;
    const kv::SeqRows q = {rows.x, rows.y, rows.w, rows.z, 0, false};
    const int share = job.x > kAhead ? 4 : 1, slice = threadIdx.x % share;
    for (int item = threadIdx.x / share; item < S::ROWS * kVecs; item += 256 / share) {        // (whole warps)
        const int r = item / kVecs, d0 = item % kVecs * 8;
        const bool live = job.w + r < q.n * p.group && r < job.y;
        float x[8], m = kNone, l = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.0f;
        for (int k0 = slice; live && k0 < job.x; k0 += share * kAhead) {
            float2 ml[kAhead];
            float4 a[kAhead], b[kAhead];
            float to = m;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int k = k0 + share * u;
                if (k < job.x) {
                    const float* part = p.partial + static_cast<size_t>(k ? 2 * (blockIdx.x + k) : 2 * blockIdx.x + 1) * S::PART;
                    ml[u] = *reinterpret_cast<const float2*>(part + S::ROWS * D + 2 * r);
                    a[u] = reinterpret_cast<const float4*>(part + r * D + d0)[0];
                    b[u] = reinterpret_cast<const float4*>(part + r * D + d0)[1];
                } else {
                    ml[u] = make_float2(kNone, 0.0f);
                    a[u] = b[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) to = fmaxf(to, ml[u].x);
            const float was = ex2(m - to);
            m = to;
            l *= was;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= was;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const float is = ex2(ml[u].x - to);
                l = fmaf(ml[u].y, is, l);
                x[0] = fmaf(a[u].x, is, x[0]); x[1] = fmaf(a[u].y, is, x[1]); x[2] = fmaf(a[u].z, is, x[2]); x[3] = fmaf(a[u].w, is, x[3]);
                x[4] = fmaf(b[u].x, is, x[4]); x[5] = fmaf(b[u].y, is, x[5]); x[6] = fmaf(b[u].z, is, x[6]); x[7] = fmaf(b[u].w, is, x[7]);
            }
        }
        if (share > 1) {
            float top = m;
#pragma unroll
            for (int d = 1; d < 4; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            const float by = ex2(m - top);
            m = top;
            l *= by;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= by;
#pragma unroll
            for (int d = 1; d < 4; d <<= 1) {
                l += __shfl_xor_sync(0xffffffffu, l, d);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] += __shfl_xor_sync(0xffffffffu, x[e], d);
            }
        }
        if (live && slice == 0) store_out(p, q, job.z, job.w + r, D, d0, x, m, l);
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

constexpr int kMaxRows = 16;                    // rows of the largest tile
inline size_t align256(size_t x) { return (x + 255) / 256 * 256; }
inline size_t attend_bytes(int head_dim) { return align256(2 * kMaxCtas * sizeof(int4)) + static_cast<size_t>(2 * kMaxCtas) * kMaxRows * (head_dim + 2) * 4; }

// ---- accumulated weights: w[j] = keep * w[j] + sum over heads and rows of 2^(s2[r, j] - lse2[r])
struct WeighParams {
    AttendParams a;
    const float* lse;
    float keep;
    float* weights;
};

constexpr int kWeighWarps = 8, kWeighTokens = kWeighWarps * 16, kWeighGroups = 16;

// A CTA has 128 tokens of a sequence, a warp 16 of them: keys only, the products as in attend_kernel.  The rows of all heads come in chunks of 16
// groups of 8 (as many heads as that holds), so that the CTA seldom has to meet; a head's keys are loaded while the one before is multiplied.
// Sums stay in a lane's registers over all heads and rows; the lanes of one token meet at the end.  So every sum has one order.
// Issue-bound: 25 rows x 4 key heads of 64, 33 sequences of up to 3000 tokens 20 us (64 or 96 tokens per CTA: 2 us more, rows are brought in more often; 192: the same).
template <int D>
__global__ void __launch_bounds__(kWeighWarps * 32) weigh_kernel(const WeighParams w)
{
    constexpr int KS = D / 16, UB = kv::unit_bytes(D), WORDS = D / 32, G = kWeighGroups, THREADS = kWeighWarps * 32, kVecs = D / 8;
    __shared__ __align__(16) uint32_t frag[G * KS * 64];
    __shared__ __align__(16) float4 of_row[G * 8];             // factor, scaled sum, logarithm of the denominator (base 2), first slot it does not see
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
    const int rows = q.granted * p.group, head_groups = (rows + 7) / 8, groups = head_groups * p.kv_heads;        // a head's rows in groups of 8
    // the next head's keys; zeros where there are none
    uint32_t next[2][WORDS], next_pair[2];
    auto load_keys = [&](int head) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            next_pair[u] = 0;
#pragma unroll
            for (int i = 0; i < WORDS; ++i) next[u][i] = 0;
            if (unit[u] != 0xffffffffu && head < p.kv_heads) {
                const unsigned char* at = p.pool + (static_cast<size_t>(unit[u]) + static_cast<size_t>(head) * p.units_per_page) * UB;
#pragma unroll
                for (int i = 0; i < WORDS; i += 2) {
                    const uint2 x = *reinterpret_cast<const uint2*>(at + lane * (WORDS * 4) + i * 4);
                    next[u][i] = x.x; next[u][i + 1] = x.y;
                }
                next_pair[u] = *reinterpret_cast<const uint32_t*>(at + 4 * D + g8 * 4);
            }
        }
    };
    if (groups) load_keys(0);
    uint32_t kw[2][WORDS], kp[2];
    float acc[2] = {0.0f, 0.0f};                // tokens g8, g8 + 8
    int head = -1;
    for (int group0 = 0; group0 < groups; group0 += G) {
        const int n_groups = min(G, groups - group0);
        __syncthreads();                        // the rows of the chunk before have been read
        // a row per kVecs lanes: into fragments, scaled by a power of two of its own into fp16's upper range
        for (int item = threadIdx.x; item < n_groups * 8 * kVecs; item += THREADS) {
            const int n = item / (8 * kVecs), r = item / kVecs & 7, h = (group0 + n) / head_groups, row = (group0 + n) % head_groups * 8 + r;
            const int i = row / p.group, of = h * p.group + row % p.group;
            uint4 raw = make_uint4(0, 0, 0, 0);
            float lse = 0.0f;
            if (row < rows) {
                raw = *reinterpret_cast<const uint4*>(p.q + (q.row0 + i) * p.q_stride + of * D + item % kVecs * 8);
                lse = w.lse[static_cast<size_t>(q.row0 + i) * p.q_heads + of] * 1.44269504088896340736f;
            }
            const uint32_t* y = reinterpret_cast<const uint32_t*>(&raw);
            float x[8], sum = 0.0f, top = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[2 * e] = low(y[e]); x[2 * e + 1] = high(y[e]); sum = fmaf(x[2 * e], p.scale_log2, fmaf(x[2 * e + 1], p.scale_log2, sum)); }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (fabsf(x[e]) <= 3.4e38f) top = fmaxf(top, fabsf(x[e]));
#pragma unroll
            for (int d = 1; d < kVecs; d <<= 1) {
                sum += __shfl_xor_sync(0xffffffffu, sum, d);
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            }
            float factor;
            const float by = row_scale(p, top, &factor);
            store_fragment<D>(frag, n * 8 + r, item % kVecs, x, by);
            if (item % kVecs == 0) of_row[n * 8 + r] = make_float4(factor, sum, lse, __int_as_float(row < rows ? row_limit(q, i) : 0));
        }
        __syncthreads();
        for (int n = 0; n < n_groups; ++n) {
            const int h = (group0 + n) / head_groups;
            if (h != head) {
                head = h;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    kp[u] = next_pair[u];
#pragma unroll
                    for (int i = 0; i < WORDS; ++i) kw[u][i] = next[u][i];
                }
                load_keys(head + 1);
            }
            float sc[4] = {0.0f, 0.0f, 0.0f, 0.0f}, sd[4] = {0.0f, 0.0f, 0.0f, 0.0f};         // (two chains of products)
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const uint2 x = reinterpret_cast<const uint2*>(frag)[(n * KS + s) * 32 + lane];
                mma(s & 1 ? sd : sc, code_pair(kw[0][s >> 1], 2 * (s & 1)), code_pair(kw[1][s >> 1], 2 * (s & 1)), code_pair(kw[0][s >> 1], 2 * (s & 1) + 1),
                    code_pair(kw[1][s >> 1], 2 * (s & 1) + 1), x.x, x.y);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4 row = of_row[n * 8 + 2 * t4 + j];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const float x = fmaf(sc[2 * u + j] + sd[2 * u + j], low(kp[u]) * row.x, fmaf(row.y, high(kp[u]), -row.z));
                    if (unit[u] != 0xffffffffu && key0 + 8 * u + g8 < __float_as_int(row.w)) acc[u] += ex2(x);
                }
            }
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        acc[u] += __shfl_xor_sync(0xffffffffu, acc[u], 1);
        acc[u] += __shfl_xor_sync(0xffffffffu, acc[u], 2);
        const int slot = key0 + 8 * u + g8;
        if (t4 == 0 && slot < q.len) {
            float* to = w.weights + static_cast<size_t>(b) * p.s.max_pages * p.s.page_tokens + slot;
            *to = fmaf(w.keep, *to, acc[u]);
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
    if (!(scale >= -1.0e30f && scale <= 1.0e30f)) return POLYSPEC_ERR_INVALID_ARG;
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
    p.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + align256(2 * kMaxCtas * sizeof(int4)));
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    // rows of a sequence times the heads that share a key head, on average: one group of 8, or tiles of two.  (36 rows of 128 elements: tiles of 16 rows
    // 259 us; of 24 rows 272, of 32 rows 275, with two passes fewer over the cache but fewer warps.)
    const bool few = static_cast<long long>(r->rows) * p.group <= 8LL * s->n_seqs;
    cudaError_t e;
    if (head_dim == 128) e = few ? launch_attend<Shape<128, 1, 8, 2, 2>>(p, stream) : launch_attend<Shape<128, 2, 4, 3, 3>>(p, stream);
    else e = few ? launch_attend<Shape<64, 1, 8, 3, 2>>(p, stream) : launch_attend<Shape<64, 2, 4, 4, 3>>(p, stream);
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
