// Keys and values of new rows into a cache's 4-bit pages: per token and head an offset, a scale and a code per element.
//
//   offset = min(x), scale = (max(x) - offset) / 15 rounded up to bf16, code = rint((x - offset) / scale)
//
// A word of eight codes is one 16-byte vector of a head.  A lane takes two, half a head apart (in units of values their words are neighbours), a head
// head_dim / 16 lanes: what is computed once per head and lane (ends, scale, addresses) costs as much as the codes themselves, so half as many lanes are
// faster (54 -> 47 us at the size below).  Rounding the scale up keeps every code at 15 or below, so nothing is cut off.
//
// Measured (B200): 17500 rows of 8 heads of 128, 72 MB in and as much of held values out, 19 MB of codes: 36 us, 4.5 TB/s (a copy of as much 25); four rows per CTA
// of 128 threads (two or eight rows 38, eight of 256 threads 39, four of 64 threads 37).  A block of 420 rows 4.4 us: the chain of loads that finds a row's place.
#include <cuda_bf16.h>

#include "kv_pages.cuh"
#include "number_pairs.cuh"

namespace polyspec {
namespace {

using namespace numbers;

constexpr int kThreads = 128;
// 1.5 * 2^23 as bits (the form of whole numbers below), at the places of all eight codes of a word
constexpr uint32_t kMagicSum = 0x4b400000u * 0x11111111u;

__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b)
{
    uint32_t x;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(x) : "r"(a), "r"(b));
    return x;
}

__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b)
{
    uint32_t x;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(x) : "r"(a), "r"(b));
    return x;
}

struct AppendParams {
    polyspec_cache_pages s;
    polyspec_block_rows r;
    const __nv_bfloat16 *k, *v;
    long long k_stride, v_stride;
    unsigned char* pool;
    size_t page_bytes;
    __nv_bfloat16 *k_held, *v_held;
    float* weights;
    int32_t* status;
    int kv_heads;
};

// D: head_dim.  A CTA has ROWS rows; its teams of D / 16 lanes take turns over (row, head, keys or values), an item ahead with their loads; the first are on
// their way while the rows' places are looked up (a chain of four loads: sequence, length, page, its holders).
template <int D, int ROWS>
__global__ void __launch_bounds__(kThreads) append_kernel(const AppendParams p)
{
    constexpr int kLanes = D / 16, kTeams = kThreads / kLanes;
    __shared__ int found[ROWS];
    __shared__ uint32_t units[ROWS];            // the row's unit of head 0, or ~0: not written
    __shared__ int tokens[ROWS];                // its token of the unit
    wait_for_stream();
    const int row0 = blockIdx.x * ROWS, tid = threadIdx.x, w = tid % kLanes, team = tid / kLanes;
    const int per_row = 2 * p.kv_heads, items = min(ROWS, p.r.rows - row0) * per_row;
    uint4 raw[2], coming[2];
    // an item's row of the CTA and its number in the row; a turn further on without a division
    struct At { int i, j; };
    const int turn_rows = kTeams / per_row, turn_rest = kTeams % per_row;
    auto next = [&](At& at) {
        at.i += turn_rows;
        at.j += turn_rest;
        if (at.j >= per_row) { at.j -= per_row; ++at.i; }
    };
    const int rows = min(ROWS, p.r.rows - row0);
    const __nv_bfloat16 *k_rows = p.k + row0 * p.k_stride + w * 8, *v_rows = p.v + row0 * p.v_stride + w * 8;
    At read = {team / per_row, team % per_row}, at = read;
    auto load = [&](uint4* raw) {
        raw[0] = raw[1] = make_uint4(0, 0, 0, 0);
        if (read.i < rows) {
            const uint4* from = reinterpret_cast<const uint4*>((read.j & 1 ? v_rows + read.i * p.v_stride : k_rows + read.i * p.k_stride) + (read.j >> 1) * D);
            raw[0] = from[0];
            raw[1] = from[kLanes];
        }
        next(read);
    };
    load(coming);
    if (row0 == 0)              // numbers that make no sense are reported even where no row belongs to them
        for (int b = tid; b < p.s.n_seqs; b += kThreads)
            if (kv::seq_rows(p.s, p.r, b).bad) kv::report(p.status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE);
    if (tid < ROWS) found[tid] = -1;
    __syncthreads();
    for (int b = tid; b < p.s.n_seqs; b += kThreads) {
        const int lo = p.r.rows_at[b], hi = p.r.rows_at[b + 1];
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
            if (lo <= row0 + i && row0 + i < hi) atomicMax(&found[i], b);
    }
    __syncthreads();
    const int P = p.s.page_tokens, per_page = P / kv::kUnit;
    if (tid < ROWS) {
        const int b = found[tid];
        units[tid] = 0xffffffffu;
        if (b >= 0) {
            const kv::SeqRows q = kv::seq_rows(p.s, p.r, b);
            const int i = row0 + tid - q.row0;
            if (i < q.granted) {
                const int slot = q.base + i, at = slot / P;
                const int page = p.s.table[static_cast<size_t>(b) * p.s.max_pages + at];
                if (page < 0 || page >= p.s.n_pages || p.s.refs[page] > 1) {
                    kv::report(p.status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE);
                } else {
                    units[tid] = static_cast<uint32_t>(page) * p.kv_heads * per_page + (slot - at * P) / kv::kUnit;
                    tokens[tid] = slot % kv::kUnit;
                    if (p.weights) p.weights[static_cast<size_t>(b) * p.s.max_pages * P + slot] = 0.0f;
                }
            }
        }
    }
    __syncthreads();
    // (whole warps go round together: the exchange below is warp-wide)
    for (int first = 0; first < items; first += kTeams) {
        raw[0] = coming[0];
        raw[1] = coming[1];
        if (first + kTeams < items) load(coming);
        const int i = min(at.i, rows - 1), head = at.j >> 1, values = at.j & 1;
        const bool live = at.i < rows && units[i] != 0xffffffffu;
        next(at);
        const uint32_t z[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
        // largest element and, negated, smallest, two bf16 per instruction, NaN sticking
        const uint32_t sign = 0x80008000u;
        uint32_t top = z[0], bottom = z[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) { top = max2(top, z[e]); bottom = min2(bottom, z[e]); }
        bottom ^= sign;
        uint32_t ends = max2(__byte_perm(top, bottom, 0x5410), __byte_perm(top, bottom, 0x7632));
#pragma unroll
        for (int d = 1; d < kLanes; d <<= 1) ends = max2(ends, __shfl_xor_sync(0xffffffffu, ends, d));
        float offset = __uint_as_float((ends ^ sign) & 0xffff0000u) + 0.0f;         // (not -0)
        const float range = __uint_as_float(ends << 16) - offset;
        // range / 15, of which only the bits above the last sixteen are wanted, rounded up: the product says which they are unless it is next to one of their steps
        float step = range * (1.0f / 15.0f);
        if (((__float_as_uint(step) + 8u) & 0xffffu) < 17u) step = __fdiv_rn(range, 15.0f);
        const uint32_t up = (__float_as_uint(step) + 0xffffu) & 0xffff0000u;
        float scale = up ? fmaxf(__uint_as_float(up), 1.17549435e-38f) : 1.0f;      // at least the smallest normal number
        const bool broken = !(range < INFINITY);
        if (broken) scale = offset = __uint_as_float(0x7fc00000u);
        // Quotients as a division rounds them, by Markstein's correction: with the reciprocal rounded to nearest, q' = a * inv, r = a - q' * scale (exact),
        // q = q' + r * inv.  (Numbers this coarse often lie in the very middle between two codes: an approximate quotient would not do, and a look at the
        // remainders, with a division where they are near the half, divided almost always.)  Then the nearest whole number, by adding 1.5 * 2^23.
        const float magic = 12582912.0f, inv = __frcp_rn(scale);
        const uint64_t inv2 = pair(inv, inv), minus = pair(-scale, -scale), less = pair(-offset, -offset), more = pair(magic, magic), back = pair(-magic, -magic);
        uint64_t t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint64_t a = add2(pair(__uint_as_float(z[e] << 16), __uint_as_float(z[e] & 0xffff0000u)), less), q = mul2(a, inv2);
            t[e] = add2(fma2(fma2(q, minus, a), inv2, q), more);
        }
        if (scale < 1e-25f) {                   // remainders would leave the normal numbers
#pragma unroll
            for (int e = 0; e < 8; ++e)
                t[e] = pair(__fadd_rn(__fdiv_rn(__uint_as_float(z[e] << 16) - offset, scale), magic), __fadd_rn(__fdiv_rn(__uint_as_float(z[e] & 0xffff0000u) - offset, scale), magic));
        }
        if (!live) continue;
        uint32_t words[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float t0, t1;
            unpair(t[e], &t0, &t1);
            words[e >> 2] += (__float_as_uint(t0) << (4 * (e & 3))) + (__float_as_uint(t1) << (4 * (e & 3) + 16));
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) words[h] = broken ? 0 : words[h] - kMagicSum;
        unsigned char* plane = p.pool + (values ? static_cast<size_t>(p.s.n_pages) * p.page_bytes : 0);
        uint32_t* to = reinterpret_cast<uint32_t*>(plane + static_cast<size_t>(units[i] + static_cast<uint32_t>(head * per_page)) * kv::unit_bytes(D));
        const int r = tokens[i];
        if (D == 128 && values) {
            *reinterpret_cast<uint2*>(to + kv::value_word(r, w, D)) = make_uint2(words[0], words[1]);
        } else {
            to[values ? kv::value_word(r, w, D) : kv::key_word(r, w, D)] = words[0];
            to[values ? kv::value_word(r, w + kLanes, D) : kv::key_word(r, w + kLanes, D)] = words[1];
        }
        if (w == 0) to[D + r] = (__float_as_uint(scale) >> 16) | (__float_as_uint(offset) & 0xffff0000u);
        __nv_bfloat16* out = values ? p.v_held : p.k_held;
        if (out) {
            uint32_t held[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float y0, y1;               // (a scale of 8 bits times a code is exact; a NaN scale makes all of them NaN)
                unpair(fma2(add2(t[e], back), pair(scale, scale), pair(offset, offset)), &y0, &y1);
                const __nv_bfloat162 y = __floats2bfloat162_rn(y0, y1);
                held[e] = *reinterpret_cast<const uint32_t*>(&y);
            }
            uint4* held_to = reinterpret_cast<uint4*>(out + (static_cast<size_t>(row0 + i) * p.kv_heads + head) * D) + w;
            held_to[0] = make_uint4(held[0], held[1], held[2], held[3]);
            held_to[kLanes] = make_uint4(held[4], held[5], held[6], held[7]);
        }
    }
}

template <int D>
cudaError_t launch_append(const AppendParams& p, cudaStream_t stream)
{
    // four rows share the look-up of their places where there are rows enough for all SMs
    if (p.r.rows >= 4096) return launch_early(append_kernel<D, 4>, dim3(static_cast<unsigned>((p.r.rows + 3) / 4)), kThreads, 0, stream, p);
    return launch_early(append_kernel<D, 1>, dim3(static_cast<unsigned>(p.r.rows)), kThreads, 0, stream, p);
}

}  // namespace
}  // namespace polyspec

using namespace polyspec;

extern "C" polyspec_status polyspec_cache_append(const polyspec_cache_pages* s, const polyspec_block_rows* r, const void* k, long long k_stride,
                                                 const void* v, long long v_stride, int kv_heads, int head_dim, void* pool, void* k_held,
                                                 void* v_held, float* weights, int32_t* device_status, void* cuda_stream)
{
    polyspec_status st = kv::check_state(s);
    if (st == POLYSPEC_OK) st = kv::check_rows(r);
    if (st == POLYSPEC_OK) st = kv::check_heads(kv_heads, kv_heads, head_dim);
    if (st != POLYSPEC_OK) return st;
    if (!kv::rows_ok(k, k_stride, kv_heads, head_dim) || !kv::rows_ok(v, v_stride, kv_heads, head_dim)) return POLYSPEC_ERR_INVALID_ARG;
    if (!pool || !kv::aligned16(pool) || !kv::aligned16(k_held) || !kv::aligned16(v_held) || !aligned4(weights, device_status)) return POLYSPEC_ERR_INVALID_ARG;
    AppendParams p;
    p.s = *s; p.r = *r;
    p.k = static_cast<const __nv_bfloat16*>(k); p.v = static_cast<const __nv_bfloat16*>(v);
    p.k_stride = k_stride; p.v_stride = v_stride;
    p.pool = static_cast<unsigned char*>(pool);
    p.page_bytes = kv::page_bytes(*s, kv_heads, head_dim);
    p.k_held = static_cast<__nv_bfloat16*>(k_held); p.v_held = static_cast<__nv_bfloat16*>(v_held);
    p.weights = weights; p.status = device_status; p.kv_heads = kv_heads;
    if (s->n_pages * (p.page_bytes / kv::unit_bytes(head_dim)) >= 0xffffffffull) return POLYSPEC_ERR_UNSUPPORTED;       // units of a plane are counted in 32 bits
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = head_dim == 128 ? launch_append<128>(p, stream) : launch_append<64>(p, stream);
    return cuda_failed(e) ? POLYSPEC_ERR_CUDA : POLYSPEC_OK;
}
