// Keys and values of new rows into a cache's 4-bit pages: per token and head an offset, a scale and a code per element.
//
//   offset = min(x), scale = (max(x) - offset) / 15 rounded up to bf16, code = rint((x - offset) / scale)
//
// A word of eight codes is one lane's 16-byte vector, a head head_dim / 8 lanes; keys and values of a row's head are neighbours in a warp.
// Rounding the scale up keeps every code at 15 or below, so nothing is cut off.
#include <cuda_bf16.h>

#include "kv_pages.cuh"

namespace polyspec {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b)
{
    uint32_t x;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(x) : "r"(a), "r"(b));
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

// D: head_dim.  A CTA has ROWS rows; its teams of D / 8 lanes take turns over (row, head, keys or values), kAhead items at a time, whose loads are on
// their way while the rows' places are looked up (a chain of four loads: sequence, length, page, its holders).
template <int D, int ROWS>
__global__ void __launch_bounds__(kThreads) append_kernel(const AppendParams p)
{
    constexpr int kLanes = D / 8, kTeams = kThreads / kLanes, kAhead = 2;
    __shared__ int found[ROWS];
    __shared__ uint32_t units[ROWS];            // the row's unit of head 0, or ~0: not written
    __shared__ int tokens[ROWS];                // its token of the unit
    wait_for_stream();
    const int row0 = blockIdx.x * ROWS, tid = threadIdx.x, w = tid % kLanes, team = tid / kLanes;
    const int per_row = 2 * p.kv_heads, items = min(ROWS, p.r.rows - row0) * per_row;
    uint4 raw[kAhead], coming[kAhead];
    auto load = [&](uint4* raw, int first) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int item = first + u * kTeams + team, row = row0 + item / per_row, j = item % per_row;
            raw[u] = make_uint4(0, 0, 0, 0);
            if (item < items) raw[u] = reinterpret_cast<const uint4*>((j & 1 ? p.v + row * p.v_stride : p.k + row * p.k_stride) + (j >> 1) * D)[w];
        }
    };
    load(coming, 0);
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
    for (int first = 0; first < items; first += kAhead * kTeams) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) raw[u] = coming[u];
        if (first + kAhead * kTeams < items) load(coming, first + kAhead * kTeams);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int item = first + u * kTeams + team;
            if (first + u * kTeams >= items) break;
            const int i = min(item, items - 1) / per_row, j = item % per_row, head = j >> 1, values = j & 1;
            const bool live = item < items && units[i] != 0xffffffffu;
            float x[8];
            x[0] = __uint_as_float(raw[u].x << 16); x[1] = __uint_as_float(raw[u].x & 0xffff0000u);
            x[2] = __uint_as_float(raw[u].y << 16); x[3] = __uint_as_float(raw[u].y & 0xffff0000u);
            x[4] = __uint_as_float(raw[u].z << 16); x[5] = __uint_as_float(raw[u].z & 0xffff0000u);
            x[6] = __uint_as_float(raw[u].w << 16); x[7] = __uint_as_float(raw[u].w & 0xffff0000u);
            // largest element and largest of the negated ones, two bf16 per instruction, NaN sticking
            const uint32_t sign = 0x80008000u;
            const uint32_t top = max2(max2(raw[u].x, raw[u].y), max2(raw[u].z, raw[u].w));
            const uint32_t bottom = max2(max2(raw[u].x ^ sign, raw[u].y ^ sign), max2(raw[u].z ^ sign, raw[u].w ^ sign));
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
            const bool broken = !(range <= 3.4e38f);
            if (broken) scale = offset = __uint_as_float(0x7fc00000u);
            const float inv = __fdividef(1.0f, scale), near = scale * 0.49999f;
            uint32_t word = 0, held[4];
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // the nearest whole number, by adding 1.5 * 2^23; the quotient itself is only divided out where the remainder says that it is near the
                // middle between two
                const float a = x[e] - offset;
                float t = __fadd_rn(__fmul_rn(a, inv), 12582912.0f), code = t - 12582912.0f;
                if (!(fabsf(fmaf(-code, scale, a)) <= near)) {
                    t = __fadd_rn(__fdiv_rn(a, scale), 12582912.0f);
                    code = t - 12582912.0f;
                }
                word |= (__float_as_uint(t) & 15u) << (4 * (e / 2) + 16 * (e % 2));
                y[e] = __fadd_rn(__fmul_rn(scale, code), offset);
            }
            if (broken) {
                word = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = scale;
            }
            // words 8 h + g of a row's values are neighbours for all h: lanes of lower words store both
            const uint32_t other = __shfl_xor_sync(0xffffffffu, word, 8);
            if (!live) continue;
            unsigned char* plane = p.pool + (values ? static_cast<size_t>(p.s.n_pages) * p.page_bytes : 0);
            uint32_t* to = reinterpret_cast<uint32_t*>(plane + static_cast<size_t>(units[i] + static_cast<uint32_t>(head * per_page)) * kv::unit_bytes(D));
            const int r = tokens[i];
            if (!values) to[kv::key_word(r, w, D)] = word;
            else if (D == 64) to[kv::value_word(r, w, D)] = word;
            else if (w < 8) *reinterpret_cast<uint2*>(to + kv::value_word(r, w, D)) = make_uint2(word, other);
            if (w == 0) to[D + r] = (__float_as_uint(scale) >> 16) | (__float_as_uint(offset) & 0xffff0000u);
            __nv_bfloat16* out = values ? p.v_held : p.k_held;
            if (out) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const __nv_bfloat162 z = __floats2bfloat162_rn(y[2 * e], y[2 * e + 1]);
                    held[e] = *reinterpret_cast<const uint32_t*>(&z);
                }
                reinterpret_cast<uint4*>(out + (static_cast<size_t>(row0 + i) * p.kv_heads + head) * D)[w] = make_uint4(held[0], held[1], held[2], held[3]);
            }
        }
    }
}

template <int D>
cudaError_t launch_append(const AppendParams& p, cudaStream_t stream)
{
    // eight rows share the look-up of their places where there are rows enough for all SMs
    if (p.r.rows >= 4096) return launch_early(append_kernel<D, 8>, dim3(static_cast<unsigned>((p.r.rows + 7) / 8)), kThreads, 0, stream, p);
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
