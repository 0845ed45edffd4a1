// Norm of every query and key head and its rotation by position, in one pass over the rows of a projection.
//
//   y = x / sqrt(mean(x^2) + eps) * weight;  (a, b) -> (a cos - b sin, a sin + b cos),  angle = position * frequency
//
// A head is head_dim / 16 lanes of two 16-byte vectors each.  A lane's vectors hold whole pairs: elements 8c .. 8c + 7 and their
// partners rotary_dim / 2 further on, or 16 neighbours where pairs are neighbours or nothing is rotated; so the mean is
// the only exchange, and the 8 angles of a lane are the same for every head that it meets in a row.
// Angles in turns: position * frequency / 2 pi in fp64, the whole turns taken off, the rest to sincospi in fp32.  (A position of a million
// times a frequency of 1 leaves fp32 an error of 0.06 radians.)
//
// HBM-bound where there are many rows.  Measured (B200): 8195 rows of 40 heads of 128, 168 MB: 33.8 us, 5.0 TB/s (a copy of as much 25.6; two heads ahead
// instead of one take registers, 38 us); a block of 9 rows 1.8 us, the launch and two loads.
#include <cuda_bf16.h>

#include "kv_pages.cuh"
#include "number_pairs.cuh"

namespace polyspec {
namespace {

using namespace numbers;

constexpr int kThreads = 64;                    // (128: 34.3 us at the size above, 256: 40)

struct RotateParams {
    const __nv_bfloat16 *q, *k, *q_weight, *k_weight;
    __nv_bfloat16 *q_out, *k_out;
    long long q_stride, k_stride, q_out_stride, k_out_stride;
    const int32_t* positions;
    const float* frequencies;
    int q_heads, kv_heads, rows, head_dim, rotary, interleaved;
    int parts;                  // warps that share a row's heads
    float eps;
};

// A lane's two vectors as the first and the second numbers of its eight pairs, two pairs to a 64-bit number: partners are the vectors themselves, or
// neighbours in them.
template <bool NEIGHBOURS>
__device__ __forceinline__ void unpack(const uint4& r0, const uint4& r1, uint64_t* a, uint64_t* b)
{
    const uint32_t x[8] = {r0.x, r0.y, r0.z, r0.w, r1.x, r1.y, r1.z, r1.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = NEIGHBOURS ? pair(low(x[2 * i]), low(x[2 * i + 1])) : pair(low(x[i]), high(x[i]));
        b[i] = NEIGHBOURS ? pair(high(x[2 * i]), high(x[2 * i + 1])) : pair(low(x[4 + i]), high(x[4 + i]));
    }
}
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&x);
}
template <bool NEIGHBOURS>
__device__ __forceinline__ void pack(const uint64_t* a, const uint64_t* b, uint4& r0, uint4& r1)
{
    uint32_t x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a0, a1, b0, b1;
        unpair(a[i], &a0, &a1);
        unpair(b[i], &b0, &b1);
        x[NEIGHBOURS ? 2 * i : i] = NEIGHBOURS ? pack2(a0, b0) : pack2(a0, a1);
        x[NEIGHBOURS ? 2 * i + 1 : 4 + i] = NEIGHBOURS ? pack2(a1, b1) : pack2(b0, b1);
    }
    r0 = make_uint4(x[0], x[1], x[2], x[3]);
    r1 = make_uint4(x[4], x[5], x[6], x[7]);
}

// L lanes per head (a power of two, at least head_dim / 16); NEIGHBOURS: neighbours are rotated together.
template <int L, bool NEIGHBOURS>
__global__ void __launch_bounds__(kThreads) rotate_kernel(const RotateParams p)
{
    constexpr int kHeads = 32 / L; // heads a warp holds at a time
    const int lane = threadIdx.x & 31, at = lane % L, slot = lane / L;
    const long long item = static_cast<long long>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
    const int row = static_cast<int>(item / p.parts), part = static_cast<int>(item % p.parts);
    const int vectors = p.head_dim / 8, half = p.rotary / 16, chunk = 2 * at;
    const bool mine = chunk < vectors;
    // the lane's two vectors: partners of a rotation by halves, else neighbours
    const bool turned = chunk * 8 < p.rotary, halves = turned && !NEIGHBOURS;
    const int v0 = halves ? at : chunk, v1 = halves ? at + half : chunk + 1;
    wait_for_stream();
    if (row >= p.rows) return;                  // (whole warps)

    const int heads = p.q_heads + p.kv_heads;
    const __nv_bfloat16 *q_row = p.q + row * p.q_stride, *k_row = p.k + row * p.k_stride - p.q_heads * p.head_dim;
    __nv_bfloat16 *q_to = p.q_out + row * p.q_out_stride, *k_to = p.k_out + row * p.k_out_stride - p.q_heads * p.head_dim;
    auto load = [&](int h, uint4& r0, uint4& r1) {
        r0 = r1 = make_uint4(0, 0, 0, 0);
        if (mine && h < heads) {
            const uint4* x = reinterpret_cast<const uint4*>((h < p.q_heads ? q_row : k_row) + h * p.head_dim);
            r0 = x[v0];
            r1 = x[v1];
        }
    };
    uint4 n0, n1;                               // the next heads: on their way while the angles are computed
    load(part * kHeads + slot, n0, n1);

    float c[8], s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) { c[i] = 1.0f; s[i] = 0.0f; }
    if (p.rotary) {
        // the lanes that stand at one place of different heads share its eight angles
        constexpr int kOwn = kHeads < 8 ? 8 / kHeads : 1;
        const double turns = static_cast<double>(p.positions[row]) * 0.15915494309189533577;       // 1 / 2 pi
        float cs[kOwn], sn[kOwn];
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int k = at * 8 + (slot * kOwn + i) % 8;
            const double x = turns * p.frequencies[min(k, p.rotary / 2 - 1)];
            sincospif(2.0f * static_cast<float>(x - rint(x)), &sn[i], &cs[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = __shfl_sync(0xffffffffu, cs[i % kOwn], i / kOwn * L + at), b = __shfl_sync(0xffffffffu, sn[i % kOwn], i / kOwn * L + at);
            if (turned) { c[i] = a; s[i] = b; }
        }
    }
    uint4 weight[2][2];                         // of queries, of keys
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint4* from = reinterpret_cast<const uint4*>(i ? p.k_weight : p.q_weight);
        weight[i][0] = weight[i][1] = make_uint4(0, 0, 0, 0);
        if (from && mine) { weight[i][0] = from[v0]; weight[i][1] = from[v1]; }
    }
    uint64_t c2[4], s2[4], n2[4];               // cosines, sines, sines with their sign turned
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        c2[i] = pair(c[2 * i], c[2 * i + 1]);
        s2[i] = pair(s[2 * i], s[2 * i + 1]);
        n2[i] = pair(-s[2 * i], -s[2 * i + 1]);
    }
    const float over = 1.0f / p.head_dim;
    for (int h0 = part * kHeads; h0 < heads; h0 += p.parts * kHeads) {
        const int h = h0 + slot;
        const bool live = mine && h < heads, is_q = h < p.q_heads;
        const uint4 r0 = n0, r1 = n1;
        load(h + p.parts * kHeads, n0, n1);
        uint64_t a[4], b[4];
        unpack<NEIGHBOURS>(r0, r1, a, b);
        if (p.q_weight || p.k_weight) {
            uint64_t both = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) both = fma2(a[i], a[i], fma2(b[i], b[i], both));
            float sum, odd;
            unpair(both, &sum, &odd);
            sum += odd;
#pragma unroll
            for (int d = 1; d < L; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            const float norm = 1.0f / sqrtf(sum * over + p.eps);
            if (is_q ? p.q_weight : p.k_weight) {
                uint64_t w[4], v[4];
                const uint64_t norm2 = pair(norm, norm);
                unpack<NEIGHBOURS>(is_q ? weight[0][0] : weight[1][0], is_q ? weight[0][1] : weight[1][1], w, v);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    a[i] = mul2(a[i], mul2(norm2, w[i]));
                    b[i] = mul2(b[i], mul2(norm2, v[i]));
                }
            }
        }
        if (!live) continue;
        if (turned) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint64_t x = a[i], y = b[i];
                a[i] = fma2(x, c2[i], mul2(y, n2[i]));
                b[i] = fma2(x, s2[i], mul2(y, c2[i]));
            }
        }
        uint4* y = reinterpret_cast<uint4*>((is_q ? q_to : k_to) + h * p.head_dim);
        uint4 y0, y1;
        pack<NEIGHBOURS>(a, b, y0, y1);
        y[v0] = y0;
        y[v1] = y1;
    }
}

template <int L>
cudaError_t launch(const RotateParams& p, cudaStream_t stream)
{
    const long long warps = static_cast<long long>(p.rows) * p.parts;
    const dim3 grid(static_cast<unsigned>((warps + kThreads / 32 - 1) / (kThreads / 32)));
    return p.interleaved ? launch_early(rotate_kernel<L, true>, grid, kThreads, 0, stream, p) : launch_early(rotate_kernel<L, false>, grid, kThreads, 0, stream, p);
}

}  // namespace
}  // namespace polyspec

using namespace polyspec;

extern "C" polyspec_status polyspec_rotate_heads(const void* q, long long q_stride, int q_heads, const void* k, long long k_stride, int kv_heads,
                                                 int rows, int head_dim, int rotary_dim, int interleaved, const int32_t* positions,
                                                 const float* frequencies, const void* q_weight, const void* k_weight, float eps,
                                                 void* q_out, long long q_out_stride, void* k_out, long long k_out_stride, void* cuda_stream)
{
    if (rows < 1 || head_dim < 1 || rotary_dim < 0 || rotary_dim > head_dim || q_heads < 1 || kv_heads < 0 || !(eps >= 0.0f) || eps > 3e38f)
        return POLYSPEC_ERR_INVALID_ARG;
    if ((k == nullptr) != (kv_heads == 0) || (k == nullptr) != (k_out == nullptr)) return POLYSPEC_ERR_INVALID_ARG;
    if (head_dim % 16 || head_dim > 256 || rotary_dim % 16 || q_heads > 4096 || kv_heads > 4096 || rows > (1 << 24)) return POLYSPEC_ERR_UNSUPPORTED;
    if (!kv::rows_ok(q, q_stride, q_heads, head_dim) || !kv::rows_ok(q_out, q_out_stride, q_heads, head_dim)) return POLYSPEC_ERR_INVALID_ARG;
    if (k && (!kv::rows_ok(k, k_stride, kv_heads, head_dim) || !kv::rows_ok(k_out, k_out_stride, kv_heads, head_dim))) return POLYSPEC_ERR_INVALID_ARG;
    if (rotary_dim && (!positions || !frequencies || !aligned4(positions, frequencies))) return POLYSPEC_ERR_INVALID_ARG;
    if (!kv::aligned16(q_weight) || !kv::aligned16(k_weight)) return POLYSPEC_ERR_INVALID_ARG;
    if ((q == q_out && q_stride != q_out_stride) || (k && k == k_out && k_stride != k_out_stride)) return POLYSPEC_ERR_INVALID_ARG;

    RotateParams p;
    p.q = static_cast<const __nv_bfloat16*>(q); p.k = static_cast<const __nv_bfloat16*>(k);
    p.q_weight = static_cast<const __nv_bfloat16*>(q_weight); p.k_weight = static_cast<const __nv_bfloat16*>(k_weight);
    p.q_out = static_cast<__nv_bfloat16*>(q_out); p.k_out = static_cast<__nv_bfloat16*>(k_out);
    p.q_stride = q_stride; p.k_stride = k_stride; p.q_out_stride = q_out_stride; p.k_out_stride = k_out_stride;
    p.positions = positions; p.frequencies = frequencies;
    p.q_heads = q_heads; p.kv_heads = kv_heads; p.rows = rows; p.head_dim = head_dim; p.rotary = rotary_dim; p.interleaved = interleaved;
    p.eps = eps;
    int lanes = 1;
    while (lanes < head_dim / 16) lanes *= 2;
    // few rows: a row's heads are spread over warps until there are some for every SM; many rows: one warp has them all, and its angles serve all of them
    const int most = (q_heads + kv_heads + 32 / lanes - 1) / (32 / lanes);
    p.parts = rows >= 2048 ? 1 : most < (2048 + rows - 1) / rows ? most : (2048 + rows - 1) / rows;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = lanes == 1 ? launch<1>(p, stream) : lanes == 2 ? launch<2>(p, stream) : lanes == 4 ? launch<4>(p, stream)
                          : lanes == 8 ? launch<8>(p, stream) : launch<16>(p, stream);
    return cuda_failed(e) ? POLYSPEC_ERR_CUDA : POLYSPEC_OK;
}
