// LM-head projection with 4-bit weights and group scales (the paper's M_2 is a 4-bit, group-128 copy of M_1, Section 4.1):
//   logits[r, v] = sum_g s[v, g] * ( sum_{k in g} h[r, k] * (q[v, k] - z[v, g]) )
// h bf16, q 4-bit codes, s bf16, z 4-bit zero points (8 where none are given).
//
// Numerics: q - z is an integer in [-15, 15], exact in bf16, so the tensor core sees exact operands; a group's sum is
// accumulated in fp32 and the group's scale multiplies that fp32 sum.  No dequantised weight is ever rounded.  The codes
// become bf16 without a conversion: 0x4300 | q is the bf16 number 128 + q, and 128 + z is subtracted exactly (one packed
// subtraction for two weights).  A word holds its eight weights in the order 0 2 4 6 1 3 5 7 from bit 0 up, so that
// (word >> 4 p) & 0x000f000f is the pair (2 p, 2 p + 1) as the matrix instructions want it.
//
// w4_stream_kernel, few rows: HBM-bound, every code is read once.  mma.sync.m16n8k16 with the vocabulary on the M axis:
// codes go from global memory straight into the A fragments, nothing passes through shared memory but the hidden rows
// (staged once per CTA in fragment order).  With at most 16 columns the tensor work is a small part of the time, and
// tcgen05 would want the expanded weights written to tensor memory or shared memory first.
// A tile is 32 vocabulary entries; `split` warps share a tile along d and add up through shared memory in a fixed order.
#include <cuda_bf16.h>

#include <algorithm>
#include <mutex>

#include "polyspec_kernels.cuh"
#include "stream_device.cuh"
#include "w4_kernels.cuh"

namespace polyspec {
namespace {

constexpr int kWarpsS = 16;                     // warps per CTA, one CTA per SM
constexpr int kThreadsS = 32 * kWarpsS;
constexpr int kTileS = 32;                      // vocabulary entries per tile (two m16 tiles)
constexpr int kStreamRows = 16;                 // more rows go to the tensor-core kernel
constexpr int kChunk = 128;                     // d elements per step: 16 bytes of codes per lane and row

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The 16 bytes of codes a lane takes of one row and chunk: words 0..3.  Lane t of a quad takes, of every group of G
// elements, G/4 consecutive ones: so that each MMA stays inside one group.
template <int G>
__device__ __forceinline__ uint4 load_codes(const uint32_t* row, int chunk, int t, int groups_left)
{
    uint4 w = make_uint4(0, 0, 0, 0);
    const uint32_t* p = row + chunk * (kChunk / 8);
    if (G == 128) {
        w = streamdev::ld_stream(p + t * 4);
    } else if (G == 64) {
        uint2 x = make_uint2(0, 0), y = make_uint2(0, 0);
        x = __ldg(reinterpret_cast<const uint2*>(p + t * 2));
        if (groups_left > 1) y = __ldg(reinterpret_cast<const uint2*>(p + 8 + t * 2));
        w = make_uint4(x.x, x.y, y.x, y.y);
    } else {
        w.x = __ldg(p + t);
        if (groups_left > 1) w.y = __ldg(p + 4 + t);
        if (groups_left > 2) w.z = __ldg(p + 8 + t);
        if (groups_left > 3) w.w = __ldg(p + 12 + t);
    }
    return w;
}

struct StreamParams {
    const __nv_bfloat16* hidden;
    const uint32_t* codes;
    const __nv_bfloat16* scales;
    const unsigned char* zeros;         // or nullptr: 8
    int rows, V, d, groups;             // groups = d / G
    int split;                          // warps per tile, a divisor of kWarpsS
    int chunks_per_warp;                // ceil(chunks / split)
    int tiles;
    uint32_t exponent;                  // w4::kExponent
    void* out;
};

template <int G, int NT, int DT>
__global__ void __launch_bounds__(kThreadsS, 1) w4_stream_kernel(const StreamParams p)
{
    extern __shared__ uint4 smem_w4[];
    constexpr int GPC = kChunk / G;             // groups per chunk
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int g = lane >> 2, t = lane & 3;
    const int chunks = (p.d + kChunk - 1) / kChunk;
    const int row0 = blockIdx.y * (NT * 8);     // first hidden row of this CTA
    const int rows = min(NT * 8, p.rows - row0);

    // hidden rows in fragment order: the 16 bytes of (chunk, n tile, word, lane) are the eight elements of row nt * 8 + g
    // that multiply word `word` of the codes lane (g, t) holds
    const int kept = chunks * NT * 4 * 32;
    for (int i = threadIdx.x; i < kept; i += kThreadsS) {
        const int l = i & 31, word = (i >> 5) & 3, nt = (i >> 7) % NT, c = (i >> 7) / NT;
        const int n = nt * 8 + (l >> 2), q = l & 3;
        const int k = c * kChunk + (G == 128 ? q * 32 + word * 8 : G == 64 ? (word >> 1) * 64 + q * 16 + (word & 1) * 8 : word * 32 + q * 8);
        uint4 x = make_uint4(0, 0, 0, 0);
        if (n < rows && k < p.d) x = *reinterpret_cast<const uint4*>(p.hidden + static_cast<size_t>(row0 + n) * p.d + k);
        smem_w4[i] = x;
    }
    __syncthreads();

    const int team = warp / p.split, part = warp % p.split, teams = kWarpsS / p.split;
    float* joined = reinterpret_cast<float*>(smem_w4 + kept);       // [2][kWarpsS][2 * NT * 4][32]
    const int c_first = part * p.chunks_per_warp, c_end = min(chunks, c_first + p.chunks_per_warp);
    uint32_t turn = 0;
    for (int tile = blockIdx.x + team * gridDim.x; tile < p.tiles; tile += teams * gridDim.x, turn ^= 1u) {
        const uint32_t* codes[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)             // the lane's four entries: g, g + 8, g + 16, g + 24 (those past V read the last one)
            codes[i] = p.codes + static_cast<size_t>(min(tile * kTileS + i * 8 + g, p.V - 1)) * (p.d / 8);
        // scale and zero point of entry g + 8 t, which the quad's lanes hand one another when they use them
        const size_t own = static_cast<size_t>(min(tile * kTileS + t * 8 + g, p.V - 1)) * p.groups;
        struct Raw { unsigned short scale[GPC]; unsigned char zero[GPC]; };
        auto load_raw = [&](int c) {
            Raw r;
#pragma unroll
            for (int gi = 0; gi < GPC; ++gi) {
                const int group = GPC == 1 ? c : min(c * GPC + gi, p.groups - 1);
                r.scale[gi] = __ldg(reinterpret_cast<const unsigned short*>(p.scales) + own + group);
                r.zero[gi] = p.zeros ? __ldg(p.zeros + own + group) : 8;
            }
            return r;
        };
        float sum[2][NT][4];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[m][nt][i] = 0.0f;

        constexpr int kAhead = 2;               // chunks of codes in flight
        uint4 w[kAhead][4];
        Raw raw[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            if (c_first + a < c_end) {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[a][i] = load_codes<G>(codes[i], c_first + a, t, p.groups - (c_first + a) * GPC);
                raw[a] = load_raw(c_first + a);
            }
        for (int c0 = c_first; c0 < c_end; c0 += kAhead) {
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int c = c0 + a;
                if (c >= c_end) break;
                uint32_t x[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) { x[i][0] = w[a][i].x; x[i][1] = w[a][i].y; x[i][2] = w[a][i].z; x[i][3] = w[a][i].w; }
                uint32_t sz[GPC];
#pragma unroll
                for (int gi = 0; gi < GPC; ++gi) sz[gi] = static_cast<uint32_t>(raw[a].scale[gi]) << 16 | (raw[a].zero[gi] & 15u);
                if (c + kAhead < c_end) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[a][i] = load_codes<G>(codes[i], c + kAhead, t, p.groups - (c + kAhead) * GPC);
                    raw[a] = load_raw(c + kAhead);
                }
                const uint4* hid = smem_w4 + c * NT * 4 * 32 + lane;
#pragma unroll
                for (int gi = 0; gi < GPC; ++gi) {
                    const int group = c * GPC + gi;
                    if (GPC > 1 && group >= p.groups) break;
                    float s[4];
                    uint32_t z[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t x = __shfl_sync(0xffffffffu, sz[gi], g * 4 + i);
                        s[i] = __uint_as_float(x & 0xffff0000u);
                        z[i] = p.exponent | (x & 15u) * 0x00010001u;
                    }
                    float acc[2][NT][4];
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int i = 0; i < 4; ++i) acc[m][nt][i] = 0.0f;
#pragma unroll
                    for (int wi = 0; wi < 4 / GPC; ++wi) {
                        const int word = gi * (4 / GPC) + wi;
                        uint4 h[NT];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) h[nt] = hid[(nt * 4 + word) * 32];
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            uint32_t lo[4], hi[4];
                            w4::expand(x[2 * m][word], z[2 * m], p.exponent, lo);
                            w4::expand(x[2 * m + 1][word], z[2 * m + 1], p.exponent, hi);
                            const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]}, a1[4] = {lo[2], hi[2], lo[3], hi[3]};
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                mma_bf16(acc[m][nt], a0, h[nt].x, h[nt].y);
                                mma_bf16(acc[m][nt], a1, h[nt].z, h[nt].w);
                            }
                        }
                    }
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int i = 0; i < 4; ++i) sum[m][nt][i] = fmaf(s[2 * m + (i >> 1)], acc[m][nt][i], sum[m][nt][i]);
                }
            }
        }
        // entry (m, half) * 8 + g, row nt * 8 + 2 t + (i & 1)
        if (p.split > 1) {
            float* mine = joined + (turn * kWarpsS + warp) * (2 * NT * 4 * 32);
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) mine[((m * NT + nt) * 4 + i) * 32 + lane] = sum[m][nt][i];
            asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(32 * p.split) : "memory");
            const float* all = joined + (turn * kWarpsS + team * p.split) * (2 * NT * 4 * 32);
            for (int r = part; r < 2 * NT * 4; r += p.split) {
                float x = 0.0f;
                for (int q = 0; q < p.split; ++q) x += all[(q * 2 * NT * 4 + r) * 32 + lane];
                const int i = r & 3, nt = (r >> 2) % NT, m = (r >> 2) / NT;
                const int v = tile * kTileS + m * 16 + (i >> 1) * 8 + g, n = nt * 8 + 2 * t + (i & 1);
                if (v < p.V && n < rows) w4::store_logit<DT>(p.out, static_cast<size_t>(row0 + n) * p.V + v, x);
            }
        } else {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int v = tile * kTileS + m * 16 + (i >> 1) * 8 + g, n = nt * 8 + 2 * t + (i & 1);
                        if (v < p.V && n < rows) w4::store_logit<DT>(p.out, static_cast<size_t>(row0 + n) * p.V + v, sum[m][nt][i]);
                    }
        }
    }
}

constexpr size_t kMaxSmem = 227 * 1024;

size_t stream_smem(int d, int nt)
{
    const size_t chunks = (d + kChunk - 1) / kChunk;
    return chunks * nt * 4 * 512 + 2 * kWarpsS * (2 * nt * 4 * 32) * sizeof(float);
}

template <int G, int NT, int DT>
cudaError_t launch_stream_t(const StreamParams& p, int grid_y, int sms, cudaStream_t stream)
{
    const size_t smem = stream_smem(p.d, NT);
    cudaError_t e = cudaFuncSetAttribute(w4_stream_kernel<G, NT, DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return e;
    const dim3 grid(static_cast<unsigned>(std::min(sms, p.tiles)), static_cast<unsigned>(grid_y));
    w4_stream_kernel<G, NT, DT><<<grid, kThreadsS, smem, stream>>>(p);
    return cudaGetLastError();
}

template <int G>
cudaError_t launch_stream_g(const StreamParams& p, int nt, polyspec_dtype dt, int grid_y, int sms, cudaStream_t stream)
{
    if (dt == POLYSPEC_F32)
        return nt == 1 ? launch_stream_t<G, 1, POLYSPEC_F32>(p, grid_y, sms, stream) : launch_stream_t<G, 2, POLYSPEC_F32>(p, grid_y, sms, stream);
    return nt == 1 ? launch_stream_t<G, 1, POLYSPEC_BF16>(p, grid_y, sms, stream) : launch_stream_t<G, 2, POLYSPEC_BF16>(p, grid_y, sms, stream);
}

cudaError_t launch_stream(const W4Problem& q, int nt, polyspec_dtype dt, cudaStream_t stream)
{
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    StreamParams p;
    p.hidden = static_cast<const __nv_bfloat16*>(q.hidden);
    p.codes = q.codes;
    p.scales = static_cast<const __nv_bfloat16*>(q.scales);
    p.zeros = q.zeros;
    p.rows = q.rows;
    p.V = q.V;
    p.d = q.d;
    p.groups = q.d / q.group;
    p.out = q.out;
    p.exponent = w4::kExponent;
    p.tiles = (q.V + kTileS - 1) / kTileS;
    const int chunks = (q.d + kChunk - 1) / kChunk;
    // as many warps per tile as leave each two chunks (the prefetch depth) to work on
    p.split = kWarpsS;
    while (p.split > 1 && chunks < 2 * p.split) p.split >>= 1;
    p.chunks_per_warp = (chunks + p.split - 1) / p.split;
    const int grid_y = (q.rows + 8 * nt - 1) / (8 * nt);
    switch (q.group) {
        case 128: return launch_stream_g<128>(p, nt, dt, grid_y, sms, stream);
        case 64: return launch_stream_g<64>(p, nt, dt, grid_y, sms, stream);
        default: return launch_stream_g<32>(p, nt, dt, grid_y, sms, stream);
    }
}

// codes [V, d] one byte each -> packed words
__global__ void pack_kernel(const unsigned char* codes, uint32_t* out, long long words)
{
    const long long step = static_cast<long long>(gridDim.x) * blockDim.x;
    for (long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x; i < words; i += step) {
        const uint2 c = *reinterpret_cast<const uint2*>(codes + i * 8);
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t q = ((e < 4 ? c.x : c.y) >> (8 * (e & 3))) & 15u;
            w |= q << (4 * (e >> 1) + 16 * (e & 1));
        }
        out[i] = w;
    }
}

}  // namespace
}  // namespace polyspec

using namespace polyspec;

extern "C" {

polyspec_status polyspec_pack_quantized(const void* codes, int V, int d, void* qweight, void* cuda_stream)
{
    if (!codes || !qweight || V <= 0 || d <= 0) return POLYSPEC_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(codes) & 15u) != 0 || (reinterpret_cast<uintptr_t>(qweight) & 15u) != 0) return POLYSPEC_ERR_INVALID_ARG;
    if (d % 32 != 0) return POLYSPEC_ERR_UNSUPPORTED;
    const long long words = static_cast<long long>(V) * (d / 8);
    const unsigned blocks = static_cast<unsigned>(std::min<long long>((words + 255) / 256, 148 * 16));
    pack_kernel<<<blocks, 256, 0, static_cast<cudaStream_t>(cuda_stream)>>>(static_cast<const unsigned char*>(codes), static_cast<uint32_t*>(qweight), words);
    return cuda_failed(cudaGetLastError()) ? POLYSPEC_ERR_CUDA : POLYSPEC_OK;
}

polyspec_status polyspec_lm_head_quantized(const void* hidden, const void* qweight, const void* scales, const void* zero_points, int rows, int V, int d,
                                    int group, polyspec_dtype dt, void* logits, int32_t* device_status, void* cuda_stream)
{
    if (!hidden || !qweight || !scales || !logits || rows <= 0 || V <= 0 || d <= 0) return POLYSPEC_ERR_INVALID_ARG;
    if (dt != POLYSPEC_F32 && dt != POLYSPEC_BF16) return POLYSPEC_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(hidden) & 15u) != 0 || (reinterpret_cast<uintptr_t>(qweight) & 15u) != 0 ||
        (reinterpret_cast<uintptr_t>(logits) & 15u) != 0 || (reinterpret_cast<uintptr_t>(scales) & 1u) != 0)
        return POLYSPEC_ERR_INVALID_ARG;
    if (group != 32 && group != 64 && group != 128) return POLYSPEC_ERR_UNSUPPORTED;
    if (d % group != 0 || V > 0x7fffffff - 1024) return POLYSPEC_ERR_UNSUPPORTED;
    W4Problem q;
    q.hidden = hidden;
    q.codes = static_cast<const uint32_t*>(qweight);
    q.scales = scales;
    q.zeros = static_cast<const unsigned char*>(zero_points);
    q.rows = rows;
    q.V = V;
    q.d = d;
    q.group = group;
    q.out = logits;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (rows > kStreamRows || stream_smem(d, rows > 8 ? 2 : 1) > kMaxSmem)
        return cuda_failed(launch_w4_tensor(q, dt, device_status, s)) ? POLYSPEC_ERR_CUDA : POLYSPEC_OK;
    const int nt = rows > 8 ? 2 : 1;
    return cuda_failed(launch_stream(q, nt, dt, s)) ? POLYSPEC_ERR_CUDA : POLYSPEC_OK;
}

}  // extern "C"
