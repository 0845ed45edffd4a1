// Causal attention over whole prompts, packed one behind the other.  The plain form: a warp per row and head.
#include <cuda_bf16.h>

#include "kv_pages.cuh"

namespace polyspec {
namespace {

struct PromptParams {
    const unsigned short *q, *k, *v;
    long long q_stride, k_stride, v_stride;
    const int32_t* rows_at;
    int n_seqs, rows, q_heads, kv_heads;
    float scale_log2;
    unsigned short* out;
    float* lse;
    int32_t* status;
};

template <int D>
__global__ void __launch_bounds__(256) prompt_plain_kernel(const PromptParams p)
{
    constexpr int N = D / 32;
    __shared__ int found;
    wait_for_stream();
    const int row = blockIdx.x, lane = threadIdx.x & 31;
    if (row == 0)
        for (int b = threadIdx.x; b < p.n_seqs; b += blockDim.x)
            if (p.rows_at[b] < 0 || p.rows_at[b + 1] < p.rows_at[b] || p.rows_at[b + 1] > p.rows) kv::report(p.status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE);
    const int b = kv::find_seq(p.rows_at, p.n_seqs, row, &found);
    if (b < 0) return;
    const int begin = p.rows_at[b], end = p.rows_at[b + 1];
    if (begin < 0 || end > p.rows) return;
    for (int h = threadIdx.x >> 5; h < p.q_heads; h += 8) {
        const int kh = h / (p.q_heads / p.kv_heads);
        float q[N], o[N], m = -INFINITY, l = 0.0f;
        for (int i = 0; i < N; ++i) {
            q[i] = __uint_as_float(static_cast<uint32_t>(p.q[row * p.q_stride + h * D + lane + 32 * i]) << 16) * p.scale_log2;
            o[i] = 0.0f;
        }
        for (int j = begin; j <= row; ++j) {
            float s = 0.0f;
            for (int i = 0; i < N; ++i) s = fmaf(q[i], __uint_as_float(static_cast<uint32_t>(p.k[j * p.k_stride + kh * D + lane + 32 * i]) << 16), s);
            for (int d = 1; d < 32; d <<= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
            const float to = fmaxf(m, s), was = m == -INFINITY ? 0.0f : exp2f(m - to), is = exp2f(s - to);
            m = to;
            l = fmaf(l, was, is);
            for (int i = 0; i < N; ++i) o[i] = fmaf(o[i], was, is * __uint_as_float(static_cast<uint32_t>(p.v[j * p.v_stride + kh * D + lane + 32 * i]) << 16));
        }
        const size_t at = static_cast<size_t>(row) * p.q_heads + h;
        for (int i = 0; i < N; ++i) reinterpret_cast<__nv_bfloat16*>(p.out)[at * D + lane + 32 * i] = __float2bfloat16_rn(o[i] / l);
        if (p.lse && lane == 0) p.lse[at] = (m + log2f(l)) * 0.69314718055994530942f;
    }
}

}  // namespace
}  // namespace polyspec

using namespace polyspec;

extern "C" polyspec_status polyspec_prompt_attention(const void* q, long long q_stride, const void* k, long long k_stride, const void* v, long long v_stride,
                                                     const int32_t* rows_at, int n_seqs, int rows, int q_heads, int kv_heads, int head_dim, float scale,
                                                     void* out, float* lse, int32_t* device_status, void* cuda_stream)
{
    const polyspec_status st = kv::check_heads(q_heads, kv_heads, head_dim);
    if (n_seqs < 1 || rows < 1) return POLYSPEC_ERR_INVALID_ARG;
    if (st != POLYSPEC_OK) return st;
    if (rows > (1 << 24) || n_seqs > (1 << 20)) return POLYSPEC_ERR_UNSUPPORTED;
    if (!kv::rows_ok(q, q_stride, q_heads, head_dim) || !kv::rows_ok(k, k_stride, kv_heads, head_dim) || !kv::rows_ok(v, v_stride, kv_heads, head_dim))
        return POLYSPEC_ERR_INVALID_ARG;
    if (!rows_at || !out || !kv::aligned16(out) || !aligned4(rows_at, lse, device_status)) return POLYSPEC_ERR_INVALID_ARG;
    if (!(scale >= -3.0e38f && scale <= 3.0e38f)) return POLYSPEC_ERR_INVALID_ARG;
    PromptParams p = {static_cast<const unsigned short*>(q), static_cast<const unsigned short*>(k), static_cast<const unsigned short*>(v), q_stride, k_stride,
                      v_stride, rows_at, n_seqs, rows, q_heads, kv_heads, scale * 1.44269504088896340736f, static_cast<unsigned short*>(out), lse,
                      device_status};
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = head_dim == 128 ? launch_early(prompt_plain_kernel<128>, dim3(rows), 256, 0, stream, p)
                                          : launch_early(prompt_plain_kernel<64>, dim3(rows), 256, 0, stream, p);
    return cuda_failed(e) ? POLYSPEC_ERR_CUDA : POLYSPEC_OK;
}
