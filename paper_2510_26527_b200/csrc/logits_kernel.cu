// Sampling controls on the logits rows of a block: penalties for repeated tokens, biases and allowed-token masks, applied
// to every row with the context of THAT row -- the text so far and the drafted tokens before the row -- so that the
// verification that follows (Section 3.1: p_i(x | x_<=t) of every model of the chain) compares controlled distributions.
//
//   n(v)  occurrences of v in the output part of the history and in draft[0 .. j)      (row j of a block)
//   z1 = v in the history or the draft prefix ? (z > 0 ? z / r : z r) : z              repetition penalty r
//   z2 = z1 - f n(v) - p [n(v) > 0]                                                    frequency f, presence p
//   z3 = z2 + the biases listed for v;   z4 = v allowed ? z3 : -inf
// all in fp32, rounded once to the storage type.  An entry that no control touches keeps its bits.
//
// HBM-bound: every logit is read and written once, except that a vector of eight entries that the mask forbids as a whole
// is written without being read, and that in place (out == logits) only what a control touches moves at all.
// A CTA owns a slice of the vocabulary of one sequence and walks rows of the block.  It counts the history's tokens that
// fall into its slice in shared memory once (32-bit words: bit 31 seen in the prompt, bit 30 biased, below them n(v)),
// so the counts cost one read of the history per slice from L2 and no memory traffic.  Every vector of the slice belongs
// to one thread for all rows: which of its vectors hold anything is a few bits in a register, and the drafted token that
// joins the context between two rows is counted by its owner without a barrier.  Counting with integer atomics and adding
// listed biases in list order make the result independent of timing.
#include <algorithm>

#include "polyspec_kernels.cuh"
#include "stream_device.cuh"

namespace polyspec {
namespace {

constexpr int kThreads = 256;
constexpr int kVec = 8;                                 // entries per vector: one byte of the mask
constexpr uint32_t kSeenInPrompt = 1u << 31, kBiased = 1u << 30, kCountMask = kBiased - 1;

struct ControlParams {
    const void* logits;
    void* out;
    polyspec_logit_controls c;
    const int32_t* draft;
    int k;                      // row pitch of draft
    int B, rows, V;
    int mask_bytes;             // bytes of mask per row
    int slices, row_groups, rows_per_group;
    int32_t* status;
};

__device__ __forceinline__ void bad_input(int32_t* status)
{
    if (status) atomicCAS(status, 0, static_cast<int>(POLYSPEC_ERR_BAD_INPUT_ON_DEVICE));
}

// Eight logits as raw 16-byte words: one for 2-byte types, two for 4-byte types.
template <int DT> struct Vec8;
template <> struct Vec8<POLYSPEC_BF16> {
    uint4 a;
    __device__ __forceinline__ void load(const void* p, size_t e) { a = *reinterpret_cast<const uint4*>(static_cast<const char*>(p) + e * 2); }
    __device__ __forceinline__ void store(void* p, size_t e) const { *reinterpret_cast<uint4*>(static_cast<char*>(p) + e * 2) = a; }
    __device__ __forceinline__ void fill_neg_inf() { a = make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
    __device__ __forceinline__ void forbid(uint32_t allowed)
    {
        uint32_t* w = &a.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!(allowed >> (2 * i) & 1u)) w[i] = (w[i] & 0xffff0000u) | 0xff80u;
            if (!(allowed >> (2 * i + 1) & 1u)) w[i] = (w[i] & 0xffffu) | 0xff800000u;
        }
    }
    __device__ __forceinline__ float get(int i) const
    {
        const uint32_t w = (&a.x)[i >> 1];
        return __uint_as_float((i & 1) ? (w & 0xffff0000u) : (w << 16));
    }
    __device__ __forceinline__ void set(int i, float v)
    {
        uint32_t& w = (&a.x)[i >> 1];
        unsigned short h;
        asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(h) : "f"(v));
        w = (i & 1) ? ((w & 0xffffu) | (static_cast<uint32_t>(h) << 16)) : ((w & 0xffff0000u) | h);
    }
};
template <> struct Vec8<POLYSPEC_F32> {
    uint4 a, b;
    __device__ __forceinline__ void load(const void* p, size_t e)
    {
        const uint4* q = reinterpret_cast<const uint4*>(static_cast<const char*>(p) + e * 4);
        a = q[0];
        b = q[1];
    }
    __device__ __forceinline__ void store(void* p, size_t e) const
    {
        uint4* q = reinterpret_cast<uint4*>(static_cast<char*>(p) + e * 4);
        q[0] = a;
        q[1] = b;
    }
    __device__ __forceinline__ void fill_neg_inf() { a = b = make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
    __device__ __forceinline__ uint32_t& word(int i) { return i < 4 ? (&a.x)[i] : (&b.x)[i - 4]; }
    __device__ __forceinline__ void forbid(uint32_t allowed)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(allowed >> i & 1u)) word(i) = 0xff800000u;
    }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(i < 4 ? (&a.x)[i] : (&b.x)[i - 4]); }
    __device__ __forceinline__ void set(int i, float v) { word(i) = __float_as_uint(v); }
};

// One sequence's slice [v0, v0 + n) of the vocabulary, counted into `count` (and `bias`) by the whole CTA.
__device__ __forceinline__ void count_context(const ControlParams& p, int b, int v0, int n, bool report, uint32_t* count, float* bias)
{
    const int tid = threadIdx.x;
    for (int i = tid; i < n; i += kThreads) count[i] = 0;
    if (bias)
        for (int i = tid; i < n; i += kThreads) bias[i] = 0.0f;
    __syncthreads();
    const int first = p.c.vocab_begin + v0;
    if (p.c.history) {
        int len = p.c.history_len ? p.c.history_len[b] : p.c.history_cap;
        int prompt = p.c.prompt_len ? p.c.prompt_len[b] : 0;
        if (report && tid == 0 && (len < 0 || len > p.c.history_cap || prompt < 0 || prompt > len)) bad_input(p.status);
        len = min(max(len, 0), p.c.history_cap);
        prompt = min(max(prompt, 0), len);
        const int32_t* text = p.c.history + static_cast<size_t>(b) * p.c.history_cap;
        auto add = [&](int i, int t) {
            if (report && t >= p.c.vocab_size) bad_input(p.status);
            const unsigned at = static_cast<unsigned>(t) - static_cast<unsigned>(first);
            if (t >= 0 && at < static_cast<unsigned>(n)) {
                if (i < prompt) atomicOr(&count[at], kSeenInPrompt);
                else atomicAdd(&count[at], 1u);
            }
        };
        int i = tid;
        for (; i + 7 * kThreads < len; i += 8 * kThreads) {
            int t[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) t[u] = text[i + u * kThreads];
#pragma unroll
            for (int u = 0; u < 8; ++u) add(i + u * kThreads, t[u]);
        }
        for (; i < len; i += kThreads) add(i, text[i]);
    }
    if (bias && tid < 32) {
        // one warp walks the list 32 entries at a time; entries of one batch that name the same token are summed by the
        // first of them in list order
        const int32_t* toks = p.c.bias_tokens + static_cast<size_t>(b) * p.c.n_bias;
        const float* vals = p.c.bias_values + static_cast<size_t>(b) * p.c.n_bias;
        for (int i0 = 0; i0 < p.c.n_bias; i0 += 32) {
            const int i = i0 + tid;
            const int t = i < p.c.n_bias ? toks[i] : -1;
            const float x = i < p.c.n_bias ? vals[i] : 0.0f;
            if (report && t >= p.c.vocab_size) bad_input(p.status);
            const unsigned at = static_cast<unsigned>(t) - static_cast<unsigned>(first);
            const bool mine = t >= 0 && at < static_cast<unsigned>(n);
            const unsigned any = __ballot_sync(0xffffffffu, mine);
            if (!any) continue;
            const unsigned same = __match_any_sync(0xffffffffu, mine ? t : -1 - tid);
            float sum = mine ? bias[at] : 0.0f;
            for (unsigned left = any; left; left &= left - 1) {      // list order, every lane the same number of turns
                const int src = __ffs(left) - 1;
                const float y = __shfl_sync(0xffffffffu, x, src);
                if (same >> src & 1u) sum += y;
            }
            if (mine && tid == __ffs(same) - 1) {
                bias[at] = sum;
                atomicOr(&count[at], kBiased);
            }
            __syncwarp();
        }
    }
    __syncthreads();
}

// VPT vectors of eight entries per thread: a slice of kThreads * VPT * 8 entries.
// COUNTS: penalties or biases are there (the counts are needed); otherwise only a mask.
template <int DT, int VPT, bool COUNTS>
__global__ void __launch_bounds__(kThreads) logits_kernel(const ControlParams p)
{
    extern __shared__ uint4 smem_controls[];
    constexpr int kSlice = kThreads * VPT * kVec;
    const int tid = threadIdx.x;
    int at = blockIdx.x;
    const int slice = at % p.slices;
    at /= p.slices;
    const int group = at % p.row_groups, b = at / p.row_groups;
    const int v0 = slice * kSlice;
    const int n = min(kSlice, p.V - v0);
    const int j0 = group * p.rows_per_group, j1 = min(p.rows, j0 + p.rows_per_group);
    const bool report = slice == 0 && group == 0;
    const bool in_place = p.out == p.logits;

    uint32_t* count = reinterpret_cast<uint32_t*>(smem_controls);
    float* bias = COUNTS && p.c.bias_tokens ? reinterpret_cast<float*>(count + kSlice) : nullptr;
    uint32_t touched = 0;                               // bit u: vector u * kThreads + tid holds a counted or biased entry
    float r = 1.0f, f = 0.0f, pr = 0.0f;
    if (COUNTS) {
        count_context(p, b, v0, n, report, count, bias);
#pragma unroll
        for (int u = 0; u < VPT; ++u) {
            const int e = (u * kThreads + tid) * kVec;
            if (e < n) {
                const uint4 x = *reinterpret_cast<const uint4*>(count + e), y = *reinterpret_cast<const uint4*>(count + e + 4);
                if (x.x | x.y | x.z | x.w | y.x | y.y | y.z | y.w) touched |= 1u << u;
            }
        }
        if (p.c.repetition) r = p.c.repetition[b];
        if (p.c.frequency) f = p.c.frequency[b];
        if (p.c.presence) pr = p.c.presence[b];
        if (!(r > 0.0f)) {
            if (report && tid == 0) bad_input(p.status);
            r = 1.0f;
        }
    }
    // the drafted token at position j joins the context of the rows after it; its owner counts it
    auto join = [&](int j) {
        const int t = p.draft[static_cast<size_t>(b) * p.k + j];
        const unsigned e = static_cast<unsigned>(t) - static_cast<unsigned>(p.c.vocab_begin + v0);
        if (t >= 0 && e < static_cast<unsigned>(n) && static_cast<int>(e / kVec) % kThreads == tid) {
            count[e] += 1u;
            touched |= 1u << (e / kVec / kThreads);
        }
    };
    if (COUNTS && p.draft) {
        if (report && tid + 1 < p.rows && p.draft[static_cast<size_t>(b) * p.k + tid] >= p.c.vocab_size) bad_input(p.status);
        for (int j = 0; j < j0; ++j) join(j);
    }

    const unsigned char* mask = reinterpret_cast<const unsigned char*>(p.c.mask);
    auto mask_of = [&](int j, uint32_t (&m)[VPT]) {
#pragma unroll
        for (int u = 0; u < VPT; ++u) {
            const int e = (u * kThreads + tid) * kVec;
            m[u] = 0xffu;
            if (mask && j < j1 && e < n) m[u] = mask[(static_cast<size_t>(b) * p.rows + j) * p.mask_bytes + (v0 + e) / kVec];
        }
    };
    uint32_t allowed[VPT];
    mask_of(j0, allowed);
    for (int j = j0; j < j1; ++j) {
        const size_t row = (static_cast<size_t>(b) * p.rows + j) * p.V + v0;
        Vec8<DT> z[VPT];
        uint32_t next[VPT];
#pragma unroll
        for (int u = 0; u < VPT; ++u) {
            const int e = (u * kThreads + tid) * kVec;
            const bool moves = !in_place || (touched >> u & 1u) || allowed[u] != 0xffu;
            if (e < n && moves && allowed[u] != 0) z[u].load(p.logits, row + e);
        }
        mask_of(j + 1, next);
#pragma unroll
        for (int u = 0; u < VPT; ++u) {
            const int e = (u * kThreads + tid) * kVec;
            const bool moves = !in_place || (touched >> u & 1u) || allowed[u] != 0xffu;
            if (e >= n || !moves) continue;
            if (allowed[u] == 0) {
                z[u].fill_neg_inf();
            } else {
                if (COUNTS && (touched >> u & 1u)) {
#pragma unroll
                    for (int i = 0; i < kVec; ++i) {
                        const uint32_t w = count[e + i];
                        if (w == 0) continue;
                        float x = z[u].get(i);
                        const uint32_t times = w & kCountMask;
                        if (times || (w & kSeenInPrompt)) x = x > 0.0f ? x / r : x * r;
                        if (times) x = x - f * static_cast<float>(times) - pr;
                        if (w & kBiased) x += bias[e + i];
                        z[u].set(i, x);
                    }
                }
                if (allowed[u] != 0xffu) z[u].forbid(allowed[u]);
            }
            z[u].store(p.out, row + e);
        }
        if (COUNTS && p.draft && j + 1 < j1) join(j);
#pragma unroll
        for (int u = 0; u < VPT; ++u) allowed[u] = next[u];
    }
}

template <int DT, int VPT>
cudaError_t launch_vpt(ControlParams& p, bool counts, cudaStream_t stream)
{
    constexpr int kSlice = kThreads * VPT * kVec;
    p.slices = (p.V + kSlice - 1) / kSlice;
    p.row_groups = (p.rows + p.rows_per_group - 1) / p.rows_per_group;
    const long long blocks = static_cast<long long>(p.slices) * p.row_groups * p.B;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
    const size_t smem = counts ? static_cast<size_t>(kSlice) * (p.c.bias_tokens ? 8 : 4) : 0;
    if (counts) {
        if (smem > 48 * 1024) {
            cudaError_t e = cudaFuncSetAttribute(logits_kernel<DT, VPT, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
            if (e != cudaSuccess) return e;
        }
        logits_kernel<DT, VPT, true><<<static_cast<unsigned>(blocks), kThreads, smem, stream>>>(p);
    } else {
        logits_kernel<DT, VPT, false><<<static_cast<unsigned>(blocks), kThreads, 0, stream>>>(p);
    }
    return cudaGetLastError();
}

template <int DT>
cudaError_t launch_controls(ControlParams& p, bool counts, cudaStream_t stream)
{
    // Few sequences: smaller slices, then fewer rows per CTA, until there are about four CTAs for each of 148 SMs; many:
    // the largest slice and all rows of a sequence, so that the history is counted as seldom as possible.
    const long long want = 4 * 148;
    auto ctas = [&](int vpt, int rpg) {
        const long long s = (p.V + kThreads * vpt * kVec - 1) / (kThreads * vpt * kVec);
        return s * ((p.rows + rpg - 1) / rpg) * p.B;
    };
    int vpt = 4, rpg = p.rows;
    while (vpt > 1 && ctas(vpt, rpg) < want) vpt >>= 1;
    while (rpg > 1 && ctas(vpt, rpg) < want) rpg = (rpg + 1) / 2;
    p.rows_per_group = rpg;
    if (vpt == 4) return launch_vpt<DT, 4>(p, counts, stream);
    if (vpt == 2) return launch_vpt<DT, 2>(p, counts, stream);
    return launch_vpt<DT, 1>(p, counts, stream);
}

}  // namespace
}  // namespace polyspec

using namespace polyspec;

extern "C" polyspec_status polyspec_process_logits(
    const void* logits, const polyspec_logit_controls* controls, const int32_t* draft_tokens, int k, int B, int rows, int V,
    polyspec_dtype dt, void* out, int32_t* device_status, void* cuda_stream)
{
    if (!logits || !controls || !out || B <= 0 || rows <= 0 || V <= 0) return POLYSPEC_ERR_INVALID_ARG;
    if (dt != POLYSPEC_F32 && dt != POLYSPEC_BF16) return POLYSPEC_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(logits) & 15u) != 0 || (reinterpret_cast<uintptr_t>(out) & 15u) != 0) return POLYSPEC_ERR_INVALID_ARG;
    if (V % kVec != 0 || V > kMaxV) return POLYSPEC_ERR_UNSUPPORTED;
    if (static_cast<long long>(B) * ((V + kThreads * kVec - 1) / (kThreads * kVec)) * rows > 0x7fffffffLL) return POLYSPEC_ERR_UNSUPPORTED;   // CTAs
    ControlParams p;
    p.c = *controls;
    if (p.c.vocab_size == 0) p.c.vocab_size = p.c.vocab_begin == 0 ? V : 0;
    if (p.c.vocab_begin < 0 || p.c.vocab_size < V || p.c.vocab_begin > p.c.vocab_size - V) return POLYSPEC_ERR_INVALID_ARG;
    if (draft_tokens && (k < 1 || k > kMaxK || rows > k + 1)) return POLYSPEC_ERR_INVALID_ARG;
    if (p.c.history && p.c.history_cap < 1) return POLYSPEC_ERR_INVALID_ARG;
    if ((p.c.bias_tokens != nullptr) != (p.c.bias_values != nullptr)) return POLYSPEC_ERR_INVALID_ARG;
    if (p.c.bias_tokens && p.c.n_bias < 1) return POLYSPEC_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(p.c.mask) & 3u) != 0) return POLYSPEC_ERR_INVALID_ARG;
    const size_t bytes = static_cast<size_t>(B) * rows * V * (dt == POLYSPEC_BF16 ? 2 : 4);
    const uintptr_t a = reinterpret_cast<uintptr_t>(logits), o = reinterpret_cast<uintptr_t>(out);
    if (a != o && a < o + bytes && o < a + bytes) return POLYSPEC_ERR_INVALID_ARG;        // the same buffer, or none of it
    p.logits = logits;
    p.out = out;
    p.draft = draft_tokens;
    p.k = k;
    p.B = B;
    p.rows = rows;
    p.V = V;
    p.mask_bytes = (V + 31) / 32 * 4;
    p.status = device_status;
    const bool counts = p.c.history || draft_tokens || p.c.bias_tokens;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = dt == POLYSPEC_BF16 ? launch_controls<POLYSPEC_BF16>(p, counts, s) : launch_controls<POLYSPEC_F32>(p, counts, s);
    return cuda_failed(e) ? POLYSPEC_ERR_CUDA : POLYSPEC_OK;
}
