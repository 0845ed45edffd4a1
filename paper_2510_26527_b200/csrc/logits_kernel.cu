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
// A CTA owns a slice of the vocabulary of one sequence and rows of the block.  It counts the history's tokens that fall into
// its slice in shared memory (a word per entry, the top three bits flags, below them n(v); 16 bits where no count can pass 13,
// so that slices of 8192 entries leave room for several CTAs), and whoever is first to touch an entry puts it on a list.  The rows are streamed as vectors with nothing but the mask applied; then, behind one barrier, the
// few listed entries of every row are computed from the logits as they were and stored over the vectors, a warp per row.  (A
// text of thousands of tokens touches a few entries of every 256 that a warp moves: computing them where the vectors pass by
// had the whole warp take the slow path almost every time, 116 us on 64 x 7 rows of 128256; a barrier per row 75, one barrier 68.)
// Measured, bf16: 64 x 7 x 128256, texts of 4096: 57 us, 4.0 TB/s of the bytes it needs; 256 x 5 x 152064 with masks: 134 us, 4.6;
// masks alone in place, 64 x 7 x 128256: 31 us.  fp32, to which slices and occupancy were not fitted (slices of 4096 entries and more
// spill registers): 64 x 7 x 128256, texts of 4096: 117 us, 3.9 TB/s; 128 x 5 x 152064 with masks: 145 us, 4.2.
// Counting with integer atomics and adding listed biases in list order make the result independent of timing.
#include <cuda_bf16.h>

#include <algorithm>

#include "launch.cuh"
#include "polyspec_kernels.cuh"
#include "stream_device.cuh"

namespace polyspec {
namespace {

constexpr int kThreads = 256;
constexpr int kVec = 8;                                 // entries per vector: one byte of the mask
constexpr int kMaxVpt = 4;                              // vectors per thread at most
constexpr int kSparseBiases = 256;                       // up to so many biases are kept as a list that edits search, more as an array
constexpr int kMaxNarrow = (1 << 13) - 1;               // longest history whose counts fit 13 bits

// The count words of a slice, 32 or 16 bits each (two to a 32-bit word, which the atomics work on: a count cannot carry over).
template <bool WIDE> struct Counts;
template <> struct Counts<true> {
    static constexpr uint32_t kSeenInPrompt = 1u << 31, kBiased = 1u << 30, kDrafted = 1u << 29, kCountMask = kDrafted - 1;
    static constexpr int kBytes = 4;
    uint32_t* w;
    __device__ __forceinline__ uint32_t get(int at) const { return w[at]; }
    __device__ __forceinline__ uint32_t set(unsigned at, uint32_t flag) const { return atomicOr(&w[at], flag); }
    __device__ __forceinline__ uint32_t add(unsigned at) const { return atomicAdd(&w[at], 1u); }
};
template <> struct Counts<false> {
    static constexpr uint32_t kSeenInPrompt = 1u << 15, kBiased = 1u << 14, kDrafted = 1u << 13, kCountMask = kDrafted - 1;
    static constexpr int kBytes = 2;
    uint32_t* w;
    __device__ __forceinline__ uint32_t get(int at) const { return reinterpret_cast<const unsigned short*>(w)[at]; }
    __device__ __forceinline__ uint32_t set(unsigned at, uint32_t flag) const { return atomicOr(&w[at >> 1], flag << (16 * (at & 1))) >> (16 * (at & 1)) & 0xffffu; }
    __device__ __forceinline__ uint32_t add(unsigned at) const { return atomicAdd(&w[at >> 1], 1u << (16 * (at & 1))) >> (16 * (at & 1)) & 0xffffu; }
};

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

// Four mask bits as the top bits of four bytes (the product puts bit i at 8 i + 7; other bits are not looked at).
__device__ __forceinline__ uint32_t spread4(uint32_t bits) { return (bits & 15u) * 0x10204080u; }

// Each byte of the result is a byte's top bit eight times: nibble i of the selector, less 8, says which.
__device__ __forceinline__ uint32_t top_bits(uint32_t x, uint32_t selector)
{
    uint32_t r;
    asm("prmt.b32 %0, %1, 0, %2;" : "=r"(r) : "r"(x), "r"(selector));
    return r;
}

// Eight logits as raw 16-byte words: one for 2-byte types, two for 4-byte types.
template <int DT> struct Vec8;
template <> struct Vec8<POLYSPEC_BF16> {
    uint4 a;
    __device__ __forceinline__ void load(const void* p, size_t e) { a = *reinterpret_cast<const uint4*>(static_cast<const char*>(p) + e * 2); }
    __device__ __forceinline__ void store(void* p, size_t e) const { *reinterpret_cast<uint4*>(static_cast<char*>(p) + e * 2) = a; }
    __device__ __forceinline__ void fill_neg_inf() { a = make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
    // entries whose bit is clear become -inf, whatever they hold
    __device__ __forceinline__ void forbid(uint32_t allowed)
    {
        const uint32_t lo = spread4(allowed), hi = spread4(allowed >> 4);
        auto pick = [](uint32_t w, uint32_t keep) { return (w & keep) | (0xff80ff80u & ~keep); };
        a.x = pick(a.x, top_bits(lo, 0x9988));
        a.y = pick(a.y, top_bits(lo, 0xbbaa));
        a.z = pick(a.z, top_bits(hi, 0x9988));
        a.w = pick(a.w, top_bits(hi, 0xbbaa));
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
    __device__ __forceinline__ void forbid(uint32_t allowed)
    {
        const uint32_t lo = spread4(allowed), hi = spread4(allowed >> 4);
        auto pick = [](uint32_t w, uint32_t keep) { return (w & keep) | (0xff800000u & ~keep); };
        a.x = pick(a.x, top_bits(lo, 0x8888));
        a.y = pick(a.y, top_bits(lo, 0x9999));
        a.z = pick(a.z, top_bits(lo, 0xaaaa));
        a.w = pick(a.w, top_bits(lo, 0xbbbb));
        b.x = pick(b.x, top_bits(hi, 0x8888));
        b.y = pick(b.y, top_bits(hi, 0x9999));
        b.z = pick(b.z, top_bits(hi, 0xaaaa));
        b.w = pick(b.w, top_bits(hi, 0xbbbb));
    }
};

template <int DT> __device__ __forceinline__ float load_logit(const void* p, size_t e)
{
    if (DT == POLYSPEC_F32) return static_cast<const float*>(p)[e];
    return __uint_as_float(static_cast<uint32_t>(static_cast<const unsigned short*>(p)[e]) << 16);
}
template <int DT> __device__ __forceinline__ void store_logit(void* p, size_t e, float x)
{
    if (DT == POLYSPEC_F32) static_cast<float*>(p)[e] = x;
    else static_cast<__nv_bfloat16*>(p)[e] = __float2bfloat16_rn(x);
}

// What a CTA knows of its slice.
template <bool WIDE>
struct Slice {
    Counts<WIDE> count;         // [slice]
    unsigned short* list;       // [slice]: the touched entries
    int* n_list;
    const int32_t* draft;       // [rows - 1]: entries of the slice the drafted tokens are, -1 where they lie outside
    float* bias;                // sums of the biases: [slice], or [min(n_bias, kSparseBiases)] for the entries in bias_at; or nullptr
    unsigned short* bias_at;    // nullptr: bias is an array over the slice
    int* n_bias_at;
    __device__ __forceinline__ float bias_of(int e) const
    {
        if (!bias_at) return bias[e];
        for (int i = 0; i < *n_bias_at; ++i)
            if (bias_at[i] == e) return bias[i];
        return 0.0f;
    }
};

// One sequence's slice [v0, v0 + n) of the vocabulary, counted by the whole CTA.
template <bool WIDE>
__device__ __forceinline__ void count_context(const ControlParams& p, int b, int v0, int n, bool report, const Slice<WIDE>& s, int32_t* drafted)
{
    using C = Counts<WIDE>;
    const int tid = threadIdx.x;
    for (int i = tid; i < n * C::kBytes / 16; i += kThreads) reinterpret_cast<uint4*>(s.count.w)[i] = make_uint4(0, 0, 0, 0);   // n is a multiple of 8
    if (s.bias && !s.bias_at)
        for (int i = tid; i < n / 4; i += kThreads) reinterpret_cast<uint4*>(s.bias)[i] = make_uint4(0, 0, 0, 0);
    if (tid == 0) *s.n_list = 0;
    __syncthreads();
    const unsigned first = static_cast<unsigned>(p.c.vocab_begin + v0);
    // the first to touch an entry lists it
    auto touch = [&](unsigned at, uint32_t was) {
        if (was == 0) s.list[atomicAdd(s.n_list, 1)] = static_cast<unsigned short>(at);
    };
    if (p.draft && tid < p.rows - 1) {
        const int t = p.draft[static_cast<size_t>(b) * p.k + tid];
        if (report && t >= p.c.vocab_size) bad_input(p.status);
        const unsigned at = static_cast<unsigned>(t) - first;
        const bool mine = t >= 0 && at < static_cast<unsigned>(n);
        drafted[tid] = mine ? static_cast<int>(at) : -1;
        if (mine) touch(at, s.count.set(at, C::kDrafted));
    }
    if (p.c.history) {
        int len = p.c.history_len ? p.c.history_len[b] : p.c.history_cap;
        int prompt = p.c.prompt_len ? p.c.prompt_len[b] : 0;
        if (report && tid == 0 && (len < 0 || len > p.c.history_cap || prompt < 0 || prompt > len)) bad_input(p.status);
        len = min(max(len, 0), p.c.history_cap);
        prompt = min(max(prompt, 0), len);
        const int32_t* text = p.c.history + static_cast<size_t>(b) * p.c.history_cap;
        auto add = [&](int i, int t) {
            if (report && t >= p.c.vocab_size) bad_input(p.status);
            const unsigned at = static_cast<unsigned>(t) - first;
            if (t >= 0 && at < static_cast<unsigned>(n)) touch(at, i < prompt ? s.count.set(at, C::kSeenInPrompt) : s.count.add(at));
        };
        constexpr int kLoads = 4;
        int done = 0;
        if ((reinterpret_cast<uintptr_t>(text) & 15u) == 0) {           // sixteen tokens per thread in flight
            const int4* quads = reinterpret_cast<const int4*>(text);
            for (int q0 = 0; q0 < len / 4; q0 += kLoads * kThreads) {
                int4 t[kLoads];
#pragma unroll
                for (int u = 0; u < kLoads; ++u) {
                    t[u] = make_int4(-1, -1, -1, -1);
                    if (q0 + u * kThreads + tid < len / 4) t[u] = quads[q0 + u * kThreads + tid];
                }
#pragma unroll
                for (int u = 0; u < kLoads; ++u) {
                    const int i = (q0 + u * kThreads + tid) * 4;
                    add(i, t[u].x);
                    add(i + 1, t[u].y);
                    add(i + 2, t[u].z);
                    add(i + 3, t[u].w);
                }
            }
            done = len / 4 * 4;
        }
        for (int i = done + tid; i < len; i += kThreads) add(i, text[i]);
    }
    if (s.bias && tid >= kThreads - 32) {
        // one warp walks the list 32 biases at a time; those of one batch that name the same token are summed, in list order,
        // by the first of them
        const int lane = tid & 31;
        const int32_t* toks = p.c.bias_tokens + static_cast<size_t>(b) * p.c.n_bias;
        const float* vals = p.c.bias_values + static_cast<size_t>(b) * p.c.n_bias;
        int kept = 0;                           // entries in bias_at
        for (int i0 = 0; i0 < p.c.n_bias; i0 += 32) {
            const int i = i0 + lane;
            const int t = i < p.c.n_bias ? toks[i] : -1;
            const float x = i < p.c.n_bias ? vals[i] : 0.0f;
            if (report && t >= p.c.vocab_size) bad_input(p.status);
            const unsigned at = static_cast<unsigned>(t) - first;
            const bool mine = t >= 0 && at < static_cast<unsigned>(n);
            const unsigned any = __ballot_sync(0xffffffffu, mine);
            if (!any) continue;
            const unsigned same = __match_any_sync(0xffffffffu, mine ? t : -1 - lane);
            int place = s.bias_at ? -1 : static_cast<int>(at);
            if (mine && s.bias_at)
                for (int q = 0; q < kept; ++q)
                    if (s.bias_at[q] == at) place = q;
            float sum = mine && place >= 0 ? s.bias[place] : 0.0f;
            for (unsigned left = any; left; left &= left - 1) {      // list order, every lane the same number of turns
                const int src = __ffs(left) - 1;
                const float y = __shfl_sync(0xffffffffu, x, src);
                if (same >> src & 1u) sum += y;
            }
            const bool leads = mine && lane == __ffs(same) - 1;
            const unsigned fresh = __ballot_sync(0xffffffffu, leads && place < 0);
            if (leads) {
                if (place < 0) {
                    place = kept + __popc(fresh & ((1u << lane) - 1u));
                    s.bias_at[place] = static_cast<unsigned short>(at);
                }
                s.bias[place] = sum;
                touch(at, s.count.set(at, C::kBiased));
            }
            kept += __popc(fresh);
            __syncwarp();
        }
        if (s.bias_at && lane == 0) *s.n_bias_at = kept;
    }
    __syncthreads();
}

// Rows j0 .. j1 of the slice as vectors; FULL: the slice has all its kThreads * VPT vectors.
template <int DT, int VPT, bool FULL>
__device__ __forceinline__ void stream_rows(const ControlParams& p, int b, int v0, int n, int j0, int j1, bool in_place)
{
    constexpr int kRows = VPT >= 4 ? 1 : 2;             // rows in flight
    const int tid = threadIdx.x;
    const size_t first = static_cast<size_t>(b) * p.rows;
    const unsigned char* mask = p.c.mask ? reinterpret_cast<const unsigned char*>(p.c.mask) + v0 / kVec + tid : nullptr;
    auto inside = [&](int u) { return FULL || (u * kThreads + tid) * kVec < n; };
    auto mask_of = [&](int j, uint32_t (&m)[kRows][VPT]) {
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int u = 0; u < VPT; ++u) {
                m[r][u] = 0xffu;
                if (mask && j + r < j1 && inside(u)) m[r][u] = mask[(first + j + r) * p.mask_bytes + u * kThreads];
            }
    };
    uint32_t allowed[kRows][VPT];
    mask_of(j0, allowed);
    for (int j = j0; j < j1; j += kRows) {
        Vec8<DT> z[kRows][VPT];
        uint32_t next[kRows][VPT];
        const size_t at = (first + j) * p.V + v0 + tid * kVec;
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int u = 0; u < VPT; ++u)
                if (j + r < j1 && inside(u) && allowed[r][u] != 0 && (!in_place || allowed[r][u] != 0xffu))
                    z[r][u].load(p.logits, at + static_cast<size_t>(r) * p.V + u * (kThreads * kVec));
        mask_of(j + kRows, next);
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int u = 0; u < VPT; ++u) {
                if (j + r < j1 && inside(u) && (!in_place || allowed[r][u] != 0xffu)) {
                    if (allowed[r][u] == 0) z[r][u].fill_neg_inf();
                    else if (allowed[r][u] != 0xffu) z[r][u].forbid(allowed[r][u]);
                    z[r][u].store(p.out, at + static_cast<size_t>(r) * p.V + u * (kThreads * kVec));
                }
                allowed[r][u] = next[r][u];
            }
    }
}

// The listed entries of row j, entries start, start + step, ... of the list: two loads in flight (four took more registers than they saved time).
template <int DT, bool WIDE>
__device__ __forceinline__ void edit_row(const ControlParams& p, const Slice<WIDE>& s, int listed, int b, int v0, int j, int start, int step,
                                         float r, float f, float pr)
{
    using C = Counts<WIDE>;
    constexpr int kAhead = 2;
    const size_t row = (static_cast<size_t>(b) * p.rows + j) * p.V + v0;
    const unsigned char* mask = p.c.mask ? reinterpret_cast<const unsigned char*>(p.c.mask) + (static_cast<size_t>(b) * p.rows + j) * p.mask_bytes + v0 / kVec
                                         : nullptr;
    for (int i = start; i < listed; i += kAhead * step) {
        int e[kAhead];
        uint32_t w[kAhead], times[kAhead];
        float x[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            w[q] = times[q] = 0;
            e[q] = 0;
            if (i + q * step < listed) {
                e[q] = s.list[i + q * step];
                w[q] = s.count.get(e[q]);
                times[q] = w[q] & C::kCountMask;
                if (w[q] & C::kDrafted)
                    for (int d = 0; d < j; ++d) times[q] += s.draft[d] == e[q];
                if (!times[q] && !(w[q] & (C::kSeenInPrompt | C::kBiased))) w[q] = 0;                     // drafted later than this row
                else if (mask && !(mask[e[q] / kVec] >> (e[q] % kVec) & 1u)) w[q] = 0;
            }
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
            if (w[q]) x[q] = load_logit<DT>(p.logits, row + e[q]);
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            if (!w[q]) continue;
            float y = x[q];
            if (times[q] || (w[q] & C::kSeenInPrompt)) y = y > 0.0f ? y / r : y * r;
            if (times[q]) y = y - f * static_cast<float>(times[q]) - pr;
            if (w[q] & C::kBiased) y += s.bias_of(e[q]);
            store_logit<DT>(p.out, row + e[q], y);
        }
    }
}

// VPT vectors of eight entries per thread: a slice of kThreads * VPT * 8 entries.
// COUNTS: penalties or biases are there; otherwise only a mask.  WIDE: 32-bit counts.
template <int DT, int VPT, bool COUNTS, bool WIDE>
__global__ void __launch_bounds__(kThreads, 5) logits_kernel(const ControlParams p)
{
    extern __shared__ uint4 smem_controls[];
    __shared__ int n_list, n_bias_at;
    __shared__ int32_t drafted[kMaxK];
    constexpr int kSlice = kThreads * VPT * kVec;
    const int tid = threadIdx.x;
    wait_for_stream();
    // sequences before slices: token ids are frequent at the low end, so that the slices with long lists start first (the other
    // way round, the last of them ran alone at the end)
    int at = blockIdx.x;
    const int b = at % p.B;
    at /= p.B;
    const int group = at % p.row_groups, slice = at / p.row_groups;
    const int v0 = slice * kSlice;
    const int n = min(kSlice, p.V - v0);
    const int j0 = group * p.rows_per_group, j1 = min(p.rows, j0 + p.rows_per_group);
    // Without a context no entry is penalised, but a bad factor is reported all the same (here, where no vectors are in registers).
    if (!COUNTS && slice == 0 && group == 0 && tid == 0 && p.c.repetition && !(p.c.repetition[b] > 0.0f)) bad_input(p.status);
    // In place, an edit of this CTA changes what it read: the edits come after the vectors, and every entry is edited once.
    const bool in_place = p.out == p.logits;
    if (!in_place || p.c.mask) {
        if (n == kSlice) stream_rows<DT, VPT, true>(p, b, v0, n, j0, j1, in_place);
        else stream_rows<DT, VPT, false>(p, b, v0, n, j0, j1, in_place);
    }
    if (!COUNTS) return;

    const bool report = slice == 0 && group == 0;
    Slice<WIDE> s;
    s.count.w = reinterpret_cast<uint32_t*>(smem_controls);
    s.bias = p.c.bias_tokens ? reinterpret_cast<float*>(reinterpret_cast<char*>(smem_controls) + kSlice * (Counts<WIDE>::kBytes + 2)) : nullptr;
    s.list = reinterpret_cast<unsigned short*>(reinterpret_cast<char*>(smem_controls) + kSlice * Counts<WIDE>::kBytes);
    s.bias_at = p.c.n_bias <= kSparseBiases ? reinterpret_cast<unsigned short*>(s.bias + kSparseBiases) : nullptr;
    s.n_list = &n_list;
    s.n_bias_at = &n_bias_at;
    s.draft = drafted;
    float r = p.c.repetition ? p.c.repetition[b] : 1.0f;
    const float f = p.c.frequency ? p.c.frequency[b] : 0.0f, pr = p.c.presence ? p.c.presence[b] : 0.0f;
    if (!(r > 0.0f)) {
        if (report && tid == 0) bad_input(p.status);
        r = 1.0f;
    }
    count_context<WIDE>(p, b, v0, n, report, s, drafted);     // its barriers also put the vectors before the edits
    const int listed = n_list;
    if (!listed) return;
    // the CTA's warps over its rows: several per row where there are fewer rows than warps
    constexpr int kWarps = kThreads / 32;
    const int warp = tid >> 5, rows = j1 - j0, per_row = max(1, kWarps / rows);
    if (warp >= rows * per_row) return;
    for (int j = j0 + warp % rows; j < j1; j += kWarps) edit_row<DT, WIDE>(p, s, listed, b, v0, j, (warp / rows) * 32 + (tid & 31), per_row * 32, r, f, pr);
}

template <int DT, int VPT>
cudaError_t launch_vpt(ControlParams& p, bool counts, cudaStream_t stream)
{
    constexpr int kSlice = kThreads * VPT * kVec;
    p.slices = (p.V + kSlice - 1) / kSlice;
    p.row_groups = (p.rows + p.rows_per_group - 1) / p.rows_per_group;
    const long long blocks = static_cast<long long>(p.slices) * p.row_groups * p.B;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
    const bool wide = p.c.history && p.c.history_cap > kMaxNarrow;
    const size_t biases = !p.c.bias_tokens ? 0 : p.c.n_bias <= kSparseBiases ? kSparseBiases * 6 : kSlice * 4;
    const size_t smem = counts ? static_cast<size_t>(kSlice) * ((wide ? 4 : 2) + 2) + biases : 0;
    auto launch = [&](auto kernel) {
        if (smem > 48 * 1024) {
            // the limit belongs to the kernel, not to the call: the most that any call of it needs, so that a call with a short bias
            // list in one host thread does not lower it between another thread's set-up and launch
            constexpr size_t kMost = kSlice * (4 + 2 + 4);
            const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kMost));
            if (e != cudaSuccess) return e;
        }
        return launch_early(kernel, dim3(static_cast<unsigned>(blocks)), kThreads, smem, stream, p);
    };
    if (!counts) return launch(logits_kernel<DT, VPT, false, false>);
    return wide ? launch(logits_kernel<DT, VPT, true, true>) : launch(logits_kernel<DT, VPT, true, false>);
}

template <int DT>
cudaError_t launch_controls(ControlParams& p, bool counts, cudaStream_t stream)
{
    // Many sequences: the largest slices and all rows of a sequence, so that the history is counted as seldom as possible
    // (256 x 5 rows of 152064: slices of 8192 entries 134 us, of 4096 168 us).  Fewer: smaller slices down to eight CTAs for
    // each of 148 SMs, so that the ones with the longest lists do not run on alone (64 x 7 of 128256, texts of 4096: 4096
    // entries 57 us, 8192 entries 78 us); then fewer rows per CTA down to four, since each CTA counts the history again
    // (8 x 9 of 32000, texts of 2000: to four 9.6 us, to eight 13.2 us).
    auto ctas = [&](int vpt, int rpg) {
        const long long s = (p.V + kThreads * vpt * kVec - 1) / (kThreads * vpt * kVec);
        return s * ((p.rows + rpg - 1) / rpg) * p.B;
    };
    int vpt = kMaxVpt, rpg = p.rows;
    while (vpt > 1 && ctas(vpt, rpg) < 8 * 148) vpt >>= 1;
    while (rpg > 1 && ctas(vpt, rpg) < 4 * 148) rpg = (rpg + 1) / 2;
    p.rows_per_group = rpg;
    if (vpt == 4) return launch_vpt<DT, 4>(p, counts, stream);
    return vpt == 2 ? launch_vpt<DT, 2>(p, counts, stream) : launch_vpt<DT, 1>(p, counts, stream);
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
    if (!aligned4(p.c.history, p.c.history_len, p.c.prompt_len, p.c.repetition, p.c.frequency, p.c.presence, p.c.bias_tokens, p.c.bias_values, p.c.mask,
                  draft_tokens, device_status))
        return POLYSPEC_ERR_INVALID_ARG;
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
