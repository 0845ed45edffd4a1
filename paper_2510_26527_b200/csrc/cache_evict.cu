// Shortening caches to a budget by accumulated attention weight: of the tokens between the first few and the last few the
// heaviest stay, what stays moves together in every plane, pages behind it are given back.
//
// Two launches.  The first, one CTA per sequence, finds the weight of the last token that stays (radix selection over the weights' bits,
// four passes of eight bits), lists the slots that stay in order, moves the weights.  The second gives pages back and moves the contents: a CTA
// per sequence, head and run of planes goes through the kept tokens in order, kBatch at a time.  A token never moves up, so a batch that has been
// read before it is written overwrites nothing that a later batch reads.
//
// Moving is HBM-bound: each token that moves is read and written once, and of a unit of values that keeps any token everything is read (four neighbours
// share a sector).  Measured (B200): one sequence of 4300 tokens cut to 4096 in 64 planes of 8 heads of 128, 285 MB, 76 us, some 14 of them the first launch's
// chain of passes; 32 sequences of up to 2048 cut to 1024 in 64 planes of 4 heads 276 us, of which the moves are 260: 1.57 GB in and out, 6.0 TB/s.
#include <algorithm>
#include <type_traits>

#include "kv_pages.cuh"

namespace polyspec {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kMoveThreads = 256;
// Weights are held in shared memory through the selection where the tables have room for no more tokens than this: two launches for one sequence of 4300 tokens, two
// planes, 35 us against 36; 16 sequences of 8000 in tables for 65536 62.4 us read from memory each time, 63.2 with this room in shared memory.
constexpr int kKeyRoom = 49152;

struct EvictPlan {
    int32_t* head;          // [n_seqs, 4]: first new slot whose token moves, tokens kept, first page that goes, pages held (0, 0, 0, 0: sequence stays as it is)
    int32_t* from;          // [n_seqs, cap]: the slot that kept token i had
    float* weights;         // [n_seqs, cap]: its weight
    int32_t* pages;         // [n_seqs, max_pages]: the table as it was
};

inline size_t align256(size_t x) { return (x + 255) / 256 * 256; }
size_t evict_bytes(int n_seqs, int max_pages, int page_tokens)
{
    const size_t n = n_seqs, cap = static_cast<size_t>(max_pages) * page_tokens;
    return align256(n * 16) + 2 * align256(n * cap * 4) + align256(n * max_pages * 4);
}
EvictPlan evict_plan(void* workspace, int n_seqs, int max_pages, int page_tokens)
{
    const size_t n = n_seqs, cap = static_cast<size_t>(max_pages) * page_tokens;
    char* w = static_cast<char*>(workspace);
    EvictPlan p;
    p.head = reinterpret_cast<int32_t*>(w);
    w += align256(n * 16);
    p.from = reinterpret_cast<int32_t*>(w);
    w += align256(n * cap * 4);
    p.weights = reinterpret_cast<float*>(w);
    w += align256(n * cap * 4);
    p.pages = reinterpret_cast<int32_t*>(w);
    return p;
}

// Order of weights as order of unsigned numbers; both zeros alike, NaN below everything.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    if (w != w) return 0;
    const uint32_t u = __float_as_uint(w + 0.0f);
    return u >> 31 ? ~u : u | 0x80000000u;
}

// Exclusive prefix sums of two counts over the CTA; every thread calls it.
__device__ __forceinline__ int2 block_exclusive2(int2 x, int2* sums /* shared, 32 */, int2* total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int2 inc = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int a = __shfl_up_sync(0xffffffffu, inc.x, d), b = __shfl_up_sync(0xffffffffu, inc.y, d);
        if (lane >= d) { inc.x += a; inc.y += b; }
    }
    __syncthreads();
    if (lane == 31) sums[warp] = inc;
    __syncthreads();
    if (warp == 0) {
        int2 s = sums[lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int a = __shfl_up_sync(0xffffffffu, s.x, d), b = __shfl_up_sync(0xffffffffu, s.y, d);
            if (lane >= d) { s.x += a; s.y += b; }
        }
        sums[lane] = s;
    }
    __syncthreads();
    *total = sums[31];
    const int2 before = warp ? sums[warp - 1] : make_int2(0, 0);
    return make_int2(inc.x - x.x + before.x, inc.y - x.y + before.y);
}

__global__ void __launch_bounds__(kSelectThreads, 1) evict_select_kernel(const polyspec_cache_pages s, const int32_t* budgets, int first, int recent,
                                                                         float* weights, EvictPlan plan, int32_t* kept_from, int32_t* status, int key_room)
{
    extern __shared__ uint32_t keys[];          // of the slots, where there is room for all
    __shared__ int hist[256];
    __shared__ int2 sums[32];
    __shared__ uint32_t prefix;
    __shared__ int left, first_moved, shared_page;
    const int b = blockIdx.x, tid = threadIdx.x;
    const size_t cap = static_cast<size_t>(s.max_pages) * s.page_tokens;
    float* w = weights + b * cap;
    const int32_t* row = s.table + static_cast<size_t>(b) * s.max_pages;
    int32_t* from = plan.from + b * cap;
    wait_for_stream();
    const int len = s.len[b], budget = budgets[b];
    if (tid < 4) plan.head[4 * b + tid] = 0;
    bool stays = budget < 0 || len <= budget;
    if (len < 0 || len > static_cast<long long>(cap) || (!stays && budget < static_cast<long long>(first) + recent)) {
        if (tid == 0) kv::report(status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE);
        stays = true;
    }
    if (kept_from)
        for (size_t i = tid; i < cap; i += kSelectThreads) kept_from[b * cap + i] = -1;
    if (stays) return;

    const bool in_keys = len <= key_room;
    if (in_keys) {
        for (int i = tid; i < len; i += kSelectThreads) keys[i] = weight_key(w[i]);
        __syncthreads();
    }
    auto key_of = [&](int i) { return in_keys ? keys[i] : weight_key(w[i]); };

    // of the slots first .. len - recent - 1 the `need` heaviest stay
    const int end = len - recent, need = budget - first - recent;
    uint32_t bits = 0;                          // the leading bits of the last one's weight, as far as they are known
    int ties = need;                            // how many of equal leading bits stay
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int i0 = first + (tid & ~31); i0 < end; i0 += kSelectThreads) {
            const int i = i0 + (tid & 31);
            uint32_t digit = 256;               // of no interest
            if (i < end) {
                const uint32_t key = key_of(i);
                if (shift == 24 || key >> (shift + 8) == bits) digit = key >> shift & 255u;
            }
            // (weights of one size share their leading bits: one add per warp and digit)
            const uint32_t peers = __match_any_sync(0xffffffffu, digit);
            if (digit < 256 && (tid & 31) == __ffs(peers) - 1) atomicAdd(&hist[digit], __popc(peers));
        }
        __syncthreads();
        if (tid < 32) {                         // from the top digit down, eight digits a lane
            int sum = 0;
            for (int d = 0; d < 8; ++d) sum += hist[255 - tid * 8 - d];
            int inc = sum;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, inc, d);
                if (tid >= d) inc += y;
            }
            int above = inc - sum;
            if (above < ties && ties <= inc) {
                int d = 255 - tid * 8;
                while (above + hist[d] < ties) above += hist[d--];
                prefix = bits << 8 | d;
                left = ties - above;
            }
            if (tid == 0 && ties == 0) { prefix = 0xffffffffu; left = 0; }
        }
        __syncthreads();
        if (ties == 0) { bits = 0xffffffffu; break; }
        bits = prefix;
        ties = left;
    }
    // (with none to keep, no key is above ~0, which no number has)

    // slots in order, a run per thread: above the last one's weight, and equal to it
    const int per = (len + kSelectThreads - 1) / kSelectThreads;
    const int i0 = min(len, tid * per), i1 = min(len, i0 + per);
    auto state = [&](int i) {                   // 2 stays, 1 equal, 0 goes
        if (i < first || i >= end) return 2;
        const uint32_t key = key_of(i);
        return key > bits ? 2 : key == bits && need > 0 ? 1 : 0;
    };
    int2 mine = make_int2(0, 0), total;
    for (int i = i0; i < i1; ++i) {
        const int st = state(i);
        mine.x += st == 2;
        mine.y += st == 1;
    }
    if (tid == 0) { first_moved = budget; shared_page = 0; }
    const int2 before = block_exclusive2(mine, sums, &total);
    int equal = before.y, at = before.x + min(before.y, ties);
    int moved = budget;
    for (int i = i0; i < i1; ++i) {
        const int st = state(i);
        if (st == 2 || (st == 1 && equal < ties)) {
            if (at < budget) {
                from[at] = i;
                plan.weights[b * cap + at] = w[i];
                if (at != i) moved = min(moved, at);
            }
            ++at;
        }
        equal += st == 1;
    }
    if (moved < budget) atomicMin(&first_moved, moved);
    __syncthreads();

    // nobody else may hold a page that changes (none does where nothing moves); pages wholly behind what stays only lose this sequence's hold, in the second launch: until then every
    // sequence sees the holds as they were, whichever CTA comes first
    const int P = s.page_tokens, keep_pages = (budget + P - 1) / P, held = (len + P - 1) / P;
    for (int i = tid; i < held; i += kSelectThreads) {
        const int page = row[i];
        const bool there = page >= 0 && page < s.n_pages;
        if (!there || (first_moved < budget && i >= first_moved / P && i < keep_pages && s.refs[page] > 1)) shared_page = 1;
        plan.pages[static_cast<size_t>(b) * s.max_pages + i] = page;
    }
    __syncthreads();
    if (shared_page) {
        if (tid == 0) kv::report(status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE);
        return;
    }
    for (int i = first_moved + tid; i < budget; i += kSelectThreads) w[i] = plan.weights[b * cap + i];
    if (kept_from)
        for (int i = tid; i < budget; i += kSelectThreads) kept_from[b * cap + i] = from[i];
    if (tid == 0) {
        s.len[b] = budget;
        plan.head[4 * b] = first_moved;
        plan.head[4 * b + 1] = budget;
        plan.head[4 * b + 2] = keep_pages;
        plan.head[4 * b + 3] = held;
    }
}

// D: head_dim.  blockIdx.x: key head and a run of planes, blockIdx.y: sequence.  Where a batch's tokens come from and go to is found once for all of the
// CTA's planes (divisions by the page's size took more time than the copies), a batch ahead of its use.
template <int D>
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const polyspec_cache_pages s, EvictPlan plan, unsigned char* pool, size_t page_bytes,
                                                                  int kv_heads, int n_planes, int run, int32_t* status)
{
    constexpr int kBatch = kMoveThreads;        // tokens at a time
    constexpr int kPieces = D / 32;             // 16-byte pieces of a token's codes
    constexpr int UB = kv::unit_bytes(D);
    using Piece = typename std::conditional<D == 128, uint2, uint32_t>::type;         // the D / 64 words of one group of lanes
    __shared__ uint2 places[3][2][kBatch];      // [turn][from, to]: unit of the plane, token of the unit; of three batches in a row
    const int b = blockIdx.y, head = blockIdx.x % kv_heads, plane0 = blockIdx.x / kv_heads * run, planes = min(run, n_planes - plane0), tid = threadIdx.x;
    const int P = s.page_tokens, units = P / kv::kUnit;
    const size_t cap = static_cast<size_t>(s.max_pages) * P;
    const int32_t* from = plan.from + b * cap;
    const int32_t* pages = plan.pages + static_cast<size_t>(b) * s.max_pages;
    wait_for_stream();
    const int begin = plan.head[4 * b], end = plan.head[4 * b + 1];
    if (blockIdx.x == 0)                        // the sequence's hold on what lies wholly behind
        for (int i = plan.head[4 * b + 2] + tid; i < plan.head[4 * b + 3]; i += kMoveThreads) {
            const int page = pages[i], was = atomicSub(&s.refs[page], 1);
            if (was == 1) atomicOr(&s.free_bits[page >> 5], 1u << (page & 31));
            else if (was <= 0) { atomicAdd(&s.refs[page], 1); kv::report(status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE); }
            s.table[static_cast<size_t>(b) * s.max_pages + i] = -1;
        }
    if (begin >= end) return;
    auto place = [&](int slot) {
        const int unit = slot / kv::kUnit, at = unit / units;
        return make_uint2((static_cast<uint32_t>(pages[at]) * kv_heads + head) * units + (unit - at * units), slot % kv::kUnit);
    };
    auto find = [&](int turn, int i) {
        if (i < end - tid) {
            places[turn][0][tid] = place(from[i + tid]);
            places[turn][1][tid] = place(i + tid);
        }
    };
    // An item is a batch of one plane.  The next one's loads are under way while this one's are waited for and stored: what they read lies behind what
    // this one writes, or in another plane.
    struct Held { uint4 codes[kPieces]; uint32_t pair; };       // keys: pieces of tokens; values: a token's words, in the order of their groups
    struct At { int i0, k, turn; };                             // batch, plane of the run, which third of `places`
    auto unit = [&](const At& at, int which, int t) {
        return pool + (static_cast<size_t>(plane0 + at.k) * s.n_pages * page_bytes + static_cast<size_t>(places[at.turn][which][t].x) * UB);
    };
    auto next = [&](At& at) {
        if (++at.k < planes) return;
        at.k = 0;
        at.i0 += kBatch;
        at.turn = at.turn == 2 ? 0 : at.turn + 1;
    };
    auto load = [&](const At& at, Held& x) {
        const int n = min(kBatch, end - at.i0);
        if (tid < n) x.pair = reinterpret_cast<const uint32_t*>(unit(at, 0, tid))[D + places[at.turn][0][tid].y];
        if (!((plane0 + at.k) & 1)) {
#pragma unroll
            for (int u = 0; u < kPieces; ++u) {
                const int item = u * kMoveThreads + tid, t = item / kPieces, part = item % kPieces;
                if (t < n) x.codes[u] = reinterpret_cast<const uint4*>(unit(at, 0, t))[places[at.turn][0][t].y * kPieces + part];
            }
        } else if (tid < n) {                   // neighbouring lanes have neighbouring tokens: a group's words of a unit are neighbours
            const Piece* from = reinterpret_cast<const Piece*>(unit(at, 0, tid)) + places[at.turn][0][tid].y;
            Piece* y = reinterpret_cast<Piece*>(x.codes);
#pragma unroll
            for (int u = 0; u < 8; ++u) y[u] = from[8 * u];
        }
    };
    auto store = [&](const At& at, const Held& x) {
        const int n = min(kBatch, end - at.i0);
        if (!((plane0 + at.k) & 1)) {
#pragma unroll
            for (int u = 0; u < kPieces; ++u) {
                const int item = u * kMoveThreads + tid, t = item / kPieces, part = item % kPieces;
                if (t < n) reinterpret_cast<uint4*>(unit(at, 1, t))[places[at.turn][1][t].y * kPieces + part] = x.codes[u];
            }
        } else if (tid < n) {
            Piece* to = reinterpret_cast<Piece*>(unit(at, 1, tid)) + places[at.turn][1][tid].y;
            const Piece* y = reinterpret_cast<const Piece*>(x.codes);
#pragma unroll
            for (int u = 0; u < 8; ++u) to[8 * u] = y[u];
        }
        if (tid < n) reinterpret_cast<uint32_t*>(unit(at, 1, tid))[D + places[at.turn][1][tid].y] = x.pair;
    };
    Held one, two;
    At at = {begin, 0, 0};
    find(0, begin);
    __syncthreads();
    load(at, one);
    find(1, begin + kBatch);
    auto step = [&](Held& mine, Held& coming) {
        At ahead = at;
        next(ahead);
        __syncthreads();                        // everything of this item has been read; the next batch's places are known
        if (ahead.i0 < end) load(ahead, coming);
        // the places of the batch after that, by the time of the loads: they take the third of the batch before this one, which all threads have stored
        if (ahead.k == 0) find(ahead.turn == 2 ? 0 : ahead.turn + 1, ahead.i0 + kBatch);
        store(at, mine);
        at = ahead;
        return at.i0 < end;
    };
    while (step(one, two) && step(two, one)) {}
}

}  // namespace
}  // namespace polyspec

using namespace polyspec;

extern "C" {

polyspec_status polyspec_cache_evict_workspace(int n_seqs, int max_pages, int page_tokens, size_t* bytes)
{
    if (!bytes || n_seqs < 1 || max_pages < 1 || page_tokens < 1) return POLYSPEC_ERR_INVALID_ARG;
    if (static_cast<long long>(max_pages) * page_tokens > kv::kMostTokens) return POLYSPEC_ERR_UNSUPPORTED;
    *bytes = evict_bytes(n_seqs, max_pages, page_tokens);
    return POLYSPEC_OK;
}

polyspec_status polyspec_cache_evict(const polyspec_cache_pages* s, const int32_t* budget, int first, int recent, float* weights, void* pool,
                                     int n_planes, int kv_heads, int head_dim, int32_t* kept_from, int32_t* device_status, void* workspace,
                                     size_t workspace_bytes, void* cuda_stream)
{
    polyspec_status st = kv::check_state(s);
    if (st == POLYSPEC_OK) st = kv::check_heads(kv_heads, kv_heads, head_dim);
    if (st != POLYSPEC_OK) return st;
    if (!budget || first < 0 || recent < 0 || !weights || !pool || !kv::aligned16(pool) || n_planes < 2 || n_planes % 2) return POLYSPEC_ERR_INVALID_ARG;
    if (!aligned4(budget, weights, kept_from, device_status)) return POLYSPEC_ERR_INVALID_ARG;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return POLYSPEC_ERR_INVALID_ARG;
    if (s->n_pages * (kv::page_bytes(*s, kv_heads, head_dim) / kv::unit_bytes(head_dim)) >= 0xffffffffull) return POLYSPEC_ERR_UNSUPPORTED;
    if (s->n_seqs > 65535 || static_cast<long long>(n_planes) * kv_heads > 0x7fffffffLL) return POLYSPEC_ERR_UNSUPPORTED;
    if (workspace_bytes < evict_bytes(s->n_seqs, s->max_pages, s->page_tokens)) return POLYSPEC_ERR_WORKSPACE;
    const EvictPlan plan = evict_plan(workspace, s->n_seqs, s->max_pages, s->page_tokens);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const size_t cap = static_cast<size_t>(s->max_pages) * s->page_tokens;
    const int room = cap <= kKeyRoom ? static_cast<int>(cap) : 0;
    cudaError_t e = cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kKeyRoom * 4);
    if (e == cudaSuccess)
        e = launch_early(evict_select_kernel, dim3(static_cast<unsigned>(s->n_seqs)), kSelectThreads, static_cast<size_t>(room) * 4, stream, *s, budget, first,
                         recent, weights, plan, kept_from, device_status, room);
    if (e == cudaSuccess) {
        // planes per CTA: as many as leave some thousand CTAs
        const long long all = static_cast<long long>(n_planes) * kv_heads * s->n_seqs;
        const int run = static_cast<int>(std::max<long long>(1, std::min<long long>(n_planes, all / 2048)));
        const dim3 grid(static_cast<unsigned>((n_planes + run - 1) / run * kv_heads), static_cast<unsigned>(s->n_seqs));
        unsigned char* data = static_cast<unsigned char*>(pool);
        const size_t bytes = kv::page_bytes(*s, kv_heads, head_dim);
        e = head_dim == 128 ? launch_early(evict_move_kernel<128>, grid, kMoveThreads, 0, stream, *s, plan, data, bytes, kv_heads, n_planes, run, device_status)
                            : launch_early(evict_move_kernel<64>, grid, kMoveThreads, 0, stream, *s, plan, data, bytes, kv_heads, n_planes, run, device_status);
    }
    return cuda_failed(e) ? POLYSPEC_ERR_CUDA : POLYSPEC_OK;
}

}  // extern "C"
