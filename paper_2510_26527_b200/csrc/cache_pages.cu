// Page tables of a model's cache, kept on the device around the verification of a block: room for the block is reserved
// before the forward pass, what was not accepted is rolled back after it (Algorithm 1: "roll back" to the committed text),
// sequences are forked for parallel continuations, and a pool full of holes is compacted.  Nothing is read back.
//
// State: table [n_seqs, max_pages] page numbers, len [n_seqs] tokens held, refs [n_pages] table entries naming each page,
// free_bits: bit p set iff refs[p] == 0.  A set bit is the whole free list: pages are taken by ascending number in the
// order of the sequences, so the outcome depends on the state alone, never on timing; the bitmap of a pool of 100 000 pages
// is 12 KB, which one CTA reads in a single sweep.
//
// The bookkeeping calls are latency-bound: one CTA (reserve, compact) or one warp per sequence (rollback, fork), one launch.
// Moving page contents is HBM-bound: warps copy 2 KiB pieces, four independent 16-byte loads per lane before the stores.
// Measured: reserve and rollback of 64 sequences in a pool of 41500 pages 7.6 to 8.2 us together; compacting 48 planes of 4000 pages
// of 8 KiB, 114 to 118 us in the moves, 5.9 TB/s of DRAM traffic.
#include "launch.cuh"
#include "polyspec_kernels.cuh"

namespace polyspec {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPiece = 2048;                    // bytes a warp copies at a time
constexpr int kMaxPools = POLYSPEC_CACHE_MAX_POOLS;
constexpr int kMaxPages = 1 << 20;              // 1024 needs of at most this many pages each add up within 31 bits

// Workspace of reserve and compact: the number of copies, then (from, to) of each, then a scratch list of page numbers.
struct Plan {
    int32_t* n_copies;      // [1]
    int2* copies;           // [max(n_seqs, n_pages)]
    int32_t* pages;         // [n_pages]
    int32_t* starts;        // [n_seqs]
};

inline size_t align256(size_t x) { return (x + 255) / 256 * 256; }

size_t plan_bytes(int n_seqs, int n_pages)
{
    const size_t pairs = n_seqs > n_pages ? n_seqs : n_pages;
    return 256 + align256(pairs * sizeof(int2)) + align256(static_cast<size_t>(n_pages) * 4) + align256(static_cast<size_t>(n_seqs) * 4);
}

Plan plan_of(void* workspace, int n_seqs, int n_pages)
{
    char* w = static_cast<char*>(workspace);
    const size_t pairs = n_seqs > n_pages ? n_seqs : n_pages;
    Plan p;
    p.n_copies = reinterpret_cast<int32_t*>(w);
    w += 256;
    p.copies = reinterpret_cast<int2*>(w);
    w += align256(pairs * sizeof(int2));
    p.pages = reinterpret_cast<int32_t*>(w);
    w += align256(static_cast<size_t>(n_pages) * 4);
    p.starts = reinterpret_cast<int32_t*>(w);
    return p;
}

__device__ __forceinline__ void report(int32_t* status, polyspec_status what)
{
    if (status) atomicCAS(status, 0, static_cast<int>(what));
}

// Exclusive prefix sum over the CTA (kPlanThreads threads, every one calls it); *total is the sum.
__device__ __forceinline__ int block_exclusive(int x, int* sums /* shared, 33 */, int* total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int inc = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, d);
        if (lane >= d) inc += y;
    }
    __syncthreads();                            // the sums of an earlier call have been read
    if (lane == 31) sums[warp] = inc;
    __syncthreads();
    if (warp == 0) {
        int s = sums[lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, s, d);
            if (lane >= d) s += y;
        }
        sums[lane] = s;
    }
    __syncthreads();
    *total = sums[31];
    return inc - x + (warp ? sums[warp - 1] : 0);
}

__device__ __forceinline__ int pages_for(int tokens, int page_tokens) { return tokens / page_tokens + (tokens % page_tokens != 0); }

__device__ __forceinline__ long long target_len(const int32_t* base, const int32_t* extra, int plus, int b)
{
    return static_cast<long long>(base[b]) + (extra ? extra[b] : 0) + plus;
}

// One reference less; the page is free once none is left.
__device__ __forceinline__ void drop_page(const polyspec_cache_pages& s, int page, int32_t* status)
{
    if (page < 0 || page >= s.n_pages) { report(status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE); return; }
    const int was = atomicSub(&s.refs[page], 1);
    if (was == 1) atomicOr(&s.free_bits[page >> 5], 1u << (page & 31));
    else if (was <= 0) { atomicAdd(&s.refs[page], 1); report(status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE); }
}

// Word w of the free bitmap, without bits behind the last page.
__device__ __forceinline__ uint32_t free_word(const polyspec_cache_pages& s, int w)
{
    const uint32_t valid = s.n_pages >= 32 * (w + 1) ? 0xffffffffu : (1u << (s.n_pages - 32 * w)) - 1u;
    return s.free_bits[w] & valid;
}

// Sequence b's length if it is one the table can hold, else -1.
__device__ __forceinline__ int held_len(const polyspec_cache_pages& s, int b)
{
    const int len = s.len[b];
    return len >= 0 && len <= s.max_pages * s.page_tokens ? len : -1;
}

// What sequence b needs to grow to `want`: pages to add, and whether its last page, which others hold too, is copied first.
struct Need { bool grow, copy, bad, too_long; int len, want, pages; };
__device__ __forceinline__ Need need_of(const polyspec_cache_pages& s, const int32_t* base, const int32_t* extra, int plus, int b)
{
    Need q = {false, false, false, false, 0, 0, 0};
    const long long want = target_len(base, extra, plus, b);
    q.len = held_len(s, b);
    if (q.len < 0) { q.bad = true; return q; }
    if (want <= q.len) return q;
    if (want > static_cast<long long>(s.max_pages) * s.page_tokens) { q.too_long = true; return q; }
    q.grow = true;
    q.want = static_cast<int>(want);
    q.pages = pages_for(q.want, s.page_tokens) - pages_for(q.len, s.page_tokens);
    if (q.len % s.page_tokens != 0) {
        const int last = s.table[static_cast<size_t>(b) * s.max_pages + q.len / s.page_tokens];
        if (last < 0 || last >= s.n_pages) { q.bad = true; q.grow = false; q.pages = 0; return q; }
        q.copy = s.refs[last] > 1;
    }
    return q;
}

// Reserve: one CTA.  Needs are read before anything is written, so two sequences that share a last page both copy it.
__global__ void __launch_bounds__(kPlanThreads, 1) reserve_kernel(const polyspec_cache_pages s, const int32_t* base, const int32_t* extra, int plus,
                                                                  Plan plan, int32_t* status)
{
    __shared__ int sums[33];
    __shared__ int taken, n_copies;
    __shared__ unsigned long long failure;      // the lowest sequence that fails, above its status: one report, whoever comes first
    const int tid = threadIdx.x;
    const int words = (s.n_pages + 31) / 32;
    const int per = (words + kPlanThreads - 1) / kPlanThreads;          // consecutive words of the free bitmap per thread
    const int w0 = min(words, tid * per), w1 = min(words, w0 + per);
    if (tid == 0) { taken = 0; n_copies = 0; failure = ~0ull; }
    wait_for_stream();
    // the first sequences' needs are read beside the bitmap: both are chains of dependent loads
    Need first = {false, false, false, false, 0, 0, 0};
    if (tid < s.n_seqs) first = need_of(s, base, extra, plus, tid);
    int mine = 0;
    for (int w = w0; w < w1; ++w) mine += __popc(free_word(s, w));
    int n_free, total;
    const int my_rank = block_exclusive(mine, sums, &n_free);

    // sequences in order: as many as the free pages suffice for
    int before = 0;
    for (int b0 = 0; b0 < s.n_seqs; b0 += kPlanThreads) {
        const int b = b0 + tid;
        Need q = first;
        if (b0 > 0) q = b < s.n_seqs ? need_of(s, base, extra, plus, b) : Need{false, false, false, false, 0, 0, 0};
        const int n = q.grow ? q.pages + (q.copy ? 1 : 0) : 0;
        // a running sum past the pool's size says no more than the pool's size does: it is held there, so it cannot overflow
        const int start = before + block_exclusive(min(n, s.n_pages + 1), sums, &total);
        const bool ok = q.grow && (n == 0 || (start >= 0 && start <= n_free - n));
        if (b < s.n_seqs) {
            plan.starts[b] = ok ? (start << 1 | (q.copy ? 1 : 0)) : -1;
            const polyspec_status st = q.bad || q.too_long ? POLYSPEC_ERR_BAD_INPUT_ON_DEVICE : q.grow && !ok ? POLYSPEC_ERR_NO_PAGES : POLYSPEC_OK;
            if (st != POLYSPEC_OK) atomicMin(&failure, static_cast<unsigned long long>(b) << 8 | st);
            if (ok && n > 0) atomicMax(&taken, start + n);
        }
        before = min(before + total, s.n_pages + 1);
    }
    __syncthreads();
    if (tid == 0 && failure != ~0ull) report(status, static_cast<polyspec_status>(failure & 0xff));

    // the lowest `taken` free pages, ascending; they are in use from here on
    int rank = my_rank;
    for (int w = w0; w < w1 && rank < taken; ++w) {
        uint32_t bits = free_word(s, w);
        uint32_t left = bits;
        while (left && rank < taken) {
            const int bit = __ffs(left) - 1;
            left &= left - 1;
            bits &= ~(1u << bit);
            const int page = w * 32 + bit;
            plan.pages[rank++] = page;
            s.refs[page] = 1;
        }
        s.free_bits[w] = bits;
    }
    __syncthreads();

    // a warp per sequence writes its new entries
    const int lane = tid & 31;
    for (int b = tid >> 5; b < s.n_seqs; b += kPlanThreads / 32) {
        const int code = plan.starts[b];
        if (code < 0) continue;
        const int len = s.len[b];
        const int want = static_cast<int>(target_len(base, extra, plus, b));
        const int held = pages_for(len, s.page_tokens), wanted = pages_for(want, s.page_tokens);
        int32_t* row = s.table + static_cast<size_t>(b) * s.max_pages;
        const int copy = code & 1;
        const int32_t* from = plan.pages + (code >> 1) + copy;
        for (int i = lane; i < wanted - held; i += 32) row[held + i] = from[i];
        __syncwarp();
        if (lane == 0) {
            if (copy) {
                const int old = row[held - 1], fresh = plan.pages[code >> 1];
                row[held - 1] = fresh;
                drop_page(s, old, status);
                plan.copies[atomicAdd(&n_copies, 1)] = make_int2(old, fresh);
            }
            s.len[b] = want;
        }
    }
    __syncthreads();
    if (tid == 0) *plan.n_copies = n_copies;
}

// Rollback: a warp per sequence gives back the pages wholly behind the new end.
__global__ void rollback_kernel(const polyspec_cache_pages s, const int32_t* base, const int32_t* extra, int plus, int32_t* status)
{
    const int b = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    wait_for_stream();
    if (b >= s.n_seqs) return;
    const long long to = target_len(base, extra, plus, b);
    const int len = held_len(s, b);
    if (len < 0) {
        if (lane == 0) report(status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE);
        return;
    }
    if (to < 0 || to >= len) return;
    const int first = pages_for(static_cast<int>(to), s.page_tokens), end = pages_for(len, s.page_tokens);
    int32_t* row = s.table + static_cast<size_t>(b) * s.max_pages;
    for (int i = first + lane; i < end; i += 32) {
        drop_page(s, row[i], status);
        row[i] = -1;
    }
    __syncwarp();
    if (lane == 0) s.len[b] = static_cast<int>(to);
}

// Fork: a warp per pair; dst, which must hold nothing, takes src's pages and length.  A pair is refused when a number is out
// of range, dst holds tokens, src is any pair's dst, or an earlier pair names the same dst: so no two warps write one row.
__global__ void fork_kernel(const polyspec_cache_pages s, const int32_t* src, const int32_t* dst, int n, int32_t* status)
{
    const int i = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    wait_for_stream();
    if (i >= n) return;
    const int from = src[i], to = dst[i];
    if (from < 0 && to < 0) return;                                     // an unused slot of the list
    bool bad = from < 0 || to < 0 || from >= s.n_seqs || to >= s.n_seqs;
    for (int j = lane; j < n; j += 32) {
        const int d = dst[j];
        if (d == from || (j < i && d == to)) bad = true;
    }
    bad = __any_sync(0xffffffffu, bad);
    int len = -1;
    if (!bad) {
        len = held_len(s, from);
        bad = len < 0 || s.len[to] != 0;
    }
    if (bad) {
        if (lane == 0) report(status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE);
        return;
    }
    const int32_t* row = s.table + static_cast<size_t>(from) * s.max_pages;
    int32_t* out = s.table + static_cast<size_t>(to) * s.max_pages;
    const int held = pages_for(len, s.page_tokens);
    bool whole = true;
    for (int c = lane; c < held; c += 32) {
        const int page = row[c];
        whole = whole && page >= 0 && page < s.n_pages;
    }
    if (!__all_sync(0xffffffffu, whole)) {
        if (lane == 0) report(status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE);
        return;
    }
    for (int c = lane; c < held; c += 32) {
        const int page = row[c];
        out[c] = page;
        atomicAdd(&s.refs[page], 1);
    }
    __syncwarp();
    if (lane == 0) s.len[to] = len;
}

// Compact, bookkeeping: one CTA.  With n_live pages in use, the i-th used page numbered n_live or more moves to the i-th
// free page below n_live, so sources and destinations of the moves never overlap.
__global__ void __launch_bounds__(kPlanThreads, 1) compact_kernel(const polyspec_cache_pages s, Plan plan, int32_t* moved_to)
{
    __shared__ int sums[33];
    const int tid = threadIdx.x;
    const int words = (s.n_pages + 31) / 32;
    const int per = (words + kPlanThreads - 1) / kPlanThreads;
    const int w0 = min(words, tid * per), w1 = min(words, w0 + per);
    int mine = 0, n_free, n_moves;
    wait_for_stream();
    for (int w = w0; w < w1; ++w) mine += __popc(free_word(s, w));
    block_exclusive(mine, sums, &n_free);
    const int n_live = s.n_pages - n_free;
    // bits of word w that lie below n_live
    auto below = [&](int w) { return n_live >= 32 * (w + 1) ? 0xffffffffu : n_live <= 32 * w ? 0u : (1u << (n_live - 32 * w)) - 1u; };
    auto valid = [&](int w) { return s.n_pages >= 32 * (w + 1) ? 0xffffffffu : (1u << (s.n_pages - 32 * w)) - 1u; };
    int holes = 0, movers = 0;
    for (int w = w0; w < w1; ++w) {
        holes += __popc(free_word(s, w) & below(w));
        movers += __popc(~free_word(s, w) & ~below(w) & valid(w));
    }
    int hole = block_exclusive(holes, sums, &n_moves);
    int total;
    int mover = block_exclusive(movers, sums, &total);
    for (int w = w0; w < w1; ++w) {
        const uint32_t bits = free_word(s, w);
        for (uint32_t left = bits & below(w); left; left &= left - 1) plan.copies[hole++].y = w * 32 + __ffs(left) - 1;
        for (uint32_t left = ~bits & ~below(w) & valid(w); left; left &= left - 1) plan.copies[mover++].x = w * 32 + __ffs(left) - 1;
        s.free_bits[w] = ~below(w) & valid(w);
        if (moved_to)
            for (int i = w * 32; i < min(s.n_pages, w * 32 + 32); ++i) moved_to[i] = (bits >> (i & 31) & 1u) ? -1 : i;
    }
    __syncthreads();
    for (int i = tid; i < n_moves; i += kPlanThreads) {
        const int2 m = plan.copies[i];
        s.refs[m.y] = s.refs[m.x];
        s.refs[m.x] = 0;
        if (moved_to) moved_to[m.x] = m.y;
    }
    if (tid == 0) {
        *plan.n_copies = n_moves;
        plan.starts[0] = n_live;
    }
}

// Compact, tables: entries that name a page that moves are renamed; the moves are sorted by the page they start from.  Words behind
// the pages of a sequence are no entries and stay as they are, whatever they name.  (Of a length that no table can hold nothing
// follows: all words of that sequence count as entries, so that no page moves away from under one.)
__device__ __forceinline__ void rename_entries(const polyspec_cache_pages& s, const Plan& plan)
{
    const int n_live = plan.starts[0], n_moves = *plan.n_copies;
    const long long n = static_cast<long long>(s.n_seqs) * s.max_pages, step = static_cast<long long>(gridDim.x) * blockDim.x;
    for (long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x; i < n; i += step) {
        const int page = s.table[i];
        if (page < n_live || page >= s.n_pages) continue;
        const int b = static_cast<int>(i / s.max_pages), len = held_len(s, b);
        if (len >= 0 && i - static_cast<long long>(b) * s.max_pages >= pages_for(len, s.page_tokens)) continue;
        int lo = 0, hi = n_moves;               // first move from `page` or later
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (plan.copies[mid].x < page) lo = mid + 1;
            else hi = mid;
        }
        if (lo < n_moves && plan.copies[lo].x == page) s.table[i] = plan.copies[lo].y;
    }
}

struct Pools {
    polyspec_cache_pool pool[kMaxPools];
    int n;
};

// Copies the planned pages in every plane of every pool; a warp takes pieces of 2 KiB, four loads in flight per lane.
__global__ void __launch_bounds__(256) move_kernel(const polyspec_cache_pages s, Plan plan, Pools pools, int rename)
{
    wait_for_stream();
    if (rename) rename_entries(s, plan);
    const int n = *plan.n_copies;
    const int lane = threadIdx.x & 31;
    const long long warps = static_cast<long long>(gridDim.x) * (blockDim.x >> 5);
    const long long warp = static_cast<long long>(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5);
    for (int q = 0; q < pools.n; ++q) {
        const polyspec_cache_pool pool = pools.pool[q];
        const long long pieces = (static_cast<long long>(pool.page_bytes) + kPiece - 1) / kPiece;
        const long long items = static_cast<long long>(n) * pool.n_planes * pieces;
        for (long long it = warp; it < items; it += warps) {
            const long long piece = it % pieces, rest = it / pieces;
            const int plane = static_cast<int>(rest % pool.n_planes);
            const int2 m = plan.copies[rest / pool.n_planes];
            char* at = static_cast<char*>(pool.data) + static_cast<long long>(plane) * s.n_pages * pool.page_bytes + piece * kPiece;
            const long long left = pool.page_bytes - piece * kPiece;
            const uint4* from = reinterpret_cast<const uint4*>(at + m.x * pool.page_bytes);
            uint4* to = reinterpret_cast<uint4*>(at + m.y * pool.page_bytes);
            uint4 x[kPiece / 512];
#pragma unroll
            for (int u = 0; u < kPiece / 512; ++u)
                if ((u * 32 + lane) * 16 < left) x[u] = from[u * 32 + lane];
#pragma unroll
            for (int u = 0; u < kPiece / 512; ++u)
                if ((u * 32 + lane) * 16 < left) to[u * 32 + lane] = x[u];
        }
    }
}

polyspec_status check_pages(const polyspec_cache_pages* s)
{
    if (!s || s->n_seqs < 1 || s->max_pages < 1 || s->n_pages < 1 || s->page_tokens < 1) return POLYSPEC_ERR_INVALID_ARG;
    if (!s->table || !s->len || !s->refs || !s->free_bits || !aligned4(s->table, s->len, s->refs, s->free_bits)) return POLYSPEC_ERR_INVALID_ARG;
    if (static_cast<long long>(s->max_pages) * s->page_tokens > 0x7fffffffLL || s->n_pages > kMaxPages) return POLYSPEC_ERR_UNSUPPORTED;
    return POLYSPEC_OK;
}

polyspec_status check_pools(const polyspec_cache_pool* pools, int n_pools)
{
    if (n_pools < 0 || n_pools > kMaxPools || (n_pools > 0 && !pools)) return POLYSPEC_ERR_INVALID_ARG;
    for (int i = 0; i < n_pools; ++i)
        if (!pools[i].data || (reinterpret_cast<uintptr_t>(pools[i].data) & 15u) != 0 || pools[i].n_planes < 1 || pools[i].page_bytes < 16 ||
            pools[i].page_bytes % 16 != 0)
            return POLYSPEC_ERR_INVALID_ARG;
    return POLYSPEC_OK;
}

polyspec_status check_plan(const polyspec_cache_pages* s, const void* workspace, size_t workspace_bytes)
{
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return POLYSPEC_ERR_INVALID_ARG;
    return workspace_bytes < plan_bytes(s->n_seqs, s->n_pages) ? POLYSPEC_ERR_WORKSPACE : POLYSPEC_OK;
}

cudaError_t launch_move(const polyspec_cache_pages& s, const Plan& plan, const polyspec_cache_pool* pools, int n_pools, bool rename, cudaStream_t stream)
{
    Pools q;
    q.n = n_pools;
    for (int i = 0; i < n_pools; ++i) q.pool[i] = pools[i];
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    return launch_early(move_kernel, dim3(static_cast<unsigned>(sms * 8)), 256, 0, stream, s, plan, q, rename ? 1 : 0);
}

}  // namespace
}  // namespace polyspec

using namespace polyspec;

extern "C" {

polyspec_status polyspec_cache_workspace(int n_seqs, int n_pages, size_t* bytes)
{
    if (!bytes || n_seqs < 1 || n_pages < 1) return POLYSPEC_ERR_INVALID_ARG;
    *bytes = plan_bytes(n_seqs, n_pages);
    return POLYSPEC_OK;
}

polyspec_status polyspec_cache_init(const polyspec_cache_pages* s, void* cuda_stream)
{
    const polyspec_status st = check_pages(s);
    if (st != POLYSPEC_OK) return st;
    cudaStream_t q = static_cast<cudaStream_t>(cuda_stream);
    const size_t whole = s->n_pages / 32 * 4;
    if (cuda_failed(cudaMemsetAsync(s->table, 0xff, static_cast<size_t>(s->n_seqs) * s->max_pages * 4, q))) return POLYSPEC_ERR_CUDA;
    if (cuda_failed(cudaMemsetAsync(s->len, 0, static_cast<size_t>(s->n_seqs) * 4, q))) return POLYSPEC_ERR_CUDA;
    if (cuda_failed(cudaMemsetAsync(s->refs, 0, static_cast<size_t>(s->n_pages) * 4, q))) return POLYSPEC_ERR_CUDA;
    if (whole && cuda_failed(cudaMemsetAsync(s->free_bits, 0xff, whole, q))) return POLYSPEC_ERR_CUDA;
    if (s->n_pages % 32) {
        // the bits of a last, partial word, byte by byte
        unsigned char* last = reinterpret_cast<unsigned char*>(s->free_bits) + whole;
        for (int i = 0, left = s->n_pages % 32; i < 4; ++i, left -= 8) {
            const int bits = left >= 8 ? 0xff : left > 0 ? (1 << left) - 1 : 0;
            if (cuda_failed(cudaMemsetAsync(last + i, bits, 1, q))) return POLYSPEC_ERR_CUDA;
        }
    }
    return POLYSPEC_OK;
}

polyspec_status polyspec_cache_reserve(const polyspec_cache_pages* s, const int32_t* base, const int32_t* extra, int plus,
                                       const polyspec_cache_pool* pools, int n_pools, int32_t* device_status, void* workspace,
                                       size_t workspace_bytes, void* cuda_stream)
{
    polyspec_status st = check_pages(s);
    if (st == POLYSPEC_OK) st = check_pools(pools, n_pools);
    if (st == POLYSPEC_OK) st = base && aligned4(base, extra, device_status) ? check_plan(s, workspace, workspace_bytes) : POLYSPEC_ERR_INVALID_ARG;
    if (st != POLYSPEC_OK) return st;
    const Plan plan = plan_of(workspace, s->n_seqs, s->n_pages);
    cudaStream_t q = static_cast<cudaStream_t>(cuda_stream);
    if (cuda_failed(launch_early(reserve_kernel, dim3(1), kPlanThreads, 0, q, *s, base, extra, plus, plan, device_status))) return POLYSPEC_ERR_CUDA;
    if (n_pools > 0 && cuda_failed(launch_move(*s, plan, pools, n_pools, false, q))) return POLYSPEC_ERR_CUDA;
    return POLYSPEC_OK;
}

polyspec_status polyspec_cache_rollback(const polyspec_cache_pages* s, const int32_t* base, const int32_t* extra, int plus,
                                        int32_t* device_status, void* cuda_stream)
{
    const polyspec_status st = check_pages(s);
    if (st != POLYSPEC_OK) return st;
    if (!base || !aligned4(base, extra, device_status)) return POLYSPEC_ERR_INVALID_ARG;
    const dim3 grid(static_cast<unsigned>((s->n_seqs + 3) / 4));
    return cuda_failed(launch_early(rollback_kernel, grid, 128, 0, static_cast<cudaStream_t>(cuda_stream), *s, base, extra, plus, device_status))
               ? POLYSPEC_ERR_CUDA : POLYSPEC_OK;
}

polyspec_status polyspec_cache_fork(const polyspec_cache_pages* s, const int32_t* src, const int32_t* dst, int n, int32_t* device_status,
                                    void* cuda_stream)
{
    const polyspec_status st = check_pages(s);
    if (st != POLYSPEC_OK) return st;
    if (!src || !dst || n < 1 || !aligned4(src, dst, device_status)) return POLYSPEC_ERR_INVALID_ARG;
    const dim3 grid(static_cast<unsigned>((n + 3) / 4));
    return cuda_failed(launch_early(fork_kernel, grid, 128, 0, static_cast<cudaStream_t>(cuda_stream), *s, src, dst, n, device_status))
               ? POLYSPEC_ERR_CUDA : POLYSPEC_OK;
}

polyspec_status polyspec_cache_compact(const polyspec_cache_pages* s, const polyspec_cache_pool* pools, int n_pools, int32_t* moved_to,
                                       void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    polyspec_status st = check_pages(s);
    if (st == POLYSPEC_OK) st = check_pools(pools, n_pools);
    if (st == POLYSPEC_OK) st = aligned4(moved_to) ? check_plan(s, workspace, workspace_bytes) : POLYSPEC_ERR_INVALID_ARG;
    if (st != POLYSPEC_OK) return st;
    const Plan plan = plan_of(workspace, s->n_seqs, s->n_pages);
    cudaStream_t q = static_cast<cudaStream_t>(cuda_stream);
    if (cuda_failed(launch_early(compact_kernel, dim3(1), kPlanThreads, 0, q, *s, plan, moved_to))) return POLYSPEC_ERR_CUDA;
    if (cuda_failed(launch_move(*s, plan, pools, n_pools, true, q))) return POLYSPEC_ERR_CUDA;
    return POLYSPEC_OK;
}

}  // extern "C"
