// Attention over 4-bit pages for more than eight rows per sequence and key head, on the fifth-generation tensor cores (formulas and the form of
// the codes: cache_attention.cu; head_dim 128).
//
// Tokens are the rows of the first product, elements those of the second, the block's rows (up to 48) their columns:
//   S^T [128 tokens x rows] = codes of keys (tensor memory, expanded by a warpgroup, a thread per token) x Q^T (shared memory)
//   O^T [128 elements x rows] += codes of values (shared memory, expanded by a second warpgroup) x P'^T (shared memory)
// so a tile of 128 is full whatever the number of rows, a softmax thread has one token's scales in registers, and its
// weights of all rows are neighbours in shared memory.  Compared with mma.sync, whose tiles repeat the expansion for every 16 rows and whose
// products are a third of all instructions: 36 rows take 2.7 times fewer instructions per token.
//
// Persistent, one CTA per SM, an equal share of all segments' steps of 128 tokens each (cache_attention.cuh).  Roles (20 warps):
//   0      MMA issuer; allocates and frees tensor memory
//   1      finds the CTA's parts of segments and prepares their rows, a part ahead of the others
//   4-7    keys: codes from memory three steps ahead, as fp16 subnormals into tensor memory
//   8-11   values: the same into shared memory
//   12-19  softmax, a thread per token and every other group of 8 rows; at the end of a part the output, a thread per element
// What bounds it is shared memory: per step 32 KB of values written and read, queries and weights, some 900 cycles of its 128 bytes per cycle.
#include <cuda.h>

#include "cache_attention.cuh"
#include "tensor_device.cuh"

namespace polyspec {
namespace {

using namespace attend;
using namespace tensordev;

struct Wide {
    static constexpr int D = 128, ROWS = kWideRows, STEP = 128, WARPS = 20, THREADS = 640, UB = kv::unit_bytes(D);
    static constexpr int OVERHEAD = 4;          // steps' worth of work that a segment costs besides its steps
    static constexpr int PART = ROWS * (D + 2);
    static constexpr uint32_t QBOX = ROWS * 128, QTILE = 2 * QBOX, VBOX = 128 * 128, VTILE = 2 * VBOX, PTILE = 128 * 128;
    static constexpr size_t SMEM = 1024 + 2 * (QTILE + VTILE + PTILE);
    // tensor memory: two blocks of keys, two of scores, the output
    static constexpr uint32_t KCOLS = 64, S0 = 128, SCOLS = 64, O0 = 256, COLS = 512;
};

// A part of a segment: `steps` steps from step0 on.
struct Part { int steps, step0, b, head, row0, live, seen, all_see, slot, starts, ends; };

struct Bars {
    static constexpr int kKFull = 0, kKFree = 2, kVFull = 4, kVFree = 6, kSFull = 8, kSFree = 10, kPFull = 12, kPFree = 14, kOFull = 16, kPartFull = 17, kPartFree = 19,
                         kCount = 21;
};

__device__ __forceinline__ void umma_k(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 db, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
        ::"r"(d), "r"(a), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi) : "memory");
}
__device__ __forceinline__ void umma_v(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
        ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi) : "memory");
}
__device__ __forceinline__ void umma_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
                   "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_ld8(uint32_t addr, float* r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t addr, const float* r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"r"(addr), "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]) : "memory");
}
__device__ __forceinline__ void st_shared16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// The softmax warps meet, and learn whether any of their threads says so.
__device__ __forceinline__ bool meet_any(bool x)
{
    uint32_t y;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(y) : "r"(static_cast<uint32_t>(x)) : "memory");
    return y != 0;
}

__device__ __forceinline__ void raise_abort(int* abort_flag, int32_t* status)
{
    if (!*reinterpret_cast<volatile int*>(abort_flag) && status) atomicCAS(status, 0, static_cast<int>(POLYSPEC_ERR_TIMEOUT));
    *reinterpret_cast<volatile int*>(abort_flag) = 1;
}

// A bounded wait that the whole warp passes or the whole warp gives up.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag)
{
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
}

// Numbers of units in a plane, for tokens of one part: the table's word is loaded a step before it is used.
struct Units {
    const int32_t* table;
    uint32_t head_unit, page_units;             // of the page's units the head's first; units of a page over all heads
    int per_page, n_pages, seen;
    __device__ __forceinline__ void start(const AttendParams& p, const Part& part)
    {
        table = p.s.table + static_cast<size_t>(part.b) * p.s.max_pages;
        per_page = p.units_per_page;
        n_pages = p.s.n_pages;
        head_unit = static_cast<uint32_t>(part.head) * per_page;
        page_units = static_cast<uint32_t>(p.kv_heads) * per_page;
        seen = part.seen;
    }
    // (page, unit of the page) of the unit that holds `slot`; unit -1 behind what is seen.  The page is not looked at here: its load is on its way.
    __device__ __forceinline__ int2 look(long long slot) const
    {
        if (slot >= seen) return make_int2(0, -1);
        const int unit = static_cast<int>(slot >> 3), at = unit / per_page;
        return make_int2(table[at], unit - at * per_page);
    }
    __device__ __forceinline__ bool broken(int2 x) const { return x.y >= 0 && (x.x < 0 || x.x >= n_pages); }
    __device__ __forceinline__ uint32_t number(int2 x) const
    {
        return x.y < 0 || x.x < 0 || x.x >= n_pages ? 0xffffffffu : static_cast<uint32_t>(x.x) * page_units + head_unit + x.y;
    }
};

__global__ void __launch_bounds__(Wide::THREADS, 1) attend_wide_kernel(const AttendParams p)
{
    using S = Wide;
    extern __shared__ unsigned char smem_wide[];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag, hit;
    __shared__ long long warp_sums[S::WARPS], hit_at;
    __shared__ Part parts[2];
    __shared__ __align__(16) float sums[2][S::ROWS], refs[S::ROWS];            // read four at a time
    __shared__ float factors[2], tops[4][S::ROWS], parts_l[4][S::ROWS], parts_o[4][S::ROWS];
    __shared__ int limits[2][S::ROWS];
    __shared__ long long places[2][S::ROWS];    // of the rows, in [rows, q_heads]
    __shared__ __align__(8) uint64_t barriers[Bars::kCount];
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t q_tiles = (smem_addr(smem_wide) + 1023u) & ~1023u, v_tiles = q_tiles + 2 * S::QTILE, p_tiles = v_tiles + 2 * S::VTILE;
    const uint32_t bars = smem_addr(barriers);
    auto bar = [&](int n) { return bars + 8u * n; };

    if (threadIdx.x == 0) {
        abort_flag = 0;
        // who arrives: the warps of a role, or the issuer's commit; on a free slot of parts everyone that reads it
        for (int i = 0; i < Bars::kCount; ++i) {
            const bool four = i < 2 || (i >= Bars::kVFull && i < Bars::kVFree), eight = i >= Bars::kSFree && i < Bars::kPFree;
            mbar_init(bar(i), i >= Bars::kPartFree ? 17 : eight ? 8 : four ? 4 : 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        proxy_fence();
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_slot)), "r"(S::COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    volatile int* abort_p = &abort_flag;
    bool ok = true;
    wait_for_stream();

    // this CTA's share of all places, as in attend_kernel
    int seq;
    long long within;
    const long long total = locate<S>(p, -1, &seq, &within, warp_sums, &hit, &hit_at);
    const long long ctas = min(total, static_cast<long long>(gridDim.x));
    if (threadIdx.x == 0) p.joins[blockIdx.x] = make_int4(0, 0, 0, 0);
    const bool works = blockIdx.x < ctas;
    long long s0 = 0, s1 = 0;
    if (works) {
        s0 = total * blockIdx.x / ctas;
        s1 = total * (blockIdx.x + 1) / ctas;
        locate<S>(p, s0, &seq, &within, warp_sums, &hit, &hit_at);
    }

    // The next part for everyone who reads them.  n: steps before it.
    uint32_t taken = 0;
    auto take = [&](Part* part) {
        if (!works || !warp_wait(bar(Bars::kPartFull + (taken & 1)), taken >> 1 & 1, abort_p)) return false;
        *part = parts[taken & 1];
        return true;
    };
    auto give_back = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive_local(bar(Bars::kPartFree + (taken & 1)));
        ++taken;
    };
    uint32_t n = 0;                             // steps so far: buffer n & 1, its use n >> 1
    Part part;

    // 640 threads were launched with 96 registers each, 61440 in all: 128 * 56 + 256 * 88 + 256 * 120 = 60416
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == 0) {
            // ------------------------------------------------------------------ MMA issuer
            while (ok) {
                if (!take(&part)) { ok = false; break; }
                if (part.steps == 0) break;
                const uint32_t cols = static_cast<uint32_t>(part.live + 15) / 16 * 16;
                // D fp32, A and B fp16, M = 128; the second product's operands with tokens as their slow axis
                const uint32_t idesc = (1u << 4) | (cols >> 3 << 17) | (128u >> 4 << 24), idesc_o = idesc | (1u << 15) | (1u << 16);
                const uint32_t q = q_tiles + part.slot * S::QTILE;
                auto scores = [&](uint32_t k) {
                    const uint32_t at = k & 1, use = k >> 1 & 1;
                    ok = ok && warp_wait(bar(Bars::kKFull + at), use, abort_p) && warp_wait(bar(Bars::kSFree + at), use ^ 1, abort_p);
                    if (!ok) return;
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            umma_k(tmem + S::S0 + at * S::SCOLS, tmem + at * S::KCOLS + i * 8, smem_desc_lo(q) + (i >> 2) * (S::QBOX >> 4) + (i & 3) * 2, idesc, i != 0);
                        umma_commit(bar(Bars::kKFree + at));
                        umma_commit(bar(Bars::kSFull + at));
                    }
                    __syncwarp();
                };
                scores(n);
                for (int j = 0; j < part.steps && ok; ++j, ++n) {
                    if (j + 1 < part.steps) scores(n + 1);
                    const uint32_t at = n & 1, use = n >> 1 & 1;
                    ok = ok && warp_wait(bar(Bars::kVFull + at), use, abort_p) && warp_wait(bar(Bars::kPFull + at), use, abort_p);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t v = v_tiles + at * S::VTILE, w = p_tiles + at * S::PTILE;
                        const uint32_t a = ((v & 0x3ffffu) >> 4) | (S::VBOX >> 4 << 16), b = ((w & 0x3ffffu) >> 4) | (1u << 16);
#pragma unroll
                        for (int i = 0; i < 8; ++i) umma_v(tmem + S::O0, a + i * (2048 >> 4), b + i * (2048 >> 4), idesc_o, j != 0 || i != 0);
                        umma_commit(bar(Bars::kVFree + at));
                        umma_commit(bar(Bars::kPFree + at));
                        if (j + 1 == part.steps) {
                            umma_commit(bar(Bars::kOFull));
                            umma_commit(bar(Bars::kPartFree + part.slot));         // the rows have been read
                        }
                    }
                    __syncwarp();
                }
                ++taken;
            }
            if (!ok && works && lane == 0) raise_abort(&abort_flag, p.status);
        } else if (warp == 1 && works) {
            // ------------------------------------------------------------------ parts and their rows
            Segment g;
            g.b = seq;
            g.q = kv::seq_rows(p.s, p.r, seq);
            seq_segments<S::ROWS, S::STEP>(p, g);
            const int span = g.steps + S::OVERHEAD, nth = static_cast<int>(within / span), into = static_cast<int>(within % span) - S::OVERHEAD;
            g.head = nth / g.tiles;
            g.tile = nth % g.tiles;
            int step = max(into, 0), left = static_cast<int>(s1 - s0) + min(into, 0);
            for (uint32_t k = 0; ok; ++k) {
                const int slot = k & 1;
                if (!warp_wait(bar(Bars::kPartFree + slot), (k >> 1 & 1) ^ 1, abort_p)) { ok = false; break; }
                const int steps = left > 0 ? min(left, g.steps - step) : 0;
                if (steps) {
                    const int row0 = g.tile * g.tile_rows, end = min(g.q.n * p.group, row0 + g.tile_rows), live = end - row0;
                    left -= steps;
                    // rows: the largest element first, then as fp16 in the codes' order, zeros behind the last
                    const int vec = lane & 15, odd = lane >> 4;
                    float top = 0.0f;
                    auto load = [&](int r) {
                        const int row = row0 + r, i = row / p.group;
                        return r < live ? *reinterpret_cast<const uint4*>(p.q + (g.q.row0 + i) * p.q_stride + (g.head * p.group + row % p.group) * S::D + vec * 8)
                                        : make_uint4(0, 0, 0, 0);
                    };
#pragma unroll 1
                    for (int r0 = 0; r0 < live; r0 += 8) {
                        uint4 x[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) x[u] = load(r0 + 2 * u + odd);
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const uint32_t* y = reinterpret_cast<const uint32_t*>(&x[u]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float a = fabsf(low(y[e])), b = fabsf(high(y[e]));
                                if (a <= 3.4e38f) top = fmaxf(top, a);
                                if (b <= 3.4e38f) top = fmaxf(top, b);
                            }
                        }
                    }
#pragma unroll
                    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                    float factor;
                    const float by = row_scale(p, top, &factor), by16 = by * 0.0625f;
                    const uint32_t to = q_tiles + slot * S::QTILE + (vec >> 3) * S::QBOX;
#pragma unroll 1
                    for (int r0 = 0; r0 < S::ROWS; r0 += 8) {
                        if (r0 >= (live + 15) / 16 * 16) break;
                        uint4 x[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) x[u] = load(r0 + 2 * u + odd);
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const int r = r0 + 2 * u + odd;
                            const uint32_t* y = reinterpret_cast<const uint32_t*>(&x[u]);
                            float sum = 0.0f;
#pragma unroll
                            for (int e = 0; e < 4; ++e) sum += low(y[e]) + high(y[e]);
                            st_shared16(to + r * 128 + (((vec & 7) ^ (r & 7)) << 4), half2_bits(low(y[0]) * by, high(y[0]) * by),
                                        half2_bits(low(y[1]) * by16, high(y[1]) * by16), half2_bits(low(y[2]) * by, high(y[2]) * by),
                                        half2_bits(low(y[3]) * by16, high(y[3]) * by16));
#pragma unroll
                            for (int d = 1; d < 16; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                            if (vec == 0) {
                                const int row = row0 + r, i = row / p.group;
                                sums[slot][r] = sum * p.scale_log2;         // (0 behind the last row)
                                limits[slot][r] = r < live ? row_limit(g.q, i) : 0;
                                places[slot][r] = static_cast<long long>(g.q.row0 + i) * p.q_heads + g.head * p.group + row % p.group;
                            }
                        }
                    }
                    proxy_fence();
                    if (lane == 0) {
                        factors[slot] = factor;
                        Part x;
                        x.steps = steps; x.step0 = step; x.b = g.b; x.head = g.head; x.row0 = row0; x.live = live;
                        x.seen = visible(p, g); x.all_see = g.q.base + 1; x.slot = slot;
                        x.starts = step == 0; x.ends = step + steps == g.steps;
                        parts[slot] = x;
                        if (x.starts && !x.ends) {      // the CTAs that the rest of the segment falls to
                            const long long last = s1 + (g.steps - step - steps) - 1;
                            const int at = static_cast<int>(((last + 1) * ctas - 1) / total);
                            p.joins[blockIdx.x] = make_int4(at - static_cast<int>(blockIdx.x) + 1, g.b << 6 | g.tile_rows / 8, g.head, row0);
                        }
                    }
                    step += steps;
                    if (step == g.steps) {
                        next_segment<S>(p, g);
                        step = 0;
                        left -= S::OVERHEAD;
                    }
                } else if (lane == 0) {
                    parts[slot].steps = 0;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive_local(bar(Bars::kPartFull + slot));
                if (steps == 0) break;
            }
            if (!ok && lane == 0) raise_abort(&abort_flag, p.status);
        }
    } else if (warp < 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        const int quarter = warp & 3;
        constexpr int kAhead = 3;               // steps whose codes are on their way
        if (warp < 8) {
            // ------------------------------------------------------------------ keys, a thread per token
            const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
            while (ok) {
                if (!take(&part)) { ok = false; break; }
                if (part.steps == 0) break;
                Units units;
                units.start(p, part);
                const int token = quarter * 32 + lane;
                uint4 x[kAhead][4];
                int2 next = make_int2(0, -1);
                auto look = [&](int j) { return j < part.steps ? units.look(static_cast<long long>(part.step0 + j) * 128 + token) : make_int2(0, -1); };
                auto load = [&](uint4* to, int j) {
                    const uint32_t number = units.number(next);
                    next = look(j + 1);
                    const uint4* from = reinterpret_cast<const uint4*>(p.pool + static_cast<size_t>(number) * S::UB) + (token & 7) * 4;
#pragma unroll
                    for (int i = 0; i < 4; ++i) to[i] = number == 0xffffffffu ? make_uint4(0, 0, 0, 0) : from[i];
                };
                next = look(0);
#pragma unroll
                for (int u = 0; u < kAhead; ++u) load(x[u], u);
                for (int j0 = 0; j0 < part.steps && ok; j0 += kAhead) {
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        if (j0 + u >= part.steps) break;
                        const uint32_t at = n & 1, use = n >> 1 & 1;
                        if (!warp_wait(bar(Bars::kKFree + at), use ^ 1, abort_p)) { ok = false; break; }
                        tc_fence_after();
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint4 v = x[u][i];
                            const uint32_t words[4] = {v.x, v.y, v.z, v.w};
                            uint32_t y[16];
#pragma unroll
                            for (int w = 0; w < 16; ++w) y[w] = code_pair(words[w >> 2], w & 3);
                            tmem_st16(tmem + at * S::KCOLS + lanes + i * 16, y);
                        }
                        load(x[u], j0 + u + kAhead);
                        tmem_st_wait();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_local(bar(Bars::kKFull + at));
                        ++n;
                    }
                }
                if (ok) give_back();
            }
        } else {
            // ------------------------------------------------------------------ values: a warp has four units, a lane one token and two groups of words of each
            const int r = lane & 7, g = lane >> 3;
            while (ok) {
                if (!take(&part)) { ok = false; break; }
                if (part.steps == 0) break;
                Units units;
                units.start(p, part);
                uint2 x[kAhead][8];
                int2 next = make_int2(0, -1);   // of the unit that lane & 3 stands for
                auto look = [&](int j) { return j < part.steps ? units.look(static_cast<long long>(part.step0 + j) * 128 + quarter * 32 + (lane & 3) * 8) : make_int2(0, -1); };
                auto load = [&](uint2* to, int j) {
                    const uint32_t mine = units.number(next);
                    next = look(j + 1);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t number = __shfl_sync(0xffffffffu, mine, i);
                        const uint2* from = reinterpret_cast<const uint2*>(p.pool + p.plane_bytes + static_cast<size_t>(number) * S::UB);
#pragma unroll
                        for (int k = 0; k < 2; ++k) to[2 * i + k] = number == 0xffffffffu ? make_uint2(0, 0) : from[8 * (g + 4 * k) + r];
                    }
                };
                next = look(0);
#pragma unroll
                for (int u = 0; u < kAhead; ++u) load(x[u], u);
                for (int j0 = 0; j0 < part.steps && ok; j0 += kAhead) {
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        if (j0 + u >= part.steps) break;
                        const uint32_t at = n & 1, use = n >> 1 & 1;
                        if (!warp_wait(bar(Bars::kVFree + at), use ^ 1, abort_p)) { ok = false; break; }
                        const uint32_t to = v_tiles + at * S::VTILE + (quarter * 32 + r) * 128;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const uint2 w = x[u][2 * i + k];
                                const uint32_t chunk = to + i * 1024 + (((g + 4 * k) ^ r) << 4);
                                st_shared16(chunk, code_pair(w.x, 0), code_pair(w.x, 1), code_pair(w.x, 2), code_pair(w.x, 3));
                                st_shared16(chunk + S::VBOX, code_pair(w.y, 0), code_pair(w.y, 1), code_pair(w.y, 2), code_pair(w.y, 3));
                            }
                        load(x[u], j0 + u + kAhead);
                        proxy_fence();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_local(bar(Bars::kVFull + at));
                        ++n;
                    }
                }
                if (ok) give_back();
            }
        }
        if (!ok && works && lane == 0) raise_abort(&abort_flag, p.status);
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 120;");
        // ------------------------------------------------------------------ softmax, a thread per token and every other group of 8 rows
        const int quarter = warp & 3, turn = (warp - 12) >> 2, token = quarter * 32 + lane;
        const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
        constexpr int C = S::ROWS / 16;         // groups of rows: 2 c + turn
        uint32_t o_phase = 0;
        while (ok) {
            ok = take(&part);
            if (meet_any(!ok)) { ok = false; break; }
            if (part.steps == 0) break;
            const int slot = part.slot, groups = (part.live + 7) / 8;
            const float factor = factors[slot];
            Units units;
            units.start(p, part);
            // the token's scales and offsets, two steps ahead, and its page one more
            int2 next = make_int2(0, -1);
            uint32_t pair_k[2], pair_v[2];
            bool there[2];
            auto look = [&](int j) { return j < part.steps ? units.look(static_cast<long long>(part.step0 + j) * 128 + token) : make_int2(0, -1); };
            auto load = [&](int i, int j) {
                const uint32_t number = units.number(next);
                if (__builtin_expect(units.broken(next), 0)) kv::report(p.status, POLYSPEC_ERR_BAD_INPUT_ON_DEVICE);
                there[i] = number != 0xffffffffu;
                next = look(j + 1);
                const unsigned char* from = p.pool + static_cast<size_t>(number) * S::UB + 4 * S::D + (token & 7) * 4;
                pair_k[i] = there[i] ? *reinterpret_cast<const uint32_t*>(from) : 0;
                pair_v[i] = there[i] ? *reinterpret_cast<const uint32_t*>(from + p.plane_bytes) : 0x3f80u;           // (a scale of 1)
            };
            next = look(0);
            load(0, 0);
            load(1, 1);
            float l[C][8], lo[C][8];
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) l[c][e] = lo[c][e] = 0.0f;
            if (turn == 0 && token < S::ROWS) refs[token] = 0.0f;
            bool started = false;
            meet_any(false);
            for (int j = 0; j < part.steps; ++j, ++n) {
                const uint32_t at = n & 1, use = n >> 1 & 1;
                const float ks = low(pair_k[0]) * factor, ko = high(pair_k[0]), vs = low(pair_v[0]), lv = lg2(vs), iv = rcp(vs), ov = high(pair_v[0]) * iv;
                // the first rows' limits are the lowest: what is above them is masked, row by row
                const int token_slot = there[0] ? (part.step0 + j) * 128 + token : 0x7fffffff;
                const bool masked = __any_sync(0xffffffffu, token_slot >= part.all_see);
                pair_k[0] = pair_k[1]; pair_v[0] = pair_v[1]; there[0] = there[1];
                load(1, j + 2);
                ok = ok && warp_wait(bar(Bars::kSFull + at), use, abort_p);
                tc_fence_after();
                float x[C][8], most = -INFINITY;
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if (2 * c + turn < groups) tmem_ld8(tmem + S::S0 + at * S::SCOLS + lanes + (2 * c + turn) * 8, x[c]);
                tmem_ld_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_local(bar(Bars::kSFree + at));
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if (2 * c + turn < groups) {
                        const int r0 = (2 * c + turn) * 8;
                        float4 sum[2], ref[2];
                        sum[0] = *reinterpret_cast<const float4*>(&sums[slot][r0]); sum[1] = *reinterpret_cast<const float4*>(&sums[slot][r0 + 4]);
                        ref[0] = *reinterpret_cast<const float4*>(&refs[r0]); ref[1] = *reinterpret_cast<const float4*>(&refs[r0 + 4]);
                        const float* sq = &sum[0].x;
                        const float* rf = &ref[0].x;
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[c][e] = fmaf(x[c][e], ks, fmaf(sq[e], ko, lv) - rf[e]);
                        if (__builtin_expect(masked, 0)) {
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (token_slot >= limits[slot][r0 + e]) x[c][e] = -INFINITY;
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) most = fmaxf(most, x[c][e]);
                    }
                // the first tokens set the references; after that sums are rescaled only when a maximum has risen by 2^kSlack
                if (__builtin_expect(meet_any(!ok || !started || most > kLift + kSlack), 0)) {
                    if (meet_any(!ok)) { ok = false; break; }
#pragma unroll
                    for (int c = 0; c < C; ++c)
                        if (2 * c + turn < groups) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                float top = x[c][e];
#pragma unroll
                                for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                                if (lane == 0) tops[quarter][(2 * c + turn) * 8 + e] = top;
                            }
                        }
                    meet_any(false);
                    // the output of the steps before: finished, then rescaled by the threads that stand for its elements
                    if (j > 0) ok = ok && warp_wait(bar(Bars::kPFree + (at ^ 1)), (n - 1) >> 1 & 1, abort_p);
                    tc_fence_after();
                    bool some = false;
                    for (int r = 0; r < part.live; ++r) some = some || fmaxf(fmaxf(tops[0][r], tops[1][r]), fmaxf(tops[2][r], tops[3][r])) > -INFINITY;
#pragma unroll
                    for (int c = 0; c < C; ++c)
                        if (2 * c + turn < groups) {
                            float o[8];
                            if (j > 0) {
                                tmem_ld8(tmem + S::O0 + lanes + (2 * c + turn) * 8, o);
                                tmem_ld_wait();
                            }
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const int r = (2 * c + turn) * 8 + e;
                                const float top = fmaxf(fmaxf(tops[0][r], tops[1][r]), fmaxf(tops[2][r], tops[3][r]));
                                // (a row that sees none of the first tokens sees none of the later ones either)
                                const float up = !started ? (top == -INFINITY ? 0.0f : top - kLift) : fmaxf(top - kLift, 0.0f), by = started ? ex2(-up) : 1.0f;
                                x[c][e] -= up;
                                l[c][e] *= by;
                                lo[c][e] *= by;
                                o[e] *= by;
                            }
                            if (j > 0) tmem_st8(tmem + S::O0 + lanes + (2 * c + turn) * 8, o);
                        }
                    tmem_st_wait();
                    tc_fence_before();
                    meet_any(false);            // everyone has read the references
                    if (turn == 0 && token < part.live) {
                        const float top = fmaxf(fmaxf(tops[0][token], tops[1][token]), fmaxf(tops[2][token], tops[3][token]));
                        refs[token] += !started ? (top == -INFINITY ? 0.0f : top - kLift) : fmaxf(top - kLift, 0.0f);
                    }
                    meet_any(false);
                    started = started || some;
                }
                ok = ok && warp_wait(bar(Bars::kPFree + at), use ^ 1, abort_p);
                const uint32_t to = p_tiles + at * S::PTILE + token * 128;
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if (2 * c + turn < groups) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[c][e] = ex2(x[c][e]);
                        st_shared16(to + (((2 * c + turn) ^ (token & 7)) << 4), half2_bits(x[c][0], x[c][1]), half2_bits(x[c][2], x[c][3]),
                                    half2_bits(x[c][4], x[c][5]), half2_bits(x[c][6], x[c][7]));
                        if (__builtin_expect(!masked, 1)) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                l[c][e] = fmaf(x[c][e], iv, l[c][e]);
                                lo[c][e] = fmaf(x[c][e], ov, lo[c][e]);
                            }
                        } else {                // scales behind what a row sees may be anything
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (token_slot < limits[slot][(2 * c + turn) * 8 + e]) {
                                    l[c][e] = fmaf(x[c][e], iv, l[c][e]);
                                    lo[c][e] = fmaf(x[c][e], ov, lo[c][e]);
                                }
                        }
                    }
                proxy_fence();
                __syncwarp();
                if (lane == 0) mbar_arrive_local(bar(Bars::kPFull + at));
            }
            if (ok) ok = warp_wait(bar(Bars::kOFull), o_phase, abort_p);
            o_phase ^= 1u;
            if (meet_any(!ok)) { ok = false; break; }
            tc_fence_after();
            // sums over the tokens
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (2 * c + turn < groups) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
#pragma unroll
                        for (int d = 16; d; d >>= 1) {
                            l[c][e] += __shfl_xor_sync(0xffffffffu, l[c][e], d);
                            lo[c][e] += __shfl_xor_sync(0xffffffffu, lo[c][e], d);
                        }
                        if (lane == 0) { parts_l[quarter][(2 * c + turn) * 8 + e] = l[c][e]; parts_o[quarter][(2 * c + turn) * 8 + e] = lo[c][e]; }
                    }
                }
            meet_any(false);
            const bool whole = part.starts && part.ends;
            const float by = token & 2 ? 1048576.0f : 16777216.0f;      // 2^20, 2^24: what the codes' form left out
            float* partial = p.partial + static_cast<size_t>(2 * blockIdx.x + (part.starts ? 1 : 0)) * S::PART;
#pragma unroll 1
            for (int c = turn; c < groups; c += 2) {
                float o[8];
                tmem_ld8(tmem + S::O0 + lanes + c * 8, o);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int r = c * 8 + e;
                    if (r >= part.live) continue;
                    const float lt = (parts_l[0][r] + parts_l[1][r]) + (parts_l[2][r] + parts_l[3][r]);
                    const float ot = (parts_o[0][r] + parts_o[1][r]) + (parts_o[2][r] + parts_o[3][r]);
                    const float y = fmaf(o[e], by, ot);
                    if (whole) {
                        const bool none = limits[slot][r] == 0;
                        p.out[places[slot][r] * S::D + token] = none ? 0 : static_cast<unsigned short>(bf16x2_bits(y / lt, 0.0f) & 0xffffu);
                        if (p.lse && token == 0) p.lse[places[slot][r]] = none ? -INFINITY : (refs[r] + log2f(lt)) * 0.69314718055994530942f;
                    } else {
                        partial[r * S::D + token] = y;
                        if (token == 0) {
                            partial[S::ROWS * S::D + 2 * r] = lt == 0.0f ? kNone : refs[r];
                            partial[S::ROWS * S::D + 2 * r + 1] = lt;
                        }
                    }
                }
            }
            tc_fence_before();
            meet_any(false);                    // the references have been read
            give_back();
        }
        if (!ok && works && lane == 0) raise_abort(&abort_flag, p.status);
    }

    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) {
        if (*abort_p) __nanosleep(1000000);             // giving up: MMAs in flight get a bounded moment
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::COLS) : "memory");
    }
}

}  // namespace

cudaError_t attend::launch_attend_wide(const AttendParams& p, cudaStream_t stream)
{
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(attend_wide_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(Wide::SMEM));
    if (e != cudaSuccess) return e;
    const int ctas = sms < kMaxCtas ? sms : kMaxCtas;
    e = launch_early(attend_wide_kernel, dim3(static_cast<unsigned>(ctas)), Wide::THREADS, Wide::SMEM, stream, p);
    if (e == cudaSuccess) e = launch_early(join_kernel<Wide>, dim3(static_cast<unsigned>(ctas)), 256, 0, stream, p);
    return e;
}

}  // namespace polyspec
