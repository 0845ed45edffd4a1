// Causal attention over whole prompts, packed one behind the other, on the fifth-generation tensor cores.
//
//   out[i] = sum_{j <= i} softmax_j(scale * q[i] . k[j]) v[j]
//
// One pass over the keys with a running maximum and sum per row.  A work item is a pair of tiles of 128 query rows, A and B, that read the same
// keys: two heads of one group, or, in groups of odd size, two neighbouring tiles of one head.  Per 128 keys the tensor core makes S = Q K^T
// (fp32, tensor memory), a warpgroup turns its rows of S into weights P (bf16, over S in tensor memory), and the tensor core adds P V to the
// output (fp32, tensor memory, 128 columns).  While one tile's rows are with the softmax, the tensor core has the other's.
//
// Persistent, one CTA per SM; items by falling number of keys, so that the last ones are the shortest.  Roles (12 warps):
//   0     TMA producer: query tiles, then key and value tiles through one ring (boxes of 64 elements x 128 rows, 128-byte swizzle)
//   1     MMA issuer; allocates and frees tensor memory
//   2     scheduler: finds the next items in the row numbers, ahead of the others
//   3     watches values: where some row of the item does not see some key, P is 0, and 0 * NaN would be NaN.  Values that
//         are not finite are replaced by 0 there; if there were any, the epilogue adds them to the rows that see them
//   4-7   softmax and epilogue of tile A, a thread per row;  8-11 the same for tile B
// A row's maximum is only followed when it has risen by 2^8: sums and output are then rescaled, by the row's own threads.
//
// Measured (B200): prompts of 8192, 2500, 1111 and 389 rows, 32 heads of 128 over 8: 507 us, 1208 TFLOP/s, 0.74 of a library product's burst (575 us where a
// long run is held at the power cap).  Bound by the softmax and the products taking turns: tensor and exponential pipes are each active 60% of the time.  Half
// or a quarter of the exponentials as polynomials on the FMA pipe moved nothing or cost time; without the split of registers between roles scores spill
// (3300 us); weights handed over in halves and items to and fro over the CTAs were worth 577 -> 524, what is loaded from tensor memory pinned behind its wait
// 524 -> 507.  Prompts of a few hundred rows: 11 us, a launch and the longest item's steps one after the other (three for
// 384 rows of groups of odd size, without a tile B, so with half of the softmax warps idle).
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <mutex>

#include "kv_pages.cuh"
#include "number_pairs.cuh"
#include "tensor_device.cuh"

namespace polyspec {
namespace {

using namespace numbers;

using namespace tensordev;

constexpr int kTileRows = 128;                      // rows of a query tile, keys of a step
constexpr int kThreads = 384;
constexpr int kSlots = 2;                       // items known ahead
constexpr uint32_t kTmem = 512;
constexpr float kSlack = 8.0f;                  // how far (log2) a row's weights may exceed 1 before they are rescaled

struct PromptParams {
    CUtensorMap map_q, map_k, map_v;            // [rows, heads, D], boxes {64, 1, 128}
    const int32_t* rows_at;
    const unsigned short* v;
    long long v_stride;
    int n_seqs, rows, q_heads, group;
    int pairs;                                  // items per tile of rows: pairs of heads, or heads
    int tile_rows;                              // rows of an item: 128, or 256 where its tiles follow one another
    float scale_log2;
    unsigned short* out;
    float* lse;
    int32_t* status;
};

// An item: tile A and B's first rows (in the whole tensor) and heads, the steps of each (0: no such tile).
struct Item { int begin, end, row_a, row_b, head_a, head_b, steps_a, steps_b, dirty; };

template <int D_>
struct Shape {
    static constexpr int D = D_;
    static constexpr uint32_t BOX = kTileRows * 128, TILE = D / 64 * BOX;
    static constexpr int STAGES = D == 128 ? 4 : 8;
    static constexpr size_t SMEM = 1024 + 2 * TILE + static_cast<size_t>(STAGES) * TILE;
    // D fp32, A and B bf16; B of the second product with its rows (head elements) contiguous
    static constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | (kTileRows >> 4 << 24);
    static constexpr uint32_t IDESC_S = IDESC | (kTileRows >> 3 << 17), IDESC_O = IDESC | (1u << 16) | (D >> 3 << 17);
};

__device__ __forceinline__ void tma_load3(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void umma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
        ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi) : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 db, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
        ::"r"(d), "r"(a), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi) : "memory");
}
__device__ __forceinline__ void umma_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float* r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]), "=f"(r[10]),
          "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]),
          "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]),
          "=f"(r[31]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t* r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
        ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
          "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
          "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
// Waits for loads from tensor memory; what they filled is not used before.
template <int N>
__device__ __forceinline__ void tmem_ld_wait(float (&r)[N])
{
    tensordev::tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+f"(r[i]));
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void raise_abort(int* abort_flag, int32_t* status)
{
    if (!*reinterpret_cast<volatile int*>(abort_flag) && status) atomicCAS(status, 0, static_cast<int>(POLYSPEC_ERR_TIMEOUT));
    *reinterpret_cast<volatile int*>(abort_flag) = 1;
}

// A bounded wait that the whole warp passes or the whole warp gives up; long ones sleep between polls.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag)
{
    bool ok = false;
    for (uint32_t i = 0; i < kSpinLimitG; ++i) {
        if (mbar_try(bar, parity)) { ok = true; break; }
        if ((i & 63u) == 63u) {
            if (*abort_flag) break;
            if (i >= 4096u) __nanosleep(i >= 65536u ? 4000 : 500);
        }
    }
    return __all_sync(0xffffffffu, ok);
}

struct Ring {
    uint32_t at = 0, phase = 0;
    __device__ __forceinline__ void next(uint32_t n)
    {
        if (++at == n) { at = 0; phase ^= 1u; }
    }
};

// Barriers, by number.
template <class S>
struct Bars {
    static constexpr int kFull = 0, kEmpty = kFull + S::STAGES, kClean = kEmpty + S::STAGES, kQFull = kClean + S::STAGES, kQEmpty = kQFull + 2,
                         kSFull = kQEmpty + 1, kPReady = kSFull + 2, kPHalf = kPReady + 2, kOFull = kPHalf + 2, kItemFull = kOFull + 2, kItemEmpty = kItemFull + kSlots,
                         kCount = kItemEmpty + kSlots;
};

// A prompt's rows, or none where the numbers make no sense.
__device__ __forceinline__ int2 prompt_rows(const PromptParams& p, int b, bool* bad)
{
    const int lo = p.rows_at[b], hi = p.rows_at[b + 1];
    *bad = lo < 0 || hi < lo || hi > p.rows;
    return *bad ? make_int2(0, 0) : make_int2(lo, hi);
}
__device__ __forceinline__ int prompt_tiles(const PromptParams& p, int b)
{
    bool bad;
    const int2 r = prompt_rows(p, b, &bad);
    return (r.y - r.x + p.tile_rows - 1) / p.tile_rows;
}

// Items in order: tiles of all prompts by falling index (so by falling number of keys), prompts in order within one index, heads within a tile.  The
// cursor goes down from level to level; a level's tiles are counted by the warp.
struct Cursor { int level, above; };            // tiles with a higher index than `level`

__device__ __forceinline__ int tiles_from(const PromptParams& p, int level, int lane)
{
    int n = 0;
    for (int b = lane; b < p.n_seqs; b += 32) n += max(0, prompt_tiles(p, b) - level);
    return __reduce_add_sync(0xffffffffu, n);
}

// The `tile`-th tile: (prompt, index), or prompt -1 behind the last.  Calls with rising `tile`.
__device__ __forceinline__ int2 find_tile(const PromptParams& p, Cursor& c, int tile, int lane)
{
    while (c.level >= 0) {
        const int upto = tiles_from(p, c.level, lane);
        if (tile < upto) break;
        c.above = upto;
        --c.level;
    }
    if (c.level < 0) return make_int2(-1, 0);
    int nth = tile - c.above;                   // of the prompts with more tiles than `level`
    for (int b0 = 0; b0 < p.n_seqs; b0 += 32) {
        const int b = b0 + lane;
        uint32_t has = __ballot_sync(0xffffffffu, b < p.n_seqs && prompt_tiles(p, b) > c.level);
        const int n = __popc(has);
        if (nth >= n) { nth -= n; continue; }
        while (nth--) has &= has - 1;
        return make_int2(b0 + __ffs(has) - 1, c.level);
    }
    return make_int2(-1, 0);
}

template <class S>
__global__ void __launch_bounds__(kThreads, 1) prompt_kernel(const __grid_constant__ PromptParams p)
{
    constexpr int D = S::D, NS = S::STAGES;
    using B = Bars<S>;
    extern __shared__ unsigned char smem_prompt[];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    __shared__ Item items[kSlots];
    __shared__ __align__(8) uint64_t barriers[B::kCount];

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t q_tiles = (smem_addr(smem_prompt) + 1023u) & ~1023u, ring_tiles = q_tiles + 2 * S::TILE;
    const uint32_t bars = smem_addr(barriers);
    auto bar = [&](int n) { return bars + 8u * n; };

    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int i = 0; i < B::kCount; ++i) {
            const bool empty = i >= B::kEmpty && i < B::kEmpty + NS, ready = i >= B::kPReady && i < B::kPHalf + 2;
            mbar_init(bar(i), i >= B::kItemEmpty ? 11 : empty ? 2 : ready ? 4 : 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_slot)), "r"(kTmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot, tmem_o = tmem + 256;       // S (and P) of A, of B; O of A, of B
    volatile int* abort_p = &abort_flag;
    bool ok = true;
    Ring slot;                                                  // of the item at hand
    wait_for_stream();
    // the next item for everyone but the scheduler
    auto take = [&](Item* it) {
        if (!warp_wait(bar(B::kItemFull + slot.at), slot.phase, abort_p)) return false;
        *it = items[slot.at];
        return true;
    };
    auto give_back = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive_local(bar(B::kItemEmpty + slot.at));
        slot.next(kSlots);
    };

    // 384 threads were launched with 168 registers each; a softmax thread holds a row of 128 scores: 128 * 88 + 256 * 208 = 384 * 168
    if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        Ring st;
        st.phase = 1;
        uint32_t q_phase = 1, loaded = 0, n_a = 0, n_b = 0;
        Item it;
        auto load = [&](const CUtensorMap* map, int head, int row) {
            if (!warp_wait(bar(B::kEmpty + st.at), st.phase, abort_p)) return false;
            if (elect_one()) {
                mbar_expect_tx(bar(B::kFull + st.at), S::TILE);
#pragma unroll
                for (int i = 0; i < D / 64; ++i) tma_load3(ring_tiles + st.at * S::TILE + i * S::BOX, map, i * 64, head, row, bar(B::kFull + st.at));
            }
            __syncwarp();
            st.next(NS);
            ++loaded;
            return true;
        };
        auto load_q = [&](int which, int head, int row) {
            if (elect_one()) {
                mbar_expect_tx(bar(B::kQFull + which), S::TILE);
#pragma unroll
                for (int i = 0; i < D / 64; ++i) tma_load3(q_tiles + which * S::TILE + i * S::BOX, &p.map_q, i * 64, head, row, bar(B::kQFull + which));
            }
            __syncwarp();
        };
        while (ok) {
            if (!take(&it)) { ok = false; break; }
            if (it.steps_a == 0) break;
            if (!warp_wait(bar(B::kQEmpty), q_phase, abort_p)) { ok = false; break; }
            q_phase ^= 1u;
            const int kv_head = it.head_a / p.group, steps = max(it.steps_a, it.steps_b);
            load_q(0, it.head_a, it.row_a);
            ++n_a;
            if (!load(&p.map_k, kv_head, it.begin)) { ok = false; break; }
            if (it.steps_b) { load_q(1, it.head_b, it.row_b); ++n_b; }
            for (int j = 0; j < steps; ++j) {
                if (!load(&p.map_v, kv_head, it.begin + j * kTileRows)) { ok = false; break; }
                if (j + 1 < steps && !load(&p.map_k, kv_head, it.begin + (j + 1) * kTileRows)) { ok = false; break; }
            }
            if (ok) give_back();
        }
        if (!ok && lane == 0) raise_abort(&abort_flag, p.status);
        __syncwarp();
        // the copies must have landed before the CTA may exit, also when it gives up
        for (uint32_t q = loaded > NS ? loaded - NS : 0u; q < loaded; ++q)
            for (uint32_t i = 0; i < kSpinLimitG; ++i)
                if (mbar_try(bar(B::kFull + q % NS), (q / NS) & 1u)) break;
        for (int which = 0; which < 2; ++which) {
            const uint32_t n = which ? n_b : n_a;
            if (n)
                for (uint32_t i = 0; i < kSpinLimitG; ++i)
                    if (mbar_try(bar(B::kQFull + which), (n - 1) & 1u)) break;
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        Ring st, clean;
        uint32_t q_phase[2] = {0, 0}, p_phase[2] = {0, 0};
        Item it;
        auto wait = [&](int n, uint32_t phase) { ok = ok && warp_wait(bar(n), phase, abort_p); return ok; };
        // S of tile `which` from the keys in `stage`
        auto product_s = [&](int which, uint32_t stage) {
            const uint32_t a = smem_desc_lo(q_tiles + which * S::TILE), b = smem_desc_lo(ring_tiles + stage * S::TILE);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const uint32_t o = (k >> 2) * (S::BOX >> 4) + (k & 3) * 2;
                umma_ss(tmem + which * kTileRows, a + o, b + o, S::IDESC_S, k != 0);
            }
        };
        // O of tile `which` += P V with the values in `stage`: 64-element columns of values lie a box apart, groups of 8 keys 1024 bytes
        auto product_o = [&](int which, uint32_t stage, bool first, int half) {
            const uint32_t addr = ring_tiles + stage * S::TILE;
            const uint32_t b = ((addr & 0x3ffffu) >> 4) | (S::BOX >> 4 << 16);
#pragma unroll
            for (int i = 0; i < kTileRows / 32; ++i) {
                const int k = half * (kTileRows / 32) + i;
                umma_ts(tmem_o + which * 128, tmem + which * kTileRows + k * 8, b + k * (2048 >> 4), S::IDESC_O, !first || k != 0);
            }
        };
        while (ok) {
            if (!take(&it)) { ok = false; break; }
            const int steps_a = it.steps_a, steps_b = it.steps_b, steps = max(steps_a, steps_b);
            if (steps_a == 0) break;
            const int watched = steps_b ? min(steps_a, steps_b) - 1 : steps_a - 1;      // the first step whose values are watched
            uint32_t k_stage = st.at;
            if (!wait(B::kQFull, q_phase[0]) || !wait(B::kFull + st.at, st.phase)) break;
            st.next(NS);
            q_phase[0] ^= 1u;
            tc_fence_after();
            if (elect_one()) {
                product_s(0, k_stage);
                umma_commit(bar(B::kSFull));
            }
            __syncwarp();
            if (steps_b) {
                if (!wait(B::kQFull + 1, q_phase[1])) break;
                q_phase[1] ^= 1u;
                tc_fence_after();
            }
            if (elect_one()) {
                if (steps_b) {
                    product_s(1, k_stage);
                    umma_commit(bar(B::kSFull + 1));
                }
                umma_commit(bar(B::kEmpty + k_stage));
                if (steps == 1) umma_commit(bar(B::kQEmpty));
            }
            __syncwarp();
            for (int j = 0; j < steps && ok; ++j) {
                const uint32_t v_stage = st.at, v_phase = st.phase;
                st.next(NS);
                if (j >= watched) {
                    if (!wait(B::kClean + clean.at, clean.phase)) break;
                    clean.next(NS);
                } else if (!wait(B::kFull + v_stage, v_phase)) break;
                const bool more = j + 1 < steps;
                if (more) {
                    k_stage = st.at;
                    if (!wait(B::kFull + st.at, st.phase)) break;
                    st.next(NS);
                }
#pragma unroll
                for (int which = 0; which < 2; ++which) {
                    const int mine = which ? steps_b : steps_a;
                    const bool live = j < mine;
                    if (live) {
                        if (!wait(B::kPHalf + which, p_phase[which])) break;
                        tc_fence_after();
                        if (elect_one()) product_o(which, v_stage, j == 0, 0);
                        __syncwarp();
                        if (!wait(B::kPReady + which, p_phase[which])) break;
                        p_phase[which] ^= 1u;
                        tc_fence_after();
                    }
                    if (elect_one()) {
                        if (live) {
                            product_o(which, v_stage, j == 0, 1);
                            if (j + 1 == mine) umma_commit(bar(B::kOFull + which));
                        }
                        if (which == 1) umma_commit(bar(B::kEmpty + v_stage));
                        if (j + 1 < mine) {
                            product_s(which, k_stage);
                            umma_commit(bar(B::kSFull + which));
                        }
                        if (which == 1 && more) {
                            umma_commit(bar(B::kEmpty + k_stage));
                            if (j + 2 == steps) umma_commit(bar(B::kQEmpty));
                        }
                    }
                    __syncwarp();
                }
            }
            if (ok) give_back();
        }
        if (!ok && lane == 0) raise_abort(&abort_flag, p.status);
    } else if (warp == 2) {
        // ------------------------------------------------------------------ scheduler
        Ring out;
        out.phase = 1;
        int most = 0;
        for (int b = lane; b < p.n_seqs; b += 32) {
            bool bad;
            prompt_rows(p, b, &bad);
            if (bad && blockIdx.x == 0 && p.status) atomicCAS(p.status, 0, static_cast<int>(POLYSPEC_ERR_BAD_INPUT_ON_DEVICE));
            most = max(most, prompt_tiles(p, b));
        }
        most = __reduce_max_sync(0xffffffffu, most);
        Cursor c = {most - 1, 0};
        // to and fro over the CTAs, so that none gets the longest item of every round
        for (int round = 0;; ++round) {
            const int n = round * gridDim.x + (round & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
            const int2 t = find_tile(p, c, n / p.pairs, lane);
            Item it = {0, 0, 0, 0, 0, 0, 0, 0, 0};
            if (t.x >= 0) {
                bool bad;
                const int2 r = prompt_rows(p, t.x, &bad);
                const int pair = n % p.pairs, row = t.y * p.tile_rows;
                it.begin = r.x;
                it.end = r.y;
                it.row_a = r.x + row;
                it.steps_a = row / kTileRows + 1;
                if (p.tile_rows == kTileRows) {
                    it.head_a = 2 * pair;
                    it.head_b = 2 * pair + 1;
                    it.row_b = it.row_a;
                    it.steps_b = it.steps_a;
                } else {
                    it.head_a = it.head_b = pair;
                    it.row_b = it.row_a + kTileRows;
                    it.steps_b = it.row_b < r.y ? it.steps_a + 1 : 0;
                }
            }
            if (!warp_wait(bar(B::kItemEmpty + out.at), out.phase, abort_p)) { ok = false; break; }
            if (lane == 0) {
                items[out.at] = it;
                mbar_arrive_local(bar(B::kItemFull + out.at));
            }
            __syncwarp();
            out.next(kSlots);
            if (t.x < 0) break;
        }
        if (!ok && lane == 0) raise_abort(&abort_flag, p.status);
    } else {
        // ------------------------------------------------------------------ values that are not finite
        Ring st, clean;
        Item it;
        while (ok) {
            if (!take(&it)) { ok = false; break; }
            const int steps = max(it.steps_a, it.steps_b);
            if (steps == 0) break;
            const int watched = it.steps_b ? min(it.steps_a, it.steps_b) - 1 : it.steps_a - 1;
            for (int n = 0; n < 2 * steps; ++n) {               // K0 V0 K1 V1 ...
                if (!warp_wait(bar(B::kFull + st.at), st.phase, abort_p)) { ok = false; break; }
                if ((n & 1) && n / 2 >= watched) {
                    const uint32_t tile = ring_tiles + st.at * S::TILE + lane * 16;
                    for (uint32_t o = 0; o < S::TILE; o += 2048) {
                        uint32_t x[4][4];
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                                         : "=r"(x[u][0]), "=r"(x[u][1]), "=r"(x[u][2]), "=r"(x[u][3]) : "r"(tile + o + u * 512) : "memory");
                        uint32_t some = 0;
#pragma unroll
                        for (int u = 0; u < 4; ++u)
#pragma unroll
                            for (int e = 0; e < 4; ++e) some |= (x[u][e] & 0x7f807f80u) + 0x00800080u;     // a carry out of an exponent of all ones
                        if (!(some & 0x80008000u)) continue;
                        *reinterpret_cast<volatile int*>(&items[slot.at].dirty) = 1;
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const uint32_t over = ((x[u][e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
                                x[u][e] &= ~((over >> 15) * 0xffffu);
                            }
                            asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};"
                                         ::"r"(tile + o + u * 512), "r"(x[u][0]), "r"(x[u][1]), "r"(x[u][2]), "r"(x[u][3]) : "memory");
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __threadfence_block();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_local(bar(B::kClean + clean.at));
                    clean.next(NS);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive_local(bar(B::kEmpty + st.at));
                st.next(NS);
            }
            if (ok) give_back();
        }
        if (!ok && lane == 0) raise_abort(&abort_flag, p.status);
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        // ------------------------------------------------------------------ softmax and epilogue
        const int which = (warp - 4) >> 2, quarter = warp & 3, r = quarter * 32 + lane;
        const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
        const uint32_t s_at = tmem + which * kTileRows + lanes, o_at = tmem_o + which * 128 + lanes;
        const float c = p.scale_log2;
        uint32_t s_phase = 0, o_phase = 0;
        Item it;
        while (ok) {
            if (!take(&it)) { ok = false; break; }
            if (it.steps_a == 0) break;
            const int steps = which ? it.steps_b : it.steps_a;
            float m = -INFINITY, l = 0.0f;
            for (int j = 0; j < steps; ++j) {
                if (!warp_wait(bar(B::kSFull + which), s_phase, abort_p)) { ok = false; break; }
                s_phase ^= 1u;
                tc_fence_after();
                float s[kTileRows];
#pragma unroll
                for (int i = 0; i < 4; ++i) tmem_ld32(s_at + i * 32, s + i * 32);
                tmem_ld_wait(s);
                if (j + 1 == steps) {
#pragma unroll
                    for (int i = 0; i < kTileRows; ++i)
                        if (i > r) s[i] = -INFINITY;
                }
                float top[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
                for (int i = 4; i + 1 < kTileRows; i += 2) top[i >> 1 & 3] = max3(top[i >> 1 & 3], s[i], s[i + 1]);
                const float most = fmaxf(max3(top[0], top[1], top[2]), top[3]);
                if (j == 0) m = most;
                else if (__any_sync(0xffffffffu, (most - m) * c > kSlack)) {
                    const float to = fmaxf(m, most), by = to == m ? 1.0f : ex2((m - to) * c);
                    m = to;
                    l *= by;
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) {
                        float o[32];
                        tmem_ld32(o_at + i * 32, o);
                        tmem_ld_wait(o);
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] *= by;
                        tmem_st32(o_at + i * 32, reinterpret_cast<const uint32_t*>(o));
                    }
                }
                const float mc = m == -INFINITY ? 0.0f : m * c;
                const uint64_t c2 = pair(c, c), mc2 = pair(-mc, -mc);
                uint64_t sum0 = 0, sum1 = 0;                    // two pairs of zeros
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t x[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        float a, b;
                        unpair(fma2(pair(s[64 * h + 2 * i], s[64 * h + 2 * i + 1]), c2, mc2), &a, &b);
                        a = ex2(a);
                        b = ex2(b);
                        if (i & 1) sum1 = add2(sum1, pair(a, b));
                        else sum0 = add2(sum0, pair(a, b));
                        x[i] = bf16x2_bits(a, b);
                    }
                    tmem_st32(s_at + 32 * h, x);
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_local(bar((h ? B::kPReady : B::kPHalf) + which));
                }
                {
                    float a, b;
                    unpair(add2(sum0, sum1), &a, &b);
                    l += a + b;
                }
            }
            if (!ok) break;
            if (steps) {
                if (!warp_wait(bar(B::kOFull + which), o_phase, abort_p)) { ok = false; break; }
                o_phase ^= 1u;
                tc_fence_after();
                const int row = (which ? it.row_b : it.row_a) + r, head = which ? it.head_b : it.head_a;
                const bool live = row < it.end, dirty = *reinterpret_cast<volatile int*>(&items[slot.at].dirty) != 0;
                const float inv = 1.0f / l;
                const size_t at = static_cast<size_t>(row) * p.q_heads + head;
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    float o[32];
                    tmem_ld32(o_at + i * 32, o);
                    tmem_ld_wait(o);
                    if (dirty && live) {
                        // the values that were replaced by 0, from the first key that was watched up to the row's own
                        const int first = it.begin + (it.row_a - it.begin) / kTileRows * kTileRows;
                        for (int key = first; key <= row; ++key) {
                            const unsigned short* v = p.v + key * p.v_stride + head / p.group * D + i * 32;
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if ((v[e] & 0x7f80u) == 0x7f80u) o[e] += __uint_as_float(static_cast<uint32_t>(v[e]) << 16);
                        }
                    }
                    if (live) {
                        uint4* to = reinterpret_cast<uint4*>(p.out + at * D + i * 32);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            to[e] = make_uint4(bf16x2_bits(o[8 * e] * inv, o[8 * e + 1] * inv), bf16x2_bits(o[8 * e + 2] * inv, o[8 * e + 3] * inv),
                                               bf16x2_bits(o[8 * e + 4] * inv, o[8 * e + 5] * inv), bf16x2_bits(o[8 * e + 6] * inv, o[8 * e + 7] * inv));
                    }
                }
                if (live && p.lse) p.lse[at] = (m * c + log2f(l)) * 0.69314718055994530942f;
                tc_fence_before();
            }
            give_back();
        }
        if (!ok && lane == 0) raise_abort(&abort_flag, p.status);
    }

    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) {
        if (*abort_p) __nanosleep(1000000);             // giving up: MMAs in flight get a bounded moment
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmem) : "memory");
    }
}

std::mutex g_mutex;
EncodeTiledFn g_encode = nullptr;

bool encode_rows(CUtensorMap* map, const void* base, int head_dim, int heads, int rows, long long stride)
{
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(head_dim), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(head_dim) * 2, static_cast<cuuint64_t>(stride) * 2};
    const cuuint32_t box[3] = {64, 1, kTileRows}, one[3] = {1, 1, 1};
    return g_encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Tensors { const void *q, *k, *v; long long q_stride, k_stride, v_stride; int kv_heads; };

template <class S>
cudaError_t launch_prompt(PromptParams& p, const Tensors& t, cudaStream_t stream)
{
    {
        std::lock_guard<std::mutex> lock(g_mutex);
        if (!g_encode) {
            const cudaError_t e = find_encoder(&g_encode);
            if (e != cudaSuccess) return e;
        }
    }
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    // before the encoding: that is a driver call, which wants a context current in this host thread, and this binds one
    if (e == cudaSuccess) e = cudaFuncSetAttribute(prompt_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(S::SMEM));
    if (e != cudaSuccess) return e;
    if (!encode_rows(&p.map_q, t.q, S::D, p.q_heads, p.rows, t.q_stride) || !encode_rows(&p.map_k, t.k, S::D, t.kv_heads, p.rows, t.k_stride) ||
        !encode_rows(&p.map_v, t.v, S::D, t.kv_heads, p.rows, t.v_stride))
        return cudaErrorInvalidValue;
    const long long items = (static_cast<long long>(p.rows) / p.tile_rows + p.n_seqs) * p.pairs;         // at most
    return launch_early(prompt_kernel<S>, dim3(static_cast<unsigned>(std::min<long long>(sms, items))), kThreads, S::SMEM, stream, p);
}

}  // namespace
}  // namespace polyspec

using namespace polyspec;

extern "C" polyspec_status polyspec_prompt_attention(const void* q, long long q_stride, const void* k, long long k_stride, const void* v, long long v_stride,
                                                     const int32_t* rows_at, int n_seqs, int rows, int q_heads, int kv_heads, int head_dim, float scale,
                                                     void* out, float* lse, int32_t* device_status, void* cuda_stream)
{
    if (n_seqs < 1 || rows < 1) return POLYSPEC_ERR_INVALID_ARG;
    const polyspec_status st = kv::check_heads(q_heads, kv_heads, head_dim);
    if (st != POLYSPEC_OK) return st;
    if (rows > (1 << 24) || n_seqs > (1 << 20)) return POLYSPEC_ERR_UNSUPPORTED;
    if (!kv::rows_ok(q, q_stride, q_heads, head_dim) || !kv::rows_ok(k, k_stride, kv_heads, head_dim) || !kv::rows_ok(v, v_stride, kv_heads, head_dim))
        return POLYSPEC_ERR_INVALID_ARG;
    if (!rows_at || !out || !kv::aligned16(out) || !aligned4(rows_at, lse, device_status)) return POLYSPEC_ERR_INVALID_ARG;
    if (!(scale >= 0.0f && scale <= 1.0e30f)) return POLYSPEC_ERR_INVALID_ARG;
    PromptParams p;
    p.rows_at = rows_at;
    p.v = static_cast<const unsigned short*>(v);
    p.v_stride = v_stride;
    p.n_seqs = n_seqs; p.rows = rows; p.q_heads = q_heads; p.group = q_heads / kv_heads;
    p.pairs = p.group % 2 ? q_heads : q_heads / 2;
    p.tile_rows = p.group % 2 ? 2 * kTileRows : kTileRows;
    p.scale_log2 = std::max(scale * 1.44269504088896340736f, 1.0e-37f);         // (0 times a masked score, -inf, would be NaN)
    p.out = static_cast<unsigned short*>(out);
    p.lse = lse;
    p.status = device_status;
    const Tensors t = {q, k, v, q_stride, k_stride, v_stride, kv_heads};
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = head_dim == 128 ? launch_prompt<Shape<128>>(p, t, stream) : launch_prompt<Shape<64>>(p, t, stream);
    return cuda_failed(e) ? POLYSPEC_ERR_CUDA : POLYSPEC_OK;
}
