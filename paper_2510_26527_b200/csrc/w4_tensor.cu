// LM-head projection with 4-bit weights on the fifth-generation tensor cores, for more rows than the streaming kernel takes
// (formula, numerics and weight format: w4_head.cu).
//
// The vocabulary is the MMA's M axis (128 entries per tile = the 128 lanes of tensor memory), the hidden rows its N axis.
// The expanded weights never touch shared memory: dequantising warps read the packed tile, turn codes into exact bf16
// integers q - z and write them with tcgen05.st into tensor memory, from where the MMA takes its A operand.  Each group of
// weights is accumulated by the tensor core into a slot of its own, and the epilogue warps multiply the slot's fp32 sums by
// the group's scale -- one scale per lane, since a lane is a vocabulary entry -- and add them to the running sums in their
// registers.  So the scale costs one FMA per (entry, row, group) instead of a rounding per weight.
//
// Persistent, one CTA per SM; work items are (vocabulary tile, block of hidden rows), the row blocks of one tile neighbours so
// that its codes come from L2 the second time.  Warp roles (18 warps):
//   0        TMA producer: per K block, the packed tile (boxes of 128 rows x 64 bytes, 64-byte swizzle) and the hidden tile (boxes
//            of 64 elements, 128-byte swizzle)
//   1        MMA issuer; allocates and frees tensor memory
//   then     dequantisers, in sets of four warps (one per lane quarter): a set takes every second or third K block, so that the
//            latencies of one (shared-memory reads, tensor-memory stores, barriers) pass behind the arithmetic of another
//   last     epilogue, one or two warps per lane quarter, each its share of the columns
// Tensor memory: A blocks in a ring, then accumulator slots in a ring; a slot takes as many of a block's groups as leave two
// slots, so that small groups do not multiply the handshakes.
// With few rows an MMA is short and what a block costs is the MMA warp's own handshakes (some 90 cycles per wait that passes at
// once, by time stamps): blocks of 256 elements up to 64 rows, 128 above.
// Measured as a replayed graph, 32000 x 4096 in groups of 128: 9 rows 23.3 us, 288 rows 83 us, 909 TFLOP/s (95 us, 793 TFLOP/s in calls
// queued by the host; tensor pipe 40%, issue slots 60%; every tile of 128 entries reads all hidden rows, 0.58 GB from L2);
// 37 x 12807 x 2080 in groups of 32 17.1 us (101 tiles on 148 SMs).  The shapes were chosen on groups of 128; small groups leave
// fewer MMAs to each slot's handshake: 288 rows 123 us in groups of 64, 203 us in groups of 32; 64 rows 32 us, in groups of 32 57 us.
//
// Every wait on an mbarrier is bounded: one that runs out raises an abort flag that all roles poll, sets POLYSPEC_ERR_TIMEOUT,
// and the kernel still lets its copies land, frees tensor memory and returns.
#include <cuda.h>

#include <algorithm>
#include <mutex>

#include "launch.cuh"
#include "polyspec_kernels.cuh"
#include "tensor_device.cuh"
#include "w4_kernels.cuh"

namespace polyspec {
namespace {

using namespace tensordev;

constexpr int kTileV = 128;
constexpr int kSub = 128;                               // K elements per box of codes
constexpr int kSubBytes = kTileV * kSub / 2;            // 8 KiB
constexpr int kSetWarps = 4;                            // dequantising warps per K block
constexpr int kMaxStages = 12, kMaxSlots = 8, kMaxABlocks = 4;
constexpr int kTmemCols = 512;
constexpr int kMaxRowsPerItem = 144;                    // an epilogue thread holds half of them as accumulators
constexpr size_t kSmemLimit = 227 * 1024;

struct TensorParams {
    CUtensorMap map_codes;      // [V, d / 2] bytes, box {64, 128}
    CUtensorMap map_hidden;     // [rows, d] bf16, box {64, N}
    const unsigned short* scales;       // bf16 bits
    const unsigned char* zeros;
    void* out;
    int out_bf16;
    int rows, V, group, groups; // groups: of a whole row
    int kblocks;
    int row_blocks, items;
    int vectors;                // groups a multiple of eight, scales and zero points aligned for vector loads
    uint32_t idesc, exponent;
    int32_t* status;
};

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

// D (tensor memory) = or += A (tensor memory) B (shared memory descriptor)
__device__ __forceinline__ void umma_from_tmem(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc, uint32_t accumulate)
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

__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
        ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
          "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
          "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_ld8(uint32_t addr, uint32_t* r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(addr) : "memory");
}

__device__ __forceinline__ void raise_abort(int* abort_flag, int32_t* status)
{
    if (!*reinterpret_cast<volatile int*>(abort_flag) && status) atomicCAS(status, 0, static_cast<int>(POLYSPEC_ERR_TIMEOUT));
    *reinterpret_cast<volatile int*>(abort_flag) = 1;
}

// A bounded wait that the whole warp passes or the whole warp gives up (what follows are warp-wide instructions).  Plain polls: with
// a suspend-time hint on the tries, wake-ups came late and 288 rows took 95 instead of 90 microseconds.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag)
{
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
}

// The same for two barriers at once: what a passing wait costs is its latency, and the two overlap.
__device__ __forceinline__ bool warp_wait2(uint32_t bar0, uint32_t parity0, uint32_t bar1, uint32_t parity1, volatile int* abort_flag)
{
    const bool first = mbar_try(bar0, parity0), second = mbar_try(bar1, parity1);
    if (__all_sync(0xffffffffu, first && second)) return true;
    return warp_wait(bar0, parity0, abort_flag) && warp_wait(bar1, parity1, abort_flag);
}

// A position in a ring of n: its index and the parity a consumer waits for.
struct Ring {
    uint32_t at = 0, phase = 0;
    __device__ __forceinline__ void next(uint32_t n)
    {
        if (++at == n) { at = 0; phase ^= 1u; }
    }
};

// Sizes of an instantiation.  NC: columns (hidden rows) per epilogue warp; EPI: epilogue warps; SETS: sets of dequantising warps;
// BLOCK: K elements per block; ABLOCKS: A blocks in tensor memory.
template <int NC_, int EPI_, int SETS_, int BLOCK_, int ABLOCKS_>
struct Shape {
    static constexpr int NC = NC_, EPI = EPI_, SETS = SETS_, BLOCK = BLOCK_, kABlocks = ABLOCKS_;
    static constexpr int N = NC * (EPI / 4);
    static constexpr int kThreads = 32 * (2 + kSetWarps * SETS + EPI);
    static constexpr int kSubs = BLOCK / kSub;
    static constexpr uint32_t kCodeBytes = kSubs * kSubBytes, kBoxBytes = N * 128, kStage = kCodeBytes + BLOCK / 64 * kBoxBytes;
    static constexpr int kACols = BLOCK / 2;                // two bf16 per 32-bit column
    static constexpr int kAccCols = kTmemCols - kABlocks * kACols;
    static constexpr int kStages = (kSmemLimit - 4096) / kStage < kMaxStages ? (kSmemLimit - 4096) / kStage : kMaxStages;
    static constexpr size_t kSmem = 1024 + static_cast<size_t>(kStages) * kStage;
    static_assert(2 * N <= kAccCols && kStages >= 3 && kStage % 1024 == 0 && kBoxBytes % 1024 == 0 && kABlocks <= kMaxABlocks, "sizes");
    // A wait tells a phase from the one before it, not from the one two before.  A set that comes to block b has seen the MMAs of
    // block b - SETS - kABlocks done.  So the A block of b was last used by b - kABlocks, whose own predecessor there must be
    // among those: SETS <= kABlocks; and the stage of b by b - kStages, which must be among those or the set's own.
    static_assert(SETS <= kABlocks && (kStages >= SETS + kABlocks || kStages % SETS == 0), "phases");
};
// With GROUPS groups in a K block: groups per slot, slots.
template <class S, int GROUPS>
struct Slots {
    static constexpr int kUnit = GROUPS >= 4 && 8 * S::N <= S::kAccCols ? 4 : GROUPS >= 2 && 4 * S::N <= S::kAccCols ? 2 : 1;
    static constexpr int kCols = kUnit * S::N;
    static constexpr int kCount = S::kAccCols / kCols < kMaxSlots ? S::kAccCols / kCols : kMaxSlots;
};

struct Barriers { uint32_t full, empty, a_full, a_empty, acc_full, acc_empty; };

// The MMA issuer's whole run.  The number of groups per K block is a template argument so that a block's MMAs are straight-line
// code on uniform registers: with the loop bounds read from the parameters 288 x 32000 x 4096 took 121 us
// instead of 90 (sets on alternating blocks, introduced with it, included).
// A full A block was made from the stage's codes after its copies, the hidden tile's among them, had landed: no wait for those.
// One commit per slot is all the issuer signals with: whoever has seen a block's last slot full knows that its stage and its A
// block have been read, and an epilogue warp hands both back (288 x 32000 x 4096: three commits a block 91 us, one 84).
template <class S, int GROUPS>
__device__ __forceinline__ bool issue_all(const TensorParams& p, const Barriers& bar, uint32_t tiles, uint32_t tmem, uint32_t tmem_acc, volatile int* abort_p)
{
    using L = Slots<S, GROUPS>;
    constexpr int kMmas = S::BLOCK / 16 / GROUPS;       // per group
    Ring st, ab, slot;
    slot.phase = 1;
    for (int item = blockIdx.x; item < p.items; item += gridDim.x) {
        for (int kb = 0; kb < p.kblocks; ++kb) {
            if (!warp_wait2(bar.a_full + 8u * ab.at, ab.phase, bar.acc_empty + 8u * slot.at, slot.phase, abort_p)) return false;
            tc_fence_after();
            const uint32_t b_lo = smem_desc_lo(tiles + st.at * S::kStage + S::kCodeBytes);
            const uint32_t a = tmem + ab.at * S::kACols;
#pragma unroll
            for (int g0 = 0; g0 < GROUPS; g0 += L::kUnit) {
                if (kb * GROUPS + g0 >= p.groups) break;
                if (g0 > 0) {
                    if (!warp_wait(bar.acc_empty + 8u * slot.at, slot.phase, abort_p)) return false;
                    tc_fence_after();
                }
                const uint32_t d = tmem_acc + slot.at * L::kCols;
                if (elect_one()) {
#pragma unroll
                    for (int u = 0; u < L::kUnit; ++u) {
                        if (u > 0 && kb * GROUPS + g0 + u >= p.groups) break;
#pragma unroll
                        for (int m = 0; m < kMmas; ++m) {
                            const int kk = (g0 + u) * kMmas + m;        // 16-element slice of the block
                            umma_from_tmem(d + u * S::N, a + kk * 8, b_lo + (kk >> 2) * (S::kBoxBytes >> 4) + (kk & 3) * 2, p.idesc, m != 0);
                        }
                    }
                    umma_commit(bar.acc_full + 8u * slot.at);
                }
                __syncwarp();
                slot.next(L::kCount);
            }
            st.next(S::kStages);
            ab.next(S::kABlocks);
        }
    }
    return true;
}

// Zero points, scales of the aligned run `run` of eight groups of one row, as vectors where rows hold a multiple of eight groups.
__device__ __forceinline__ uint2 load_zeros8(const TensorParams& p, const unsigned char* zero, int run)
{
    if (!zero) return make_uint2(0x08080808u, 0x08080808u);
    if (p.vectors) return reinterpret_cast<const uint2*>(zero)[run];
    uint32_t z[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i >> 2] |= static_cast<uint32_t>(zero[min(run * 8 + i, p.groups - 1)]) << (8 * (i & 3));
    return make_uint2(z[0], z[1]);
}
__device__ __forceinline__ uint4 load_scales8(const TensorParams& p, const unsigned short* scale, int run)
{
    if (p.vectors) return reinterpret_cast<const uint4*>(scale)[run];
    uint32_t s[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i >> 1] |= static_cast<uint32_t>(scale[min(run * 8 + i, p.groups - 1)]) << (16 * (i & 1));
    return make_uint4(s[0], s[1], s[2], s[3]);
}

// An epilogue warp's whole run: for every item, the groups in order, a slot at a time, scaled and added to the running sums.
template <class S, int GROUPS>
__device__ __forceinline__ bool run_epilogue(const TensorParams& p, const Barriers& bar, uint32_t tmem_acc, int quarter, int share, int lane,
                                             volatile int* abort_p)
{
    using L = Slots<S, GROUPS>;
    constexpr int kBatch = S::NC >= 48 ? 24 : 32;        // columns read at a time, as the registers allow
    Ring slot, st, ab;
    const bool hands_back = quarter == 0 && share == 0;         // this warp returns stages and A blocks
    const uint32_t t0 = tmem_acc + (static_cast<uint32_t>(quarter * 32) << 16) + share * S::NC;
    for (int item = blockIdx.x; item < p.items; item += gridDim.x) {
        const int v = item / p.row_blocks * kTileV + quarter * 32 + lane, row0 = item % p.row_blocks * S::N + share * S::NC;
        const unsigned short* scale = p.scales + static_cast<size_t>(min(v, p.V - 1)) * p.groups;
        float sum[S::NC];
#pragma unroll
        for (int i = 0; i < S::NC; ++i) sum[i] = 0.0f;
        // scales in aligned runs of eight groups, the next run loaded while this one is used
        uint4 run = make_uint4(0, 0, 0, 0), run_next = load_scales8(p, scale, 0);
        for (int g = 0; g < p.groups; g += L::kUnit) {
            if ((g & 7) == 0) {
                run = run_next;
                if (g + 8 < p.groups) run_next = load_scales8(p, scale, g / 8 + 1);
            }
            float s[L::kUnit];
#pragma unroll
            for (int u = 0; u < L::kUnit; ++u) {
                const uint32_t at = (g + u) & 7, pair = at & 4 ? (at & 2 ? run.w : run.z) : (at & 2 ? run.y : run.x);
                s[u] = __uint_as_float(at & 1 ? pair & 0xffff0000u : pair << 16);
            }
            if (!warp_wait(bar.acc_full + 8u * slot.at, slot.phase, abort_p)) return false;
            tc_fence_after();
            if (hands_back && ((g + L::kUnit) % GROUPS == 0 || g + L::kUnit >= p.groups)) {         // the block's last slot
                tc_fence_before();
                if (lane == 0) {
                    mbar_arrive_local(bar.a_empty + 8u * ab.at);
                    mbar_arrive_local(bar.empty + 8u * st.at);
                }
                st.next(S::kStages);
                ab.next(S::kABlocks);
            }
            const uint32_t t = t0 + slot.at * L::kCols;
            const int left = p.groups - g;
#pragma unroll
            for (int c = 0; c < L::kUnit * S::NC; c += kBatch) {
                uint32_t x[kBatch];
#pragma unroll
                for (int q = 0; q < kBatch; q += 8) {
                    const int u = (c + q) / S::NC, col = (c + q) % S::NC;           // (compile-time)
                    if (u < L::kUnit && (u == 0 || u < left)) tmem_ld8(t + u * S::N + col, x + q);
                }
                tmem_ld_wait();
#pragma unroll
                for (int q = 0; q < kBatch; ++q) {
                    const int u = (c + q) / S::NC, col = (c + q) % S::NC;
                    if (u < L::kUnit && (u == 0 || u < left)) sum[col] = fmaf(s[u], __uint_as_float(x[q]), sum[col]);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_local(bar.acc_empty + 8u * slot.at);
            slot.next(L::kCount);
        }
        if (v >= p.V) continue;
        const int n = min(S::NC, p.rows - row0);
#pragma unroll
        for (int i = 0; i < S::NC; ++i) {
            if (i >= n) continue;
            const size_t at = static_cast<size_t>(row0 + i) * p.V + v;
            if (p.out_bf16) w4::store_logit<POLYSPEC_BF16>(p.out, at, sum[i]);
            else w4::store_logit<POLYSPEC_F32>(p.out, at, sum[i]);
        }
    }
    return true;
}

template <class S>
__global__ void __launch_bounds__(S::kThreads, 1) w4_tensor_kernel(const __grid_constant__ TensorParams p)
{
    extern __shared__ unsigned char smem_tensor[];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    __shared__ __align__(8) uint64_t barriers[2 * kMaxStages + 2 * kMaxABlocks + 2 * kMaxSlots];

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t tiles = (smem_addr(smem_tensor) + 1023u) & ~1023u;
    Barriers bar;
    bar.full = smem_addr(barriers);
    bar.empty = bar.full + 8u * kMaxStages;
    bar.a_full = bar.empty + 8u * kMaxStages;
    bar.a_empty = bar.a_full + 8u * kMaxABlocks;
    bar.acc_full = bar.a_empty + 8u * kMaxABlocks;
    bar.acc_empty = bar.acc_full + 8u * kMaxSlots;

    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int i = 0; i < kMaxStages; ++i) { mbar_init(bar.full + 8u * i, 1); mbar_init(bar.empty + 8u * i, kSetWarps + 1); }
        for (int i = 0; i < kMaxABlocks; ++i) { mbar_init(bar.a_full + 8u * i, kSetWarps); mbar_init(bar.a_empty + 8u * i, 1); }
        for (int i = 0; i < kMaxSlots; ++i) { mbar_init(bar.acc_full + 8u * i, 1); mbar_init(bar.acc_empty + 8u * i, S::EPI); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_slot)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot, tmem_acc = tmem + S::kABlocks * S::kACols;
    volatile int* abort_p = &abort_flag;
    const int per_sub = kSub / p.group;                 // groups per 128 elements: 1, 2 or 4
    bool ok = true;
    wait_for_stream();

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        Ring st;
        st.phase = 1;                                   // a fresh "empty" barrier passes a wait on parity 1
        uint32_t it = 0;
        for (int item = blockIdx.x; ok && item < p.items; item += gridDim.x) {
            const int v0 = item / p.row_blocks * kTileV, row0 = item % p.row_blocks * S::N;
            for (int kb = 0; kb < p.kblocks; ++kb, ++it) {
                if (!warp_wait(bar.empty + 8u * st.at, st.phase, abort_p)) { ok = false; break; }
                const uint32_t full = bar.full + 8u * st.at, dst = tiles + st.at * S::kStage;
                if (elect_one()) {
                    mbar_expect_tx(full, S::kStage);
#pragma unroll
                    for (int i = 0; i < S::kSubs; ++i) tma_load(dst + i * kSubBytes, &p.map_codes, (kb * S::kSubs + i) * (kSub / 2), v0, full);
#pragma unroll
                    for (int i = 0; i < S::BLOCK / 64; ++i)
                        tma_load(dst + S::kCodeBytes + i * S::kBoxBytes, &p.map_hidden, kb * S::BLOCK + i * 64, row0, full);
                }
                __syncwarp();
                st.next(S::kStages);
            }
        }
        if (!ok && lane == 0) raise_abort(&abort_flag, p.status);
        __syncwarp();
        // the copies must have landed before the CTA may exit, also when it gives up
        for (uint32_t q = it > S::kStages ? it - S::kStages : 0u; q < it; ++q)
            for (uint32_t i = 0; i < kSpinLimitG; ++i)
                if (mbar_try(bar.full + 8u * (q % S::kStages), (q / S::kStages) & 1u)) break;
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        if (per_sub == 1) ok = issue_all<S, S::kSubs>(p, bar, tiles, tmem, tmem_acc, abort_p);
        else if (per_sub == 2) ok = issue_all<S, 2 * S::kSubs>(p, bar, tiles, tmem, tmem_acc, abort_p);
        else ok = issue_all<S, 4 * S::kSubs>(p, bar, tiles, tmem, tmem_acc, abort_p);
        if (!ok && lane == 0) raise_abort(&abort_flag, p.status);
    } else if (warp < 2 + kSetWarps * S::SETS) {
        // ------------------------------------------------------------------ dequantisers
        const int quarter = warp & 3, set = (warp - 2) >> 2;
        const int r = quarter * 32 + lane;              // row of the tile
        Ring st, ab;
        ab.phase = 1;
        const uint32_t swizzle = (static_cast<uint32_t>(r) >> 1) & 3u;
        int turn = 0;                                   // whose K block the next one is
        for (int item = blockIdx.x; ok && item < p.items; item += gridDim.x) {
            const size_t v = static_cast<size_t>(min(item / p.row_blocks * kTileV + r, p.V - 1));
            const unsigned char* zero = p.zeros ? p.zeros + v * p.groups : nullptr;
            // The zero points of the eight groups (an aligned run of them) that the next block of this set belongs to, loaded a
            // turn ahead: arithmetic on a fresh load would wait for it.
            constexpr int kBlockSubs = S::kSubs;
            auto run_of = [&](int kb) { return min(kb * kBlockSubs * per_sub, p.groups - 1) / 8; };
            int run_next = run_of((set - turn + S::SETS) % S::SETS);
            uint2 z_next = load_zeros8(p, zero, run_next);
            for (int kb = 0; kb < p.kblocks; ++kb, turn = turn + 1 == S::SETS ? 0 : turn + 1) {
                if (turn != set) {
                    st.next(S::kStages);
                    ab.next(S::kABlocks);
                    continue;
                }
                const uint2 z = z_next;
                if (run_of(kb + S::SETS) != run_next) {
                    run_next = run_of(kb + S::SETS);
                    z_next = load_zeros8(p, zero, run_next);
                }
                if (!warp_wait(bar.full + 8u * st.at, st.phase, abort_p)) { ok = false; break; }
                const uint32_t row = tiles + st.at * S::kStage + static_cast<uint32_t>(r) * 64u;
                const uint32_t a = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + ab.at * S::kACols;
#pragma unroll
                for (int sub = 0; sub < S::kSubs; ++sub) {
                    uint32_t w[16];
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                                     : "=r"(w[4 * c]), "=r"(w[4 * c + 1]), "=r"(w[4 * c + 2]), "=r"(w[4 * c + 3])
                                     : "r"(row + sub * kSubBytes + ((c ^ swizzle) << 4)));
                    uint32_t magic[4];                  // of the four runs of 32 elements
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        // group of run i, counted from the aligned run of eight (32 i elements into sub-block `sub`)
                        const uint32_t at = ((kb * S::kSubs + sub) * per_sub + (per_sub == 1 ? 0 : per_sub == 2 ? i >> 1 : i)) & 7u;
                        const uint32_t x = (at & 4u ? z.y : z.x) >> (8u * (at & 3u));
                        magic[i] = p.exponent | (x & 15u) * 0x00010001u;
                    }
                    if (sub == S::kSubs - 1) {
                        __syncwarp();
                        if (lane == 0) mbar_arrive_local(bar.empty + 8u * st.at);           // the codes are in registers
                    }
                    if (sub == 0) {
                        if (!warp_wait(bar.a_empty + 8u * ab.at, ab.phase, abort_p)) { ok = false; break; }
                        tc_fence_after();
                    }
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        uint32_t x[32];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            uint32_t pairs[4];
                            w4::expand(w[half * 8 + i], magic[half * 2 + (i >> 2)], p.exponent, pairs);
#pragma unroll
                            for (int j = 0; j < 4; ++j) x[4 * i + j] = pairs[j];
                        }
                        tmem_st32(a + sub * (kSub / 2) + half * 32, x);
                    }
                }
                if (!ok) break;
                st.next(S::kStages);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_local(bar.a_full + 8u * ab.at);
                ab.next(S::kABlocks);
            }
        }
        if (!ok && lane == 0) raise_abort(&abort_flag, p.status);
    } else {
        // ------------------------------------------------------------------ epilogue
        const int quarter = warp & 3, share = (warp - 2 - kSetWarps * S::SETS) >> 2;
        if (per_sub == 1) ok = run_epilogue<S, S::kSubs>(p, bar, tmem_acc, quarter, share, lane, abort_p);
        else if (per_sub == 2) ok = run_epilogue<S, 2 * S::kSubs>(p, bar, tmem_acc, quarter, share, lane, abort_p);
        else ok = run_epilogue<S, 4 * S::kSubs>(p, bar, tmem_acc, quarter, share, lane, abort_p);
        if (!ok && lane == 0) raise_abort(&abort_flag, p.status);
    }

    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) {
        if (*abort_p) __nanosleep(1000000);             // giving up: MMAs in flight get a bounded moment
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

std::mutex g_mutex;
EncodeTiledFn g_encode = nullptr;

bool encode(CUtensorMap* map, CUtensorMapDataType type, const void* base, size_t inner, size_t outer, size_t pitch, int box_inner, int box_outer,
            CUtensorMapSwizzle swizzle)
{
    const cuuint64_t dims[2] = {inner, outer};
    const cuuint64_t strides[1] = {pitch};
    const cuuint32_t box[2] = {static_cast<cuuint32_t>(box_inner), static_cast<cuuint32_t>(box_outer)};
    const cuuint32_t one[2] = {1, 1};
    return g_encode(map, type, 2, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                    CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class S>
cudaError_t launch_shape(TensorParams& p, const W4Problem& q, int sms, cudaStream_t stream)
{
    p.kblocks = (q.d + S::BLOCK - 1) / S::BLOCK;
    p.row_blocks = (q.rows + S::N - 1) / S::N;
    const long long items = static_cast<long long>((q.V + kTileV - 1) / kTileV) * p.row_blocks;
    if (items > 0x7fffffffLL - sms) return cudaErrorInvalidValue;
    p.items = static_cast<int>(items);
    // D fp32, A and B bf16, both K-major, M = 128, N
    p.idesc = (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(S::N >> 3) << 17) | (static_cast<uint32_t>(kTileV >> 4) << 24);
    // before the encoding: that is a driver call, which wants a context current in this host thread, and this binds one
    cudaError_t e = cudaFuncSetAttribute(w4_tensor_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(S::kSmem));
    if (e != cudaSuccess) return e;
    if (!encode(&p.map_codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, q.codes, q.d / 2, q.V, q.d / 2, kSub / 2, kTileV, CU_TENSOR_MAP_SWIZZLE_64B) ||
        !encode(&p.map_hidden, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, q.hidden, q.d, q.rows, static_cast<size_t>(q.d) * 2, 64, S::N, CU_TENSOR_MAP_SWIZZLE_128B))
        return cudaErrorInvalidValue;
    return launch_early(w4_tensor_kernel<S>, dim3(static_cast<unsigned>(std::min(sms, p.items))), S::kThreads, S::kSmem, stream, p);
}

}  // namespace

cudaError_t launch_w4_tensor(const W4Problem& q, polyspec_dtype dt, int32_t* device_status, cudaStream_t stream)
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
    if (e != cudaSuccess) return e;
    TensorParams p;
    p.scales = static_cast<const unsigned short*>(q.scales);
    p.zeros = q.zeros;
    p.out = q.out;
    p.out_bf16 = dt == POLYSPEC_BF16;
    p.rows = q.rows;
    p.V = q.V;
    p.group = q.group;
    p.groups = q.d / q.group;
    p.status = device_status;
    p.exponent = w4::kExponent;
    p.vectors = p.groups % 8 == 0 && (reinterpret_cast<uintptr_t>(q.scales) & 15u) == 0 && (reinterpret_cast<uintptr_t>(q.zeros) & 7u) == 0;
    // columns of an item: the rows cut evenly into blocks of at most 144, in the next size there is
    const int blocks = (q.rows + kMaxRowsPerItem - 1) / kMaxRowsPerItem, cols = (q.rows + blocks - 1) / blocks;
    if (cols <= 16) return launch_shape<Shape<16, 4, 3, 256, 3>>(p, q, sms, stream);
    if (cols <= 32) return launch_shape<Shape<32, 4, 2, 256, 2>>(p, q, sms, stream);
    if (cols <= 48) return launch_shape<Shape<24, 8, 2, 256, 2>>(p, q, sms, stream);
    if (cols <= 64) return launch_shape<Shape<32, 8, 2, 256, 2>>(p, q, sms, stream);
    if (cols <= 96) return launch_shape<Shape<48, 8, 2, 128, 2>>(p, q, sms, stream);
    if (cols <= 128) return launch_shape<Shape<64, 8, 2, 128, 3>>(p, q, sms, stream);
    return launch_shape<Shape<72, 8, 2, 128, 3>>(p, q, sms, stream);
}

}  // namespace polyspec
