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
// w4_stream_kernel, up to eight rows: HBM-bound, every code is read once.  mma.sync.m16n8k16 with the vocabulary on the M axis:
// codes become A fragments in the registers of the lane that reads them.  With eight columns the tensor work is a small part of
// the time, and tcgen05 would want the expanded weights written to tensor memory or shared memory first (w4_tensor.cu).
// The codes are cut into pieces of 32 vocabulary entries (a tile) x 128 elements (2 KiB, one TMA box).  A CTA owns a contiguous
// range of tiles and its warps equal, contiguous shares of the pieces of that range, whatever tile borders they cross, each
// streamed through a private ring in shared memory: warps meet once, at the end, when the sums of tiles that several of them
// worked on are added up in a fixed order.  (Whole tiles per team of warps, with a reduction and two barriers per tile:
// 26.3 against 24.0 us on 1 x 32000 x 4096.)  The hidden rows are staged once per CTA in fragment
// order.
// Measured as a replayed graph: 1 x 32000 x 4096 in groups of 128, 20.5 us, 3.35 TB/s (floor 10.5; 4 to 5 us pass before the first
// piece is computed); 5 x 152064 x 8192 in groups of 64, 158 us, 4.3 TB/s (173 us, 3.9 TB/s in calls queued by the host; the same
// loop without the arithmetic streams in 103).  Neither memory (51 and 66%) nor issue (53 and 64% of the slots) is full: a warp takes
// one piece at a time through one dependent chain of wait, shared loads, expansion and MMA.
// Every wait on a copy is bounded: a warp whose wait runs out sets POLYSPEC_ERR_TIMEOUT, asks for nothing more, waits (again with
// a limit) for the copies it has on their way and goes to the barrier at the end.
#include <cuda_bf16.h>

#include <algorithm>
#include <mutex>

#include "launch.cuh"
#include "piece_ring.cuh"
#include "polyspec_kernels.cuh"
#include "tensor_device.cuh"
#include "w4_kernels.cuh"

namespace polyspec {
namespace {

constexpr int kWarpsS = 16;                     // warps per CTA, one CTA per SM
constexpr int kThreadsS = 32 * kWarpsS;
constexpr int kTileS = 32;                      // vocabulary entries per tile (two m16 tiles)
constexpr int kStreamRows = 8;                  // more rows go to the tensor-core kernel
constexpr int kChunk = 128;                     // d elements per step: 16 bytes of codes per lane and row

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

using namespace tensordev;

constexpr int kPieceBytes = kTileS * kChunk / 2;        // 2 KiB
// 64 KiB in flight per SM.  On 1 x 32000 x 4096 and 5 x 12807 x 2080, the sizes it was chosen on, six pieces put 28 MB of requests
// before the hidden rows and scales; longer runs were not swept.
constexpr int kMaxRing = 2;
constexpr int kTableGroups = 8;                         // groups whose scales and zero points a warp holds at a time
constexpr int kTableWords = kTableGroups * 32;
constexpr int kSums = 8;                                // accumulators per lane: two m16 tiles x four

struct StreamParams {
    CUtensorMap map_codes;              // [V, d / 2] bytes, box {64, 32}, 64-byte swizzle
    const __nv_bfloat16* hidden;
    const unsigned short* scales;       // bf16 bits
    const unsigned char* zeros;         // or nullptr: 8
    int rows, V, d, groups;             // groups = d / G
    int tiles;
    int ring;                           // pieces in flight per warp
    int vectors;                        // groups a multiple of eight, scales and zero points aligned for vector loads
    uint32_t exponent;                  // w4::kExponent
    int32_t* status;
    void* out;
};

// The first of a group's products: nothing to add to.
__device__ __forceinline__ void mma_bf16_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}

// The codes a lane takes of one row of a piece, words 0..3.  Lane t of a quad takes, of every group of G elements, G/4
// consecutive ones, so that each MMA stays inside one group.  `row` is the row's first byte; 16-byte chunk c of it lies at
// chunk c ^ sw.
template <int G>
__device__ __forceinline__ void read_codes(uint32_t row, int t, uint32_t sw, uint32_t (&w)[4])
{
    if (G == 128) {
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(row + ((t ^ sw) << 4)));
    } else if (G == 64) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
            asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[2 * j]), "=r"(w[2 * j + 1]) : "r"(row + (((2 * j + (t >> 1)) ^ sw) << 4) + (t & 1) * 8));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[j]) : "r"(row + ((j ^ sw) << 4) + t * 4));
    }
}

__device__ __forceinline__ void load_piece(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar)
{
    mbar_expect_tx(bar, kPieceBytes);
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

template <int G, int DT>
__global__ void __launch_bounds__(kThreadsS, 1) w4_stream_kernel(const __grid_constant__ StreamParams p)
{
    extern __shared__ uint4 smem_w4[];
    __shared__ __align__(8) uint64_t barriers[kWarpsS * kMaxRing];
    __shared__ int gave_up;
    constexpr int GPC = kChunk / G;             // groups per chunk
    const int lane = threadIdx.x & 31, warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
    const int g = lane >> 2, t = lane & 3;
    const uint32_t sw = static_cast<uint32_t>(g) >> 1;
    const int chunks = (p.d + kChunk - 1) / kChunk;

    // shared memory: the rings (1024-byte aligned), the scale tables, the hidden rows, the sums of a warp's first tile; those of
    // its last tile go to its ring, which is idle by then
    unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_w4) + 1023) & ~static_cast<uintptr_t>(1023));
    uint32_t* table = reinterpret_cast<uint32_t*>(base + static_cast<size_t>(kWarpsS) * p.ring * kPieceBytes) + warp * kTableWords;
    uint4* hidden = reinterpret_cast<uint4*>(base + static_cast<size_t>(kWarpsS) * (p.ring * kPieceBytes + kTableWords * 4));
    float* joined = reinterpret_cast<float*>(hidden + chunks * 4 * 32);             // [kWarpsS][kSums][32]
    auto sums_of = [&](int w, bool first) {
        return first ? joined + w * (kSums * 32) : reinterpret_cast<float*>(base + static_cast<size_t>(w) * p.ring * kPieceBytes);
    };
    const uint32_t my_ring = smem_addr(base) + warp * p.ring * kPieceBytes;
    const uint32_t bars = smem_addr(barriers) + warp * kMaxRing * 8u;

    // tiles [t_first, t_first + n_tiles) are this CTA's, pieces [share(w), share(w + 1)) of them warp w's
    const int each = p.tiles / static_cast<int>(gridDim.x), more = p.tiles % static_cast<int>(gridDim.x), cta = blockIdx.x;
    const int t_first = each * cta + min(cta, more), n_tiles = each + (cta < more ? 1 : 0);
    const int pieces = n_tiles * chunks;        // at most 2^31 / 32 tiles x 64 chunks over all CTAs: 16 shares of one's fit 31 bits
    auto share = [&](int w) { return pieces * w / kWarpsS; };
    const int s_first = share(warp), s_end = share(warp + 1);
    const int tile_first = t_first + s_first / chunks, c_start = s_first % chunks;

    if (lane == 0)
        for (int i = 0; i < p.ring; ++i) mbar_init(bars + 8u * i, 1);
    if (threadIdx.x == 0) gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    wait_for_stream();
    // the hidden rows' loads go out first: behind the rings' requests they would wait for megabytes of codes
    // (in row order, so that a warp asks for whole lines: 148 CTAs read the same ones)
    constexpr int kBatch = 8;
    const int row_vecs = p.d / 8, n_vecs = p.rows * row_vecs;
    uint4 staged[kBatch];
    auto load_hidden = [&](int i0) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (i0 + u * kThreadsS < n_vecs) staged[u] = reinterpret_cast<const uint4*>(p.hidden)[i0 + u * kThreadsS];
    };
    load_hidden(threadIdx.x);

    int ask_tile = tile_first, ask_c = c_start;
    PieceRing ring(p.ring, s_end - s_first);
    auto ask = [&]() {
        if (!ring.may_ask()) return;
        if (elect_one())
            load_piece(my_ring + ring.ask_at * kPieceBytes, &p.map_codes, ask_c * (kChunk / 2), ask_tile * kTileS, bars + 8u * ring.ask_at);
        __syncwarp();
        if (++ask_c == chunks) { ask_c = 0; ++ask_tile; }
        ring.asked();
    };
    for (int i = 0; i < p.ring; ++i) ask();

    // Scales and zero points, kTableGroups groups of the tile's 32 entries at a time: lane l loads those of entry l, as vectors
    // where the groups of a row are a multiple of eight (a lane that loads them group by group reads every 32-byte sector
    // sixteen times over), one table ahead of its use; a table word is the scale's bits above 128 + z as bf16.
    constexpr int kTableChunks = kTableGroups / GPC;
    const bool vectors = p.vectors != 0;
    uint4 raw_s = make_uint4(0, 0, 0, 0);
    uint2 raw_z = make_uint2(0, 0);
    auto load_raw = [&](int tile, int c) {
        if (!vectors) return;
        const size_t own = static_cast<size_t>(min(tile * kTileS + lane, p.V - 1)) * p.groups + c / kTableChunks * kTableGroups;
        raw_s = *reinterpret_cast<const uint4*>(p.scales + own);
        raw_z = p.zeros ? *reinterpret_cast<const uint2*>(p.zeros + own) : make_uint2(0x08080808u, 0x08080808u);
    };
    auto fill_table = [&](int tile, int c) {
        const int g0 = c / kTableChunks * kTableGroups;
        const size_t own = static_cast<size_t>(min(tile * kTileS + lane, p.V - 1)) * p.groups;
        __syncwarp();                           // the table before this one has been read
        if (vectors) {
            const uint32_t pair[4] = {raw_s.x, raw_s.y, raw_s.z, raw_s.w}, z[2] = {raw_z.x & 0x0f0f0f0fu, raw_z.y & 0x0f0f0f0fu};
#pragma unroll
            for (int i = 0; i < kTableGroups; ++i)          // scale above; below, 0x43 and the zero point's byte
                table[i * 32 + lane] = __byte_perm(__byte_perm(z[i >> 2], 0x43u, 0x0040u | (i & 3)), pair[i >> 1], (i & 1) ? 0x7610 : 0x5410);
        } else {
#pragma unroll
            for (int i = 0; i < kTableGroups; ++i) {
                const int group = min(g0 + i, p.groups - 1);
                table[i * 32 + lane] = static_cast<uint32_t>(p.scales[own + group]) << 16 | 0x4300u | (p.zeros ? p.zeros[own + group] & 15u : 8u);
            }
        }
        __syncwarp();
    };
    if (s_first < s_end) load_raw(tile_first, c_start);
    // The fragment order: place (chunk, word, lane) holds the eight elements of row g that multiply word `word` of the codes lane
    // (g, t) has.  Rows there are none of are zero, and so is what lies behind d.
    for (int i = threadIdx.x; i < chunks * 4 * 32; i += kThreadsS)
        if (((i & 31) >> 2) >= p.rows || (i >> 7) * kChunk + kChunk > p.d) hidden[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    for (int i0 = threadIdx.x; i0 < n_vecs;) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int i = i0 + u * kThreadsS;
            if (i >= n_vecs) break;
            const int n = i / row_vecs, j = i - n * row_vecs, c = j / (kChunk / 8), e = j % (kChunk / 8);
            const int word = G == 128 ? e % 4 : G == 64 ? e / 8 * 2 + e % 2 : e / 4, q = G == 128 ? e / 4 : G == 64 ? e % 8 / 2 : e % 4;
            hidden[(c * 4 + word) * 32 + n * 4 + q] = staged[u];
        }
        i0 += kBatch * kThreadsS;
        if (i0 < n_vecs) load_hidden(i0);
    }
    __syncthreads();

    // entry (m, half) * 8 + g, row 2 t + (i & 1)
    auto store = [&](int tile, int q, float x) {
        const int i = q & 3, m = q >> 2;
        const int v = tile * kTileS + m * 16 + (i >> 1) * 8 + g, n = 2 * t + (i & 1);
        if (v < p.V && n < p.rows) w4::store_logit<DT>(p.out, static_cast<size_t>(n) * p.V + v, x);
    };

    int tile = tile_first;
    bool first_tile = true, lost = false;
    for (int s = s_first; s < s_end; ++tile, first_tile = false) {
        const int c_first = first_tile ? c_start : 0, c_end = min(chunks, c_first + s_end - s);
        s += c_end - c_first;
        float sum[2][4];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[m][i] = 0.0f;

        for (int c = c_first; c < c_end; ++c) {
            if (c == c_first || c % kTableChunks == 0) {
                fill_table(tile, c);
                const int next = (c / kTableChunks + 1) * kTableChunks;
                if (next < c_end) load_raw(tile, next);
                else if (s < s_end) load_raw(tile + 1, 0);
            }
            // landed, if one lane has seen it
            if (!__any_sync(0xffffffffu, mbar_wait(bars + 8u * ring.at, ring.phase, &gave_up))) {
                if (lane == 0) {
                    if (p.status) atomicCAS(p.status, 0, static_cast<int>(POLYSPEC_ERR_TIMEOUT));
                    *reinterpret_cast<volatile int*>(&gave_up) = 1;
                }
                ring.give_up([&](int slot, uint32_t parity) {
                    for (uint32_t i = 0; i < kSpinLimitG && !mbar_try(bars + 8u * slot, parity); ++i) {}
                });
                lost = true;
                break;
            }
            __syncwarp();
            uint32_t x[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) read_codes<G>(my_ring + ring.at * kPieceBytes + (i * 8 + g) * 64, t, sw, x[i]);
            const uint4* hid = hidden + c * 4 * 32 + lane;
#pragma unroll
            for (int gi = 0; gi < GPC; ++gi) {
                if (GPC > 1 && c * GPC + gi >= p.groups) break;
                float sc[4];
                uint32_t z[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t y = table[(c % kTableChunks * GPC + gi) * 32 + i * 8 + g];
                    sc[i] = __uint_as_float(y & 0xffff0000u);
                    z[i] = __byte_perm(y, 0, 0x1010);
                }
                float acc[2][4];
#pragma unroll
                for (int wi = 0; wi < 4 / GPC; ++wi) {
                    const int word = gi * (4 / GPC) + wi;
                    const uint4 h = hid[word * 32];
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        uint32_t lo[4], hi[4];
                        w4::expand(x[2 * m][word], z[2 * m], p.exponent, lo);
                        w4::expand(x[2 * m + 1][word], z[2 * m + 1], p.exponent, hi);
                        const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]}, a1[4] = {lo[2], hi[2], lo[3], hi[3]};
                        if (wi == 0) mma_bf16_first(acc[m], a0, h.x, h.y);
                        else mma_bf16(acc[m], a0, h.x, h.y);
                        mma_bf16(acc[m], a1, h.z, h.w);
                    }
                }
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[m][i] = fmaf(sc[2 * m + (i >> 1)], acc[m][i], sum[m][i]);
            }
            __syncwarp();                       // every lane has read the piece
            ask();
            ring.next();
        }
        if (lost) break;
        const bool whole = c_end - c_first == chunks;
        float* mine = sums_of(warp, first_tile) + lane;
#pragma unroll
        for (int q = 0; q < kSums; ++q) {
            if (whole) store(tile, q, sum[q >> 2][q & 3]);
            else mine[q * 32] = sum[q >> 2][q & 3];
        }
    }
    __syncthreads();
    // tiles that several warps worked on: warp after warp in order
    for (int i = warp; i < n_tiles; i += kWarpsS) {
        const int lo = i * chunks, hi = lo + chunks;
        int w = 0;
        while (share(w + 1) <= lo) ++w;
        if (share(w) <= lo && share(w + 1) >= hi) continue;             // one warp's alone
        float total[kSums];
#pragma unroll
        for (int q = 0; q < kSums; ++q) total[q] = 0.0f;
        for (; w < kWarpsS && share(w) < hi; ++w) {
            if (share(w) == share(w + 1)) continue;     // nothing to do
            const float* theirs = sums_of(w, share(w) >= lo) + lane;        // the warp's first tile, if its share begins in it
#pragma unroll
            for (int q = 0; q < kSums; ++q) total[q] += theirs[q * 32];
        }
#pragma unroll
        for (int q = 0; q < kSums; ++q) store(t_first + i, q, total[q]);
    }
}

constexpr size_t kMaxSmem = 227 * 1024, kStaticRoom = 2048;
constexpr size_t kMaxDynamic = kMaxSmem - kStaticRoom;          // of any call

// Shared memory with `ring` pieces per warp; the largest ring that fits is used, and two pieces are the least.
size_t stream_smem(int d, int ring)
{
    const size_t chunks = (d + kChunk - 1) / kChunk;
    return 1024 + static_cast<size_t>(kWarpsS) * (ring * kPieceBytes + kTableWords * 4 + kSums * 32 * sizeof(float)) + chunks * 4 * 512;
}
int stream_ring(int d)
{
    int ring = kMaxRing;
    while (ring > 0 && stream_smem(d, ring) > kMaxDynamic) --ring;
    return ring;
}

std::mutex g_mutex;
EncodeTiledFn g_encode = nullptr;

// The tensor map of the codes.
bool encode_codes(StreamParams& p, const uint32_t* codes)
{
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(p.d / 2), static_cast<cuuint64_t>(p.V)}, pitch[1] = {static_cast<cuuint64_t>(p.d / 2)};
    const cuuint32_t box[2] = {kChunk / 2, kTileS}, one[2] = {1, 1};
    return g_encode(&p.map_codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint32_t*>(codes), dims, pitch, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int G, int DT>
cudaError_t launch_stream_t(StreamParams& p, const uint32_t* codes, int sms, cudaStream_t stream)
{
    const size_t smem = stream_smem(p.d, p.ring);
    // The limit belongs to the kernel, not to the call: always the most that any call needs, so that a call for a narrow head in one
    // host thread does not lower it between another thread's set-up and launch.
    cudaError_t e = cudaFuncSetAttribute(w4_stream_kernel<G, DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kMaxDynamic));
    if (e != cudaSuccess) return e;
    // behind the attribute: encoding is a driver call, which wants a context current in this host thread, and setting one binds it
    if (!encode_codes(p, codes)) return cudaErrorInvalidValue;
    return launch_early(w4_stream_kernel<G, DT>, dim3(static_cast<unsigned>(std::min(sms, p.tiles))), kThreadsS, smem, stream, p);
}

template <int G>
cudaError_t launch_stream_g(StreamParams& p, const uint32_t* codes, polyspec_dtype dt, int sms, cudaStream_t stream)
{
    return dt == POLYSPEC_F32 ? launch_stream_t<G, POLYSPEC_F32>(p, codes, sms, stream) : launch_stream_t<G, POLYSPEC_BF16>(p, codes, sms, stream);
}

cudaError_t launch_stream(const W4Problem& q, polyspec_dtype dt, int32_t* device_status, cudaStream_t stream)
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
    StreamParams p;
    p.hidden = static_cast<const __nv_bfloat16*>(q.hidden);
    p.scales = static_cast<const unsigned short*>(q.scales);
    p.zeros = q.zeros;
    p.rows = q.rows;
    p.V = q.V;
    p.d = q.d;
    p.groups = q.d / q.group;
    p.out = q.out;
    p.exponent = w4::kExponent;
    p.status = device_status;
    p.tiles = (q.V + kTileS - 1) / kTileS;
    p.ring = stream_ring(q.d);
    p.vectors = p.groups % kTableGroups == 0 && (reinterpret_cast<uintptr_t>(q.scales) & 15u) == 0 && (reinterpret_cast<uintptr_t>(q.zeros) & 7u) == 0;
    switch (q.group) {
        case 128: return launch_stream_g<128>(p, q.codes, dt, sms, stream);
        case 64: return launch_stream_g<64>(p, q.codes, dt, sms, stream);
        default: return launch_stream_g<32>(p, q.codes, dt, sms, stream);
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
        (reinterpret_cast<uintptr_t>(logits) & 15u) != 0 || (reinterpret_cast<uintptr_t>(scales) & 1u) != 0 || !aligned4(device_status))
        return POLYSPEC_ERR_INVALID_ARG;
    if (group != 32 && group != 64 && group != 128) return POLYSPEC_ERR_UNSUPPORTED;
    if (d % group != 0 || V > 0x7fffffff - 1024 || rows > 0x7fffffff - 1024) return POLYSPEC_ERR_UNSUPPORTED;     // a tile past the end counts on
    if (static_cast<long long>((V + 127) / 128) * ((rows + 15LL) / 16) > 0x70000000LL) return POLYSPEC_ERR_UNSUPPORTED;      // work items
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
    if (rows > kStreamRows || stream_ring(d) < 2)
        return cuda_failed(launch_w4_tensor(q, dt, device_status, s)) ? POLYSPEC_ERR_CUDA : POLYSPEC_OK;
    return cuda_failed(launch_stream(q, dt, device_status, s)) ? POLYSPEC_ERR_CUDA : POLYSPEC_OK;
}

}  // extern "C"
