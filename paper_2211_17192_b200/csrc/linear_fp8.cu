// A linear layer in e4m3 with its epilogue in the kernel:
//   z[r][n] = x_scale[r] * w_scale[n] * sum_k xc[r][k] * wc[n][k] (+ bias[n]),   y = act(z) (+ residual).
//
// The weights take the M side of the MMA: a CTA owns 128 rows of W and streams them by TMA (128-byte swizzle, k-blocks of 128
// codes) through a ring of stages into tcgen05.mma (kind::f8f6f4, M = 128, N = the rows of x, K = 32); the accumulator is fp32 in
// tensor memory, products of codes are exact.  At few rows the call is bound by the weights' bytes, so all SMs have to stream:
// the CTAs of a cluster share a tile's k-blocks and exchange their sums through distributed shared memory, each finishing a share
// of the tile's elements in a fixed order - one launch, no workspace, the same bits every time.
//
// Gated activations need rows f and f + n_out of W side by side: the tile's 128 rows are fetched as four boxes of 32 - 16 gate
// rows, then the same 16 up rows (a tensor map with gate / up as an axis of its own) - so that both halves of an output lie in
// one warp's lanes, 16 apart.
//
// Every wait on an mbarrier is bounded; on expiry the kernel records an error code, waits (with a limit) for its copies and
// leaves, tensor memory freed.
#include <algorithm>

#include "fp8_util.cuh"
#include "tc_util.cuh"

namespace spec {
namespace {

using namespace tc;

constexpr int kBlockK = 128;   // codes of a k-block: one 128-byte swizzle row
constexpr int kCodesK = 32;    // K of one tcgen05.mma.kind::f8f6f4
constexpr int kThreads = 192;  // producer warp, MMA warp, four epilogue warps
constexpr int kMaxStages = 12;
constexpr int kDrainLimit = 1 << 14;
constexpr int kTileBytes = kTileM * kBlockK;

__device__ int g_linear_error;  // first device-side time-out (0 = none)

enum { kActNone = 0, kActGelu = 1, kActSilu = 2, kActGatedGelu = 3, kActSwiglu = 4 };

struct LinearArgs {
    const float *x_scales, *w_scales, *bias;
    const void* residual;
    void* y;
    int rows, n_out, k_blocks, act, tokens /* rows of x per tile: the MMA's N */, stages;
    uint32_t limit;  // of every wait
    int drill;       // nothing is requested, so that the waits run out (spec_timeout_drill)
    int tiles, token_tiles;  // wide kernel: tiles of 256 rows of W by `tokens` rows of x, those of x neighbours
};

// e4m3 x e4m3 -> fp32, both operands K-major.
__host__ __device__ constexpr uint32_t instr_desc_e4m3(int m, int n) {
    return (1u << 4) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}
__device__ __forceinline__ void mma_e4m3(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t"
        "}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* map, int x, int y, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
        ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void store_peer(uint32_t here, uint32_t rank, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    uint32_t there;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here), "r"(rank));
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(there), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

// The columns that a CTA of a cluster finishes (in fours, as they are exchanged), and the place of these from each of its CTAs.
__host__ __device__ __forceinline__ int columns_each(int columns, int splits) { return ((columns + 3) / 4 + splits - 1) / splits * 4; }
__host__ __device__ __forceinline__ int exchange_bytes(int tokens, int splits) { return splits > 1 ? splits * columns_each(tokens, splits) * kTileM * 4 : 0; }

// What a lane of an epilogue warp knows of its accumulator lane (row of W), constant over a tile.
struct LaneColumn {
    int column;  // of y, -1: none (gated: lanes 16..31, which only hand their value over)
    float scale, bias;
};
__device__ __forceinline__ LaneColumn lane_column(const LinearArgs& a, int tile, int quarter, int lane) {
    const bool gated = a.act >= kActGatedGelu;
    LaneColumn c;
    const int f = gated ? tile * (kTileM / 2) + quarter * 16 + (lane & 15) : tile * kTileM + quarter * 32 + lane;
    const bool in = f < a.n_out;
    const int row = gated && lane >= 16 ? f + a.n_out : f;
    c.scale = in ? a.w_scales[row] : 0.0f;
    c.bias = in && a.bias ? a.bias[row] : 0.0f;
    c.column = in && !(gated && lane >= 16) ? f : -1;
    return c;
}
// x * sigmoid(s): with s = x this is silu, with s = 2 sqrt(2 / pi) (x + 0.044715 x^3) it is x (1 + tanh(s / 2)) / 2, the tanh form of
// gelu.  From the hardware's 2^x and reciprocal: off by less than 2^-21 |x|.
__device__ __forceinline__ float gate(float x, float s) { return __fdividef(x, 1.0f + __expf(-s)); }
__device__ __forceinline__ float gelu_argument(float x) { return x * fmaf(0.0713548162726f * x, x, 1.5957691216057f); }

// The residual of COLS neighbouring accumulator columns (rows r0 .. of x, `count` of them) of a warp's 32 rows of W.
template <typename T, int COLS>
__device__ __forceinline__ void load_residual(const LinearArgs& a, const LaneColumn& c, int r0, int count, T (&add)[COLS]) {
    if (!a.residual) return;
    const T* from = static_cast<const T*>(a.residual) + static_cast<size_t>(r0) * a.n_out + (c.column < 0 ? 0 : c.column);
#pragma unroll
    for (int i = 0; i < COLS; ++i) add[i] = i < count && c.column >= 0 ? from[static_cast<size_t>(i) * a.n_out] : from_float<T>(0.0f);
}
// These columns to y.  Everything is loaded before anything is stored: the loads are in flight together (one column after the
// other took 0.2 to 0.4 us each).
template <typename T, int COLS>
__device__ __forceinline__ void finish(const LinearArgs& a, const LaneColumn& c, const float* scales /* of these rows of x */, int r0, int count,
                                       float (&z)[COLS], const T (&add)[COLS]) {
    float x_scale[COLS];
    T* y = static_cast<T*>(a.y) + static_cast<size_t>(r0) * a.n_out + (c.column < 0 ? 0 : c.column);
#pragma unroll
    for (int i = 0; i < COLS; ++i) x_scale[i] = i < count ? scales[i] : 0.0f;
#pragma unroll
    for (int i = 0; i < COLS; ++i) z[i] = fmaf(z[i] * x_scale[i], c.scale, c.bias);
    if (a.act == kActGelu) {
#pragma unroll
        for (int i = 0; i < COLS; ++i) z[i] = gate(z[i], gelu_argument(z[i]));
    } else if (a.act == kActSilu) {
#pragma unroll
        for (int i = 0; i < COLS; ++i) z[i] = gate(z[i], z[i]);
    } else if (a.act >= kActGatedGelu) {
        // (both halves of the warp go through the function, so that the up half's lanes need no branch of their own)
        const bool gelu = a.act == kActGatedGelu;
#pragma unroll
        for (int i = 0; i < COLS; ++i) {
            const float up = __shfl_xor_sync(kFullMask, z[i], 16);
            z[i] = gate(z[i], gelu ? gelu_argument(z[i]) : z[i]) * up;
        }
    }
    if (c.column < 0) return;
    if (a.residual) {
#pragma unroll
        for (int i = 0; i < COLS; ++i) z[i] += to_float(add[i]);
    }
#pragma unroll
    for (int i = 0; i < COLS; ++i)
        if (i < count) y[static_cast<size_t>(i) * a.n_out] = from_float<T>(z[i]);
}

// grid = (tiles of 128 rows of W x CTAs of a cluster, tiles of x), clusters along x, block = kThreads.
template <typename T>
__global__ void __launch_bounds__(kThreads)
linear_fp8_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ LinearArgs a) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int stage_bytes = kTileBytes + a.tokens * kBlockK;
    float* exchange = reinterpret_cast<float*>(smem + a.stages * stage_bytes);  // clusters of two and more: exchange_bytes() of them
    const uint32_t splits = cluster_size(), rank = cluster_rank();
    uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + a.stages * stage_bytes + exchange_bytes(a.tokens, splits));
    uint64_t* empty_bar = full_bar + kMaxStages;
    uint64_t* acc_bar = empty_bar + kMaxStages;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_bar + 1);

    const int warp = __shfl_sync(kFullMask, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;  // (uniform for the compiler)
    const int tile = blockIdx.x / splits, row0 = blockIdx.y * a.tokens;
    const int kb0 = static_cast<int>(static_cast<long long>(a.k_blocks) * rank / splits);
    const int kb1 = static_cast<int>(static_cast<long long>(a.k_blocks) * (rank + 1) / splits);
    const int tmem_cols = a.tokens <= 32 ? 32 : a.tokens <= 64 ? 64 : a.tokens <= 128 ? 128 : 256;

    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(&full_bar[s], 1);
            mbar_init(&empty_bar[s], 1);
        }
        mbar_init(acc_bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(tmem_cols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (splits > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // (this CTA's exchange may be written)
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *tmem_slot;
    bool ok = true;
    pdl_wait();

    if (warp == 0) {
        const bool leader = elect_one();
        const bool gated = a.act >= kActGatedGelu;
        int s = 0, use = 0;
        for (int kb = a.drill ? kb1 : kb0; kb < kb1; ++kb) {
            if (use > 0 && !mbar_wait_warp(&empty_bar[s], (use - 1) & 1, a.limit)) { ok = false; break; }
            if (leader) {
                uint8_t* stage = smem + s * stage_bytes;
                mbar_expect_tx(&full_bar[s], stage_bytes);
                if (gated) {
                    for (int i = 0; i < 4; ++i) tma_load_3d(stage + i * (kTileBytes / 4), &map_w, kb * kBlockK, tile * (kTileM / 2) + 16 * i, 0, &full_bar[s]);
                } else {
                    tma_load_3d(stage, &map_w, kb * kBlockK, tile * kTileM, 0, &full_bar[s]);
                }
                tma_load_2d(stage + kTileBytes, &map_x, kb * kBlockK, row0, &full_bar[s]);
            }
            if (++s == a.stages) { s = 0; ++use; }
        }
        if (!ok)  // nothing may still be on its way when the CTA leaves
            for (int i = 0; i < a.stages; ++i) {
                mbar_wait(&full_bar[i], 0, kDrainLimit);
                mbar_wait(&full_bar[i], 1, kDrainLimit);
            }
    } else if (warp == 1) {
        const bool leader = elect_one();
        const uint32_t idesc = instr_desc_e4m3(kTileM, a.tokens);
        const uint32_t base = smem_u32(smem);
        int s = 0, use = 0;
        for (int kb = kb0; kb < kb1; ++kb) {
            if (!mbar_wait_warp(&full_bar[s], use & 1, a.limit)) { ok = false; break; }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint64_t w_desc = smem_desc_sw128(base + s * stage_bytes), x_desc = smem_desc_sw128(base + s * stage_bytes + kTileBytes);
            if (leader) {
#pragma unroll
                for (int k = 0; k < kBlockK / kCodesK; ++k)
                    mma_e4m3(tmem, w_desc + ((k * kCodesK) >> 4), x_desc + ((k * kCodesK) >> 4), idesc, kb > kb0 || k > 0 ? 1u : 0u);
                mma_commit(&empty_bar[s]);
            }
            __syncwarp();
            if (++s == a.stages) { s = 0; ++use; }
        }
        if (ok && leader) mma_commit(acc_bar);
        __syncwarp();
    }
    __syncwarp();
    // The next kernel is let in when this CTA's copies and products have been asked for.  At the top it takes the places of CTAs that
    // leave, an SM here and there, and its own stream is then as uneven (3 x 4096 x 22016, call after call: 18.7 us, 16.8 so).
    if (warp < 2) pdl_trigger();
    const int quarter = warp & 3;  // accumulator lanes 32 quarter .. + 31 are what warps 2..5 may read
    const bool reader = warp >= 2;  // (of sums: every CTA has a k-block, launch_small)
    const int valid = min(a.tokens, a.rows - row0);
    LaneColumn column{};
    if (reader) {
        column = lane_column(a, tile, quarter, lane);
        if (!mbar_wait_warp(acc_bar, 0, a.limit)) ok = false;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    }
    const uint32_t acc = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    if (splits == 1) {
        if (reader && ok)
            for (int c0 = 0; c0 < valid; c0 += 16) {
                float z[16];
                T add[16];
                load_residual<T, 16>(a, column, row0 + c0, valid - c0, add);
                tmem_ld16(acc + c0, reinterpret_cast<uint32_t(&)[16]>(z));
                tmem_ld_wait();
                finish<T, 16>(a, column, a.x_scales + row0 + c0, row0 + c0, valid - c0, z, add);
            }
    } else {
        // CTA r finishes columns [r each, (r + 1) each): the others' sums of these lie in its exchange as [CTA][four columns][128][4]
        const int each = columns_each(valid, splits);
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // everyone is there
        if (reader && ok)
            for (int c0 = 0; c0 < valid; c0 += 16) {
                uint32_t v[16];
                tmem_ld16(acc + c0, v);
                tmem_ld_wait();
                int to = c0 / each, within = c0 - to * each;
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    if (c0 + i < valid) {
                        store_peer(smem_u32(exchange + (rank * each + within) * kTileM + (quarter * 32 + lane) * 4), to, v[i], v[i + 1], v[i + 2], v[i + 3]);
                        if ((within += 4) == each) { within = 0; ++to; }
                    }
            }
        cluster_sync_all();
        if (reader && ok) {
            const int c1 = min(valid, static_cast<int>(rank + 1) * each);
            for (int c0 = rank * each; c0 < c1; c0 += 8) {
                float z[8];
                T add[8];
                load_residual<T, 8>(a, column, row0 + c0, c1 - c0, add);
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = 0.0f;
                for (uint32_t p = 0; p < splits; ++p) {
                    const float4* from = reinterpret_cast<const float4*>(exchange + (p * each + c0 - rank * each) * kTileM) + quarter * 32 + lane;
#pragma unroll
                    for (int i = 0; i < 8; i += 4) {
                        if (c0 + i >= c1) continue;
                        const float4 v = from[i / 4 * kTileM];
                        z[i] += v.x;
                        z[i + 1] += v.y;
                        z[i + 2] += v.z;
                        z[i + 3] += v.w;
                    }
                }
                finish<T, 8>(a, column, a.x_scales + row0 + c0, row0 + c0, c1 - c0, z, add);
            }
        }
    }
    if (!ok) atomicCAS(&g_linear_error, 0, 1 + warp);
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols));
    }
}

// A matrix of codes [planes][rows][k] in boxes of [box_planes][box_rows][128], 128-byte swizzle on the way in, zeros past its edges.
int codes_map(const void* base, int planes, int rows, int k, int box_planes, int box_rows, CUtensorMap* out) {
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(k), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(planes)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(k), static_cast<cuuint64_t>(k) * rows};
    const cuuint32_t box[3] = {kBlockK, static_cast<cuuint32_t>(box_rows), static_cast<cuuint32_t>(box_planes)};
    return encode_map(CU_TENSOR_MAP_DATA_TYPE_UINT8, box_planes ? 3 : 2, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B, out);
}

// ---- many rows ----
// A pair of CTAs on neighbouring SMs (cta_group::2, M = 256) has 256 rows of W by up to 256 of x: each CTA fetches 128 rows of W and
// half of the rows of x, so a byte of either is used twice as often as by a CTA alone.  Persistent, one CTA per SM: a warp feeds
// the ring, a warp of the even CTA issues the MMAs, eight warps drain the accumulators, of which there are two: the next tile is
// multiplied while the last is finished and written.
constexpr int kEpilogueWarps = 8;
constexpr int kWideRows = 256;  // most rows of x per tile
constexpr int kWideThreads = 32 * (2 + kEpilogueWarps);


__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// Boxes into this CTA's shared memory, their bytes counted on `bar` (an address in either CTA of the pair).
__device__ __forceinline__ void tma_pair_2d(void* dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
        ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tma_pair_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t"
        "}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// One arrival on the barrier at this offset in both CTAs once every MMA issued so far has finished.
__device__ __forceinline__ void commit_pair(uint64_t* bar) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
        ::"r"(smem_u32(bar)), "h"(static_cast<uint16_t>(3))
        : "memory");
}
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// grid = 2 * pairs, clusters of 2, block = kWideThreads.
template <typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kWideThreads, 1)
linear_fp8_wide_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ LinearArgs a) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ float row_scales[kEpilogueWarps][kWideRows / 2];
    const int half = a.tokens / 2, stage_bytes = kTileBytes + half * kBlockK;
    uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + a.stages * stage_bytes);  // (the even CTA's count both CTAs' bytes)
    uint64_t* empty_bar = full_bar + kMaxStages;
    uint64_t* acc_full = empty_bar + kMaxStages;  // [2]
    uint64_t* acc_empty = acc_full + 2;           // [2], the even CTA's count both CTAs' epilogue warps
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);

    const int warp = __shfl_sync(kFullMask, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(&full_bar[s], 1);
            mbar_init(&empty_bar[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&acc_full[i], 1);
            mbar_init(&acc_empty[i], 2 * kEpilogueWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync_all();  // both CTAs' barriers exist
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *tmem_slot;
    bool ok = true;
    pdl_wait();
    pdl_trigger();

    if (warp == 0) {
        const bool leader = elect_one(), gated = a.act >= kActGatedGelu;
        const uint32_t full0 = in_cta(smem_u32(full_bar), 0);
        int s = 0, use = 0;
        for (int tile = a.drill ? a.tiles : pair; ok && tile < a.tiles; tile += pairs) {
            const int w_tile = (tile / a.token_tiles) * 2 + static_cast<int>(rank);  // of 128 rows
            const int row0 = (tile % a.token_tiles) * a.tokens + static_cast<int>(rank) * half;
            for (int kb = 0; kb < a.k_blocks; ++kb) {
                if (use > 0 && !mbar_wait_warp(&empty_bar[s], (use - 1) & 1, a.limit)) { ok = false; break; }
                if (leader) {
                    uint8_t* stage = smem + s * stage_bytes;
                    if (rank == 0) mbar_expect_tx(&full_bar[s], 2 * stage_bytes);
                    if (gated) {
                        for (int i = 0; i < 4; ++i) tma_pair_3d(stage + i * (kTileBytes / 4), &map_w, kb * kBlockK, w_tile * (kTileM / 2) + 16 * i, 0, full0 + 8 * s);
                    } else {
                        tma_pair_3d(stage, &map_w, kb * kBlockK, w_tile * kTileM, 0, full0 + 8 * s);
                    }
                    tma_pair_2d(stage + kTileBytes, &map_x, kb * kBlockK, row0, full0 + 8 * s);
                }
                if (++s == a.stages) { s = 0; ++use; }
            }
        }
        if (!ok && rank == 0)  // nothing may still be on its way when the CTAs leave
            for (int i = 0; i < a.stages; ++i) {
                mbar_wait(&full_bar[i], 0, kDrainLimit);
                mbar_wait(&full_bar[i], 1, kDrainLimit);
            }
    } else if (warp == 1) {
        if (rank == 0) {
            const bool leader = elect_one();
            const uint32_t idesc = instr_desc_e4m3(2 * kTileM, a.tokens);
            const uint32_t base = smem_u32(smem);
            int s = 0, use = 0;     // stage, and how often the ring has gone round
            int buf = 0, turn = 0;  // accumulator, and how often both have had their turn
            for (int tile = pair; ok && tile < a.tiles; tile += pairs) {
                if (turn > 0 && !mbar_wait_warp(&acc_empty[buf], (turn - 1) & 1, a.limit)) { ok = false; break; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                for (int kb = 0; kb < a.k_blocks; ++kb) {
                    if (!mbar_wait_warp(&full_bar[s], use & 1, a.limit)) { ok = false; break; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t w_desc = smem_desc_sw128(base + s * stage_bytes), x_desc = smem_desc_sw128(base + s * stage_bytes + kTileBytes);
                    if (leader) {
#pragma unroll
                        for (int k = 0; k < kBlockK / kCodesK; ++k)
                            mma_pair(tmem + buf * 256, w_desc + ((k * kCodesK) >> 4), x_desc + ((k * kCodesK) >> 4), idesc, kb > 0 || k > 0 ? 1u : 0u);
                        commit_pair(&empty_bar[s]);
                    }
                    __syncwarp();
                    if (++s == a.stages) { s = 0; ++use; }
                }
                if (ok && leader) commit_pair(&acc_full[buf]);
                __syncwarp();
                if (++buf == 2) { buf = 0; ++turn; }
            }
        }
    } else {
        const int quarter = warp & 3, first_col = ((warp - 2) >> 2) * 16;
        float* scales = row_scales[warp - 2];
        int buf = 0, turn = 0;
        for (int tile = pair; tile < a.tiles; tile += pairs) {
            const LaneColumn column = lane_column(a, (tile / a.token_tiles) * 2 + static_cast<int>(rank), quarter, lane);
            const int row0 = (tile % a.token_tiles) * a.tokens, valid = min(a.tokens, a.rows - row0);
            // The loads of the epilogue wait behind the ring's: the scales of the warp's rows are fetched once per tile, while it is
            // multiplied, and the residual sixteen columns ahead (2048 x 11008 x 4096 with an fp32 residual 79 -> 71 us, 2048 x 4096 x 4096
            // 46 -> 41; two or three times sixteen ahead: no better).
            __syncwarp();
#pragma unroll
            for (int i = lane; i < kWideRows / 2; i += 32) {
                const int r = first_col + i / 16 * 32 + i % 16;
                scales[i] = r < valid ? a.x_scales[row0 + r] : 0.0f;
            }
            __syncwarp();
            T coming[16];
            load_residual<T, 16>(a, column, row0 + first_col, valid - first_col, coming);
            if (!mbar_wait_warp(&acc_full[buf], turn & 1, a.limit)) { ok = false; break; }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t acc = tmem + buf * 256 + (static_cast<uint32_t>(quarter * 32) << 16);
            for (int c0 = first_col; c0 < valid; c0 += 32) {
                float z[16];
                T add[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) add[i] = coming[i];
                load_residual<T, 16>(a, column, row0 + c0 + 32, valid - c0 - 32, coming);
                tmem_ld16(acc + c0, reinterpret_cast<uint32_t(&)[16]>(z));
                tmem_ld_wait();
                finish<T, 16>(a, column, scales + (c0 - first_col) / 2, row0 + c0, valid - c0, z, add);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) arrive_at(in_cta(smem_u32(&acc_empty[buf]), 0));
            if (++buf == 2) { buf = 0; ++turn; }
        }
    }
    if (!ok) atomicCAS(&g_linear_error, 0, 16 + warp);
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync_all();  // nobody leaves while its peer may still signal or read its shared memory
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
    }
}

template <typename T>
int launch_small(const void* x, const void* w, int k, LinearArgs a, cudaStream_t stream) {
    const bool gated = a.act >= kActGatedGelu;
    const int per_tile = gated ? kTileM / 2 : kTileM, tiles = (a.n_out + per_tile - 1) / per_tile;
    a.k_blocks = (k + kBlockK - 1) / kBlockK;
    int token_tiles = (a.rows + 127) / 128;
    a.tokens = ((a.rows + token_tiles - 1) / token_tiles + 15) / 16 * 16;
    token_tiles = (a.rows + a.tokens - 1) / a.tokens;
    // One wave, all CTAs resident (a second wave starts behind the first one's epilogue: 4096 x 6144, three rows, three CTAs to a
    // cluster and one to an SM 11.8 us, since such clusters do not fill the SMs; four, two to an SM 7.6).  Up to 64 columns two
    // CTAs share an SM, and clusters grow while there are at most 200 CTAs; above, the exchange takes too much room, and clusters
    // of at most four can be placed as long as there are 128 CTAs (of eight, some wait: 112 x 2000 x 2000 14.6 us, 9 with four).
    const bool paired = a.tokens <= 64;
    int splits = 1;
    for (int s = 2; s <= (paired ? 8 : 4); ++s)
        if (tiles * token_tiles * s <= (paired ? 200 : 128) && 2 * s <= a.k_blocks) splits = s;  // (two k-blocks to a CTA at least)
    const int stage_bytes = kTileBytes + a.tokens * kBlockK, exchange = exchange_bytes(a.tokens, splits);
    const int room = (paired ? 113 : 227) * 1024 - 1024 - 512 - exchange;
    a.stages = std::min({kMaxStages, room / stage_bytes, std::max(2, (a.k_blocks + splits - 1) / splits)});
    CUtensorMap mw, mx;
    int status = codes_map(w, gated ? 2 : 1, a.n_out, k, gated ? 2 : 1, gated ? 16 : kTileM, &mw);
    if (status == SPEC_OK) status = codes_map(x, 1, a.rows, k, 0, a.tokens, &mx);
    if (status != SPEC_OK) return status;
    static std::atomic<unsigned long long> configured{0};
    status = allow_shared_memory(configured, linear_fp8_kernel<T>, 227 * 1024);
    if (status != SPEC_OK) return status;
    // 48 KB and more: at most four CTAs to an SM, whose tensor memory (128 columns each) then all fits.  A CTA that had to wait for
    // columns while its cluster waits for it could wait for ever.
    const int smem = std::max(48 * 1024, a.stages * stage_bytes + exchange + 1024 + 512);
    return launch_cluster(linear_fp8_kernel<T>, splits, dim3(tiles * splits, token_tiles), dim3(kThreads), smem, stream, mw, mx, a);
}

template <typename T>
int launch_wide(const void* x, const void* w, int k, LinearArgs a, cudaStream_t stream) {
    const bool gated = a.act >= kActGatedGelu;
    constexpr int kPairs = 74;  // one CTA per SM
    const int per_tile = gated ? kTileM : 2 * kTileM, w_tiles = (a.n_out + per_tile - 1) / per_tile;
    a.k_blocks = (k + kBlockK - 1) / kBlockK;
    // Rows of x per tile: as many as make the busiest pair's tiles the shortest, where a tile costs its rows and 60 more (a k-block brings
    // 128 rows of W to a CTA however few rows of x meet them).  4096 x 22016 gated: 224 rows in two tiles of 112, three rounds, 27.8 us, in
    // one, two rounds, 31.7; 256 rows in two of 128, three rounds, 28.6, in four of 64, five rounds, 37.6, in one, two rounds, 34.5.
    long long best = 0;
    for (int tokens = 256; tokens >= 64; tokens -= 16) {
        const int token_tiles = (a.rows + tokens - 1) / tokens;
        const long long rounds = (static_cast<long long>(w_tiles) * token_tiles + kPairs - 1) / kPairs, cost = rounds * (tokens + 60);
        if (best == 0 || cost < best) {
            best = cost;
            a.tokens = tokens;
            a.token_tiles = token_tiles;
        }
    }
    a.tiles = w_tiles * a.token_tiles;
    const int stage_bytes = kTileBytes + a.tokens / 2 * kBlockK;
    a.stages = std::min(kMaxStages, (227 * 1024 - 1024 - 512 - kEpilogueWarps * kWideRows * 2) / stage_bytes);
    CUtensorMap mw, mx;
    int status = codes_map(w, gated ? 2 : 1, a.n_out, k, gated ? 2 : 1, gated ? 16 : kTileM, &mw);
    if (status == SPEC_OK) status = codes_map(x, 1, a.rows, k, 0, a.tokens / 2, &mx);
    if (status != SPEC_OK) return status;
    static std::atomic<unsigned long long> configured{0};
    status = allow_shared_memory(configured, linear_fp8_wide_kernel<T>, 227 * 1024 - kEpilogueWarps * kWideRows * 2);
    if (status != SPEC_OK) return status;
    return launch_pdl(linear_fp8_wide_kernel<T>, dim3(2 * std::min(kPairs, a.tiles)), dim3(kWideThreads), a.stages * stage_bytes + 1024 + 512, stream, mw, mx, a);
}

}  // namespace

// A cluster of two, or a pair of CTAs, on one tile with nothing requested; `base`: 4 KB of numbers, of which the scales are read.
int launch_linear_fp8_drill(void* base, bool wide, uint32_t limit, cudaStream_t stream) {
    LinearArgs a{};
    a.x_scales = a.w_scales = static_cast<const float*>(base);
    a.y = base;  // (not written)
    a.rows = wide ? 64 : 3;
    a.n_out = wide ? 256 : 128;
    a.limit = limit;
    a.drill = 1;
    return wide ? launch_wide<float>(base, base, 4 * kBlockK, a, stream) : launch_small<float>(base, base, 4 * kBlockK, a, stream);
}

int linear_fp8_take_error() {
    int v = 0, zero = 0;
    if (cudaMemcpyFromSymbol(&v, g_linear_error, sizeof(int)) != cudaSuccess) return -1;
    if (v) cudaMemcpyToSymbol(g_linear_error, &zero, sizeof(int));
    return v;
}

}  // namespace spec

extern "C" int spec_linear_fp8(const void* x, const float* x_scales, const void* w, const float* w_scales, const float* bias, int act,
                               const void* residual, void* y, int y_dtype, int rows, int n_out, int k, void* stream) {
    using namespace spec;
    if (rows < 0 || n_out < 1 || k < 16 || k % 16 || n_out > (1 << 28) || rows > (1 << 22)) return fail(SPEC_ERR_BAD_ARG, "spec_linear_fp8: rows=%d n_out=%d k=%d (k must be a multiple of 16)", rows, n_out, k);
    if (act < 0 || act > kActSwiglu) return fail(SPEC_ERR_BAD_ARG, "spec_linear_fp8: act %d", act);
    if (!float_dtype(y_dtype)) return fail(SPEC_ERR_BAD_ARG, "spec_linear_fp8: y_dtype %d", y_dtype);
    if (rows == 0) return SPEC_OK;
    if (!x || !x_scales || !w || !w_scales || !y) return fail(SPEC_ERR_BAD_ARG, "spec_linear_fp8: null pointer");
    if (!aligned_to(x, 16) || !aligned_to(w, 16)) return fail(SPEC_ERR_BAD_ARG, "spec_linear_fp8: codes have to start on 16 bytes");
    if (!aligned_to(x_scales, 4) || !aligned_to(w_scales, 4) || !aligned_to(bias, 4) || !aligned_to(residual, dtype_bytes(y_dtype)) || !aligned_to(y, dtype_bytes(y_dtype)))
        return fail(SPEC_ERR_BAD_ARG, "spec_linear_fp8: a pointer is not aligned to its elements");
    LinearArgs a{};
    a.x_scales = x_scales;
    a.w_scales = w_scales;
    a.bias = bias;
    a.residual = residual;
    a.y = y;
    a.rows = rows;
    a.n_out = n_out;
    a.act = act;
    a.limit = tc::kSpinLimit;
    // CTA pairs fetch half as much per product, clusters that share a tile's k-blocks use more SMs where tiles are few.  11008 x 4096:
    // 192 rows 18.0 us in clusters and 20.2 in pairs, 256 rows 20.2 and 20.1; 4096 x 4096: 96 rows 9.3 and 10.4, 192 rows 11.9 and
    // 10.8; 768 x 2304: 80 rows 6.1 and 4.9; 4096 x 6144 (48 tiles): 64 rows 10.2 and 10.6, 80 rows 11.3 and 10.7.
    const int tiles = (n_out + (act >= kActGatedGelu ? 63 : 127)) / (act >= kActGatedGelu ? 64 : 128), k_blocks = (k + kBlockK - 1) / kBlockK;
    const bool wide = rows > 64 && (tiles > 37 || rows > 64 + k_blocks + k_blocks / 2);
    const auto go = [&](auto type) {
        using T = decltype(type);
        return wide ? launch_wide<T>(x, w, k, a, static_cast<cudaStream_t>(stream)) : launch_small<T>(x, w, k, a, static_cast<cudaStream_t>(stream));
    };
    return y_dtype == SPEC_DTYPE_FP32 ? go(float{}) : y_dtype == SPEC_DTYPE_BF16 ? go(__nv_bfloat16{}) : go(__half{});
}
