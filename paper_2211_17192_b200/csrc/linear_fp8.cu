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
    int rows, n_out, k_blocks, act, tokens /* rows of x per tile: the MMA's N */, stages, y_dtype;
    uint32_t limit;
    int drill;
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
__device__ __forceinline__ void store_peer(uint32_t here, uint32_t rank, float v) {
    uint32_t there;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here), "r"(rank));
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there), "f"(v) : "memory");
}

__device__ __forceinline__ float load_as_float(const void* p, int dtype, size_t i) {
    if (dtype == SPEC_DTYPE_FP32) return static_cast<const float*>(p)[i];
    if (dtype == SPEC_DTYPE_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
    return __half2float(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_from_float(void* p, int dtype, size_t i, float v) {
    if (dtype == SPEC_DTYPE_FP32) static_cast<float*>(p)[i] = v;
    else if (dtype == SPEC_DTYPE_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
    else static_cast<__half*>(p)[i] = __float2half_rn(v);
}

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
// One accumulator value per lane (a row r of x, 32 rows of W) to y.  Whole warps only.
__device__ __forceinline__ void finish(const LinearArgs& a, const LaneColumn& c, int r, float acc) {
    float z = acc * a.x_scales[r] * c.scale + c.bias;
    if (a.act >= kActGatedGelu) {
        const float up = __shfl_xor_sync(kFullMask, z, 16);
        z = (a.act == kActGatedGelu ? gelu_tanh(z) : silu(z)) * up;
    } else if (a.act == kActGelu) {
        z = gelu_tanh(z);
    } else if (a.act == kActSilu) {
        z = silu(z);
    }
    if (c.column < 0) return;
    const size_t at = static_cast<size_t>(r) * a.n_out + c.column;
    if (a.residual) z += load_as_float(a.residual, a.y_dtype, at);
    store_from_float(a.y, a.y_dtype, at, z);
}

// grid = (tiles of 128 rows of W x CTAs of a cluster, tiles of x), clusters along x, block = kThreads.
__global__ void __launch_bounds__(kThreads)
linear_fp8_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ LinearArgs a) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int stage_bytes = kTileBytes + a.tokens * kBlockK;
    float* exchange = reinterpret_cast<float*>(smem + a.stages * stage_bytes);  // clusters of two and more: tokens * 128 floats
    const uint32_t splits = cluster_size(), rank = cluster_rank();
    uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + a.stages * stage_bytes + (splits > 1 ? a.tokens * kTileM * 4 : 0));
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
    pdl_trigger();
    pdl_wait();

    if (warp == 0) {
        const bool leader = elect_one() && !a.drill;
        const bool gated = a.act >= kActGatedGelu;
        int s = 0, use = 0;
        for (int kb = kb0; kb < kb1; ++kb) {
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
    // (a CTA without a k-block has nothing to wait for and adds nothing)
    const int quarter = warp & 3;  // accumulator lanes 32 quarter .. + 31 are what warps 2..5 may read
    const bool reader = warp >= 2, have = kb1 > kb0;
    const int valid = min(a.tokens, a.rows - row0);
    LaneColumn column{};
    if (reader) {
        column = lane_column(a, tile, quarter, lane);
        if (have && !mbar_wait_warp(acc_bar, 0, a.limit)) ok = false;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    }
    const uint32_t acc = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    if (splits == 1) {
        if (reader && ok)
            for (int c0 = 0; c0 < valid; c0 += 16) {
                uint32_t v[16];
                tmem_ld16(acc + c0, v);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (c0 + i < valid) finish(a, column, row0 + c0 + i, __uint_as_float(v[i]));
            }
    } else {
        // element (token c, quarter) is unit 4 c + quarter of 32 lanes; CTA r finishes units [first(r), first(r + 1))
        const int units = 4 * valid, most = (units + splits - 1) / splits;
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // everyone is there
        if (reader && ok)
            for (int c0 = 0; c0 < valid; c0 += 16) {
                uint32_t v[16];
                if (have) {
                    tmem_ld16(acc + c0, v);
                    tmem_ld_wait();
                }
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (c0 + i < valid) {
                        const int unit = 4 * (c0 + i) + quarter, to = unit / most;
                        store_peer(smem_u32(exchange + (rank * most + unit - to * most) * 32 + lane), to, have ? __uint_as_float(v[i]) : 0.0f);
                    }
            }
        cluster_sync_all();
        if (reader && ok) {
            const int u0 = rank * most, u1 = min(units, u0 + most);
            for (int unit = u0; unit < u1; ++unit) {
                if ((unit & 3) != quarter) continue;
                float sum = 0.0f;
                for (uint32_t p = 0; p < splits; ++p) sum += exchange[(p * most + unit - u0) * 32 + lane];
                finish(a, column, row0 + (unit >> 2), sum);
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

int launch_small(const void* x, const void* w, int k, LinearArgs a, cudaStream_t stream) {
    const bool gated = a.act >= kActGatedGelu;
    const int per_tile = gated ? kTileM / 2 : kTileM, tiles = (a.n_out + per_tile - 1) / per_tile;
    a.k_blocks = (k + kBlockK - 1) / kBlockK;
    int token_tiles = (a.rows + 127) / 128;
    a.tokens = ((a.rows + token_tiles - 1) / token_tiles + 15) / 16 * 16;
    token_tiles = (a.rows + a.tokens - 1) / a.tokens;
    int splits = 1;
    while (splits < 8 && tiles * token_tiles * splits * 2 <= 148 && splits * 2 <= a.k_blocks) splits *= 2;
    const int stage_bytes = kTileBytes + a.tokens * kBlockK, exchange = splits > 1 ? a.tokens * kTileM * 4 : 0;
    a.stages = std::min({kMaxStages, (227 * 1024 - 1024 - 512 - exchange) / stage_bytes, std::max(2, (a.k_blocks + splits - 1) / splits)});
    CUtensorMap mw, mx;
    int status = codes_map(w, gated ? 2 : 1, a.n_out, k, gated ? 2 : 1, gated ? 16 : kTileM, &mw);
    if (status == SPEC_OK) status = codes_map(x, 1, a.rows, k, 0, a.tokens, &mx);
    if (status != SPEC_OK) return status;
    static std::atomic<unsigned long long> configured{0};
    status = allow_shared_memory(configured, linear_fp8_kernel, 227 * 1024);
    if (status != SPEC_OK) return status;
    // 48 KB and more: at most four CTAs to an SM, whose tensor memory (128 columns each) then all fits.  A CTA that had to wait for
    // columns while its cluster waits for it could wait for ever.
    const int smem = std::max(48 * 1024, a.stages * stage_bytes + exchange + 1024 + 512);
    return launch_cluster(linear_fp8_kernel, splits, dim3(tiles * splits, token_tiles), dim3(kThreads), smem, stream, mw, mx, a);
}

}  // namespace

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
    a.y_dtype = y_dtype;
    a.limit = tc::kSpinLimit;
    return launch_small(x, w, k, a, static_cast<cudaStream_t>(stream));
}
