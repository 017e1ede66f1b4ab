// Rows to e4m3 codes with a scale each, as they are or behind the residual's addition and a root-mean-square norm:
//   h = x + residual (stored in its own type; the norm is taken of what was stored)
//   y = (h * gain) * (mean(h^2) + eps)^(-1/2),  codes and scale of y (fp8_util.cuh).
// Codes are h * gain times 448 / max |h * gain|, which is 1 / scale with the row's factor taken out of both: two roundings instead of
// eight, and half as many codes on the other side of a tie.
// Bound by memory: every element is read once, held on chip across the row's one reduction (the sum of squares and the
// largest |h * gain| travel together: the row's factor is positive, so it moves in front of the maximum, and rounding is
// monotone), and written once.  Two kernels.  Few or narrow rows: a CTA to a row, which lies in registers, up to four groups of eight
// neighbouring elements to a thread.  Many wide rows: CTAs that stay, to which one warp brings row after row by bulk copies through
// a ring in shared memory, so that the next rows are on their way while one is reduced.
#include <algorithm>

#include "fp8_util.cuh"
#include "tc_util.cuh"

namespace spec {
namespace {

constexpr int kWidest = 32768;  // 1024 threads of four groups of eight

// max(m, |v|), a NaN if v or m is one (as bits NaNs are the largest too: both kernels give a row that has one the same scale).
__device__ __forceinline__ float larger_magnitude(float m, float v) {
    asm("{\n\t.reg .f32 a;\n\tabs.f32 a, %1;\n\tmax.NaN.f32 %0, %0, a;\n\t}" : "+f"(m) : "f"(v));
    return m;
}

// The row's scale, and what its values (before the norm's factor) are multiplied with to be its codes: first with `lift`, 1 or a power of two
// where the other alone would be past fp32's range (448 / 10^-36, or 2^48 and more in front of the least scale: not unless eps is
// below kTinyEps), then with what is returned.
constexpr float kTinyEps = 0x1p-90f;
template <bool NORM, bool TINY>
__device__ __forceinline__ float code_factor(uint32_t largest, float squares, int d, float eps, float& scale, float& lift) {
    constexpr float kLift = 0x1p64f;
    lift = 1.0f;
    if constexpr (!NORM) {
        scale = row_scale(largest, kE4m3Top);
        return __fdiv_rn(1.0f, scale);
    }
    // (squares that add up past fp32's range are no mean: a factor of zero would make a row of zeros of the largest there are)
    float factor = squares < INFINITY ? __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(squares, static_cast<float>(d)) + eps)) : NAN;
    const float most = __uint_as_float(largest);
    const uint32_t top = magnitude(most * factor);
    scale = row_scale(top, kE4m3Top);
    if (top == 0u || scale == kLeastScale || !(scale < 3.0e38f)) {  // a row of zeros, of values that no scale is small enough for, of no numbers
        if (TINY && factor > 0x1p46f) {
            lift = kLift;
            factor *= 1.0f / kLift;
        }
        return factor * __fdiv_rn(1.0f, scale);
    }
    if (TINY && most < 0x1p-118f) lift = kLift;
    return __fdiv_rn(kE4m3Top, TINY ? most * lift : most);
}

// Between its two passes a row is held as HOLD, the type it is stored in: as fp32 the registers left one CTA of a 2048 x 11008
// call to an SM, and nothing overlapped a row's reduction (19 us).
template <typename TX, typename TH, typename HOLD, int GROUPS, bool NORM>
__global__ void __launch_bounds__(1024)
rows_fp8_kernel(const TX* x, const TH* residual, TH* h, const float* __restrict__ gain, float eps, int d, int wide, uint8_t* __restrict__ codes,
                float* __restrict__ scales) {
    pdl_trigger();
    pdl_wait();
    gain = after_wait(gain);
    const size_t row = blockIdx.x;
    x += row * d;
    codes += row * d;
    __align__(16) HOLD hold[GROUPS][8];
    float squares = 0.0f;
    uint32_t largest = 0u;
    const auto take = [&](const auto* from, int c0, float(&v)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        if (wide ? c0 < d : c0 + 8 <= d) load_row(from + c0, wide, v);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c0 + i < d) v[i] = to_float(from[c0 + i]);
    };
    const auto put = [&](auto* to, int c0, const float(&v)[8]) {
        using T = std::remove_reference_t<decltype(*to)>;
        if (wide ? c0 < d : c0 + 8 <= d) store_row(to + c0, wide, v);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c0 + i < d) to[c0 + i] = from_float<T>(v[i]);
    };
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const int c0 = (g * blockDim.x + threadIdx.x) * 8;
        float v[8];
        take(x, c0, v);
        if constexpr (NORM) {
            if (residual) {
                float r[8];
                take(residual + row * d, c0, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += r[i];
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) hold[g][i] = from_float<HOLD>(v[i]);
    }
    // what the row's codes are made of, but for its factor
    const auto value = [&](int g, const float(&w)[8], int i) { return NORM ? to_float(hold[g][i]) * w[i] : to_float(hold[g][i]); };
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const int c0 = (g * blockDim.x + threadIdx.x) * 8;
        float w[8];
        if constexpr (NORM) {
            if (h) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = to_float(hold[g][i]);
                put(h + row * d, c0, v);
            }
            take(gain, c0, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) squares += to_float(hold[g][i]) * to_float(hold[g][i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) largest = max(largest, magnitude(value(g, w, i)));
    }

    __shared__ float part_squares[32];
    __shared__ uint32_t part_largest[32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    if constexpr (NORM) squares = warp_sum(squares);
    largest = __reduce_max_sync(kFullMask, largest);
    if (warps > 1) {
        if (lane == 0) {
            if constexpr (NORM) part_squares[warp] = squares;
            part_largest[warp] = largest;
        }
        __syncthreads();
        if constexpr (NORM) squares = warp_sum(lane < warps ? part_squares[lane] : 0.0f);
        largest = __reduce_max_sync(kFullMask, lane < warps ? part_largest[lane] : 0u);
    }
    float scale, lift;
    const float factor = code_factor<NORM, true>(largest, squares, d, eps, scale, lift);
    if (threadIdx.x == 0) scales[row] = scale;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const int c0 = (g * blockDim.x + threadIdx.x) * 8;
        float w[8];
        if constexpr (NORM) take(gain, c0, w);
        uint32_t packed[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) packed[i] = codes_e4m3(value(g, w, 2 * i) * lift * factor, value(g, w, 2 * i + 1) * lift * factor);
        if (wide) {
            if (c0 < d) *reinterpret_cast<uint2*>(codes + c0) = make_uint2(packed[0] | packed[1] << 16, packed[2] | packed[3] << 16);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c0 + i < d) codes[c0 + i] = static_cast<uint8_t>(packed[i >> 1] >> (8 * (i & 1)));
        }
    }
}

struct RowsArgs {
    const void *x, *residual;
    void* h;
    const float* gain;
    float eps;
    int rows, d, wide;
    uint8_t* codes;
    float* scales;
    int stages, stage_bytes;
};

// ---- many wide rows ----
constexpr int kStreamWarps = 8;  // that compute; one more fetches
constexpr int kStreamThreads = 32 * (kStreamWarps + 1);
constexpr int kStreamStages = 8;

__device__ int g_rows_error;  // set when a bounded wait for a row or for its place ran out (0 = none)

// Rows blockIdx.x, + gridDim.x, ..  A stage holds a row of x and one of the residual; a thread has the same ITER groups of eight
// columns of every row, in registers between the row's two passes, and for narrow rows their gains too.  (Issue bounds it as much as memory:
// with the second pass from shared memory and the gains from L1 a row of 2048 x 4096 took 440 instructions a warp, 17.9 us.)
template <typename TX, typename TH, typename HOLD, int ITER, bool NORM>
__global__ void __launch_bounds__(kStreamThreads)
rows_fp8_stream_kernel(const __grid_constant__ RowsArgs a) {
    using namespace tc;
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ uint64_t full_bar[kStreamStages], empty_bar[kStreamStages];
    __shared__ float part_squares[2][kStreamWarps];
    __shared__ uint32_t part_largest[2][kStreamWarps];
    const int warp = __shfl_sync(kFullMask, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(&full_bar[s], 1);
            mbar_init(&empty_bar[s], kStreamWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    pdl_wait();
    const int d = a.d, x_bytes = d * static_cast<int>(sizeof(TX));
    const bool summed = NORM && a.residual;
    uint32_t limit = kSpinLimit;  // of every wait; one that has run out leaves one try to the others, and the CTA ends with its error noted
    int stage = 0, use = 0;

    if (warp == kStreamWarps) {
        const bool leader = elect_one();
        const auto fetch = [&](void* to, const void* from, int bytes, uint64_t* bar) {
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(smem_u32(to)), "l"(from), "r"(bytes), "r"(smem_u32(bar)) : "memory");
        };
        for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
            if (use > 0 && !mbar_wait_warp(&empty_bar[stage], (use - 1) & 1, limit)) limit = 1;
            if (leader) {
                uint8_t* to = ring + stage * a.stage_bytes;
                mbar_expect_tx(&full_bar[stage], a.stage_bytes);
                fetch(to, static_cast<const TX*>(a.x) + static_cast<size_t>(row) * d, x_bytes, &full_bar[stage]);
                if (summed) fetch(to + x_bytes, static_cast<const TH*>(a.residual) + static_cast<size_t>(row) * d, a.stage_bytes - x_bytes, &full_bar[stage]);
            }
            __syncwarp();
            if (++stage == a.stages) { stage = 0; ++use; }
        }
        pdl_trigger();  // (behind the last row that is asked for: let in at the top, the next kernel's CTAs come to lie unevenly; 2048 x 4096 13.9 us, 12.2 so)
        if (limit != kSpinLimit) {  // nothing may still be on its way when the CTA leaves
            for (int s = 0; s < a.stages; ++s) {
                mbar_wait(&full_bar[s], 0, 1 << 14);
                mbar_wait(&full_bar[s], 1, 1 << 14);
            }
            if (lane == 0) atomicCAS(&g_rows_error, 0, 1);
        }
        return;
    }
    constexpr int kStep = 32 * kStreamWarps * 8;
    constexpr bool kGains = NORM && ITER <= 2;
    const int c0 = threadIdx.x * 8;
    float gains[kGains ? ITER : 1][8];
    if constexpr (kGains) {
#pragma unroll
        for (int g = 0; g < ITER; ++g)
            if (c0 + g * kStep < d) load_row(a.gain + c0 + g * kStep, true, gains[g]);
    }
    int turn = 0;
    for (int row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        if (!mbar_wait_warp(&full_bar[stage], use & 1, limit)) limit = 1;
        const TX* x = reinterpret_cast<const TX*>(ring + stage * a.stage_bytes) + c0;
        const TH* residual = reinterpret_cast<const TH*>(ring + stage * a.stage_bytes + x_bytes) + c0;
        const size_t at = static_cast<size_t>(row) * d + c0;
        float v[ITER][8], squares = 0.0f, most = 0.0f;
        uint32_t largest = 0u;
#pragma unroll
        for (int g = 0; g < ITER; ++g) {
            if (c0 + g * kStep >= d) continue;
            load_row(x + g * kStep, true, v[g]);
            if constexpr (NORM) {
                if (summed) {
                    float r[8];
                    load_row(residual + g * kStep, true, r);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[g][i] = to_float(from_float<HOLD>(v[g][i] + r[i]));
                }
                if (a.h) store_row(static_cast<TH*>(a.h) + at + g * kStep, true, v[g]);
                float w[8];
                if constexpr (!kGains) load_row(a.gain + c0 + g * kStep, true, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    squares += v[g][i] * v[g][i];
                    v[g][i] *= kGains ? gains[kGains ? g : 0][i] : w[i];
                    most = larger_magnitude(most, v[g][i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) largest = max(largest, magnitude(v[g][i]));
            }
        }
        __syncwarp();
        if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(&empty_bar[stage])) : "memory");
        if (++stage == a.stages) { stage = 0; ++use; }
        if constexpr (NORM) {
            squares = warp_sum(squares);
            largest = magnitude(most);
        }
        largest = __reduce_max_sync(kFullMask, largest);
        if (lane == 0) {
            if constexpr (NORM) part_squares[turn][warp] = squares;
            part_largest[turn][warp] = largest;
        }
        asm volatile("bar.sync 1, %0;" ::"n"(32 * kStreamWarps) : "memory");  // (one per row: the next row's parts lie in the other half)
        largest = 0u;
#pragma unroll
        for (int w = 0; w < kStreamWarps; ++w) largest = max(largest, part_largest[turn][w]);
        if constexpr (NORM) {
            squares = 0.0f;
#pragma unroll
            for (int w = 0; w < kStreamWarps; ++w) squares += part_squares[turn][w];
        }
        float scale, lift;
        const float factor = code_factor<NORM, false>(largest, squares, d, a.eps, scale, lift);
        if (threadIdx.x == 0) a.scales[row] = scale;
#pragma unroll
        for (int g = 0; g < ITER; ++g) {
            if (c0 + g * kStep >= d) continue;
            uint32_t packed[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) packed[i] = codes_e4m3(v[g][2 * i] * factor, v[g][2 * i + 1] * factor);
            *reinterpret_cast<uint2*>(a.codes + at + g * kStep) = make_uint2(packed[0] | packed[1] << 16, packed[2] | packed[3] << 16);
        }
    }
    if (limit != kSpinLimit && lane == 0) atomicCAS(&g_rows_error, 0, 2);
}

template <typename TX, typename TH, typename HOLD, bool NORM>
int launch_rows(RowsArgs a, cudaStream_t stream) {
    const bool summed = NORM && a.residual;
    a.stage_bytes = a.d * static_cast<int>(sizeof(TX) + (summed ? sizeof(TH) : 0));
    // 2048 x 4096 bf16 with a bf16 residual: 11.5 us here, 16.3 with a CTA to a row; 150 rows 2.5 and 3.5; 2048 x 1024 9.1 and 5.4 (a
    // thread has eight columns of a row, and half of them have none).  Two CTAs to an SM and 48 KB of ring to each: with 64 KB the
    // next kernel's CTAs find no room beside these before they end (14.2 us).  (A tiny eps takes one product more for a code: 13.0 for 12.7 us here.)
    if (a.wide && a.d >= 2048 && a.d <= 16384 && a.rows >= 148 && a.stage_bytes <= 56 * 1024 && (!NORM || a.eps >= kTinyEps) && (!summed || std::is_same_v<HOLD, TH>)) {
        a.stages = std::max(2, std::min(kStreamStages, 48 * 1024 / a.stage_bytes));
        const int smem = a.stages * a.stage_bytes, rounds = (a.rows + 2 * 148 - 1) / (2 * 148);
        const auto go = [&](auto kernel, std::atomic<unsigned long long>& configured) {
            const int status = allow_shared_memory(configured, kernel, 113 * 1024);
            if (status != SPEC_OK) return status;
            return launch_pdl(kernel, dim3((a.rows + rounds - 1) / rounds), dim3(kStreamThreads), smem, stream, a);
        };
        static std::atomic<unsigned long long> configured[4];
        if (a.d <= 2048) return go(rows_fp8_stream_kernel<TX, TH, HOLD, 1, NORM>, configured[0]);
        if (a.d <= 4096) return go(rows_fp8_stream_kernel<TX, TH, HOLD, 2, NORM>, configured[1]);
        if (a.d <= 8192) return go(rows_fp8_stream_kernel<TX, TH, HOLD, 4, NORM>, configured[2]);
        return go(rows_fp8_stream_kernel<TX, TH, HOLD, 8, NORM>, configured[3]);
    }
    const int eights = (a.d + 7) / 8;
    const int groups = eights <= 512 ? 1 : eights <= 1024 ? 2 : 4;
    const int threads = ((eights + groups - 1) / groups + 31) / 32 * 32;
    const auto go = [&](auto kernel) {
        return launch_pdl(kernel, dim3(a.rows), dim3(threads), 0, stream, static_cast<const TX*>(a.x), static_cast<const TH*>(a.residual),
                          static_cast<TH*>(a.h), a.gain, a.eps, a.d, a.wide, a.codes, a.scales);
    };
    if (groups == 1) return go(rows_fp8_kernel<TX, TH, HOLD, 1, NORM>);
    if (groups == 2) return go(rows_fp8_kernel<TX, TH, HOLD, 2, NORM>);
    return go(rows_fp8_kernel<TX, TH, HOLD, 4, NORM>);
}

}  // namespace

int norm_fp8_take_error() {
    int v = 0, zero = 0;
    if (cudaMemcpyFromSymbol(&v, g_rows_error, sizeof(int)) != cudaSuccess) return -1;
    if (v) cudaMemcpyToSymbol(g_rows_error, &zero, sizeof(int));
    return v;
}

}  // namespace spec

extern "C" int spec_quantize_fp8(const void* x, int x_dtype, int rows, int d, void* codes, float* scales, void* stream) {
    using namespace spec;
    if (!float_dtype(x_dtype)) return fail(SPEC_ERR_BAD_ARG, "spec_quantize_fp8: dtype %d", x_dtype);
    if (rows < 0 || d < 1 || d > kWidest) return fail(SPEC_ERR_BAD_ARG, "spec_quantize_fp8: rows=%d d=%d (d in 1..%d)", rows, d, kWidest);
    if (rows == 0) return SPEC_OK;
    if (!x || !codes || !scales) return fail(SPEC_ERR_BAD_ARG, "spec_quantize_fp8: null pointer");
    if (!aligned_to(x, dtype_bytes(x_dtype)) || !aligned_to(scales, 4)) return fail(SPEC_ERR_BAD_ARG, "spec_quantize_fp8: a pointer is not aligned to its elements");
    RowsArgs a{x, nullptr, nullptr, nullptr, 0.0f, rows, d, 0, static_cast<uint8_t*>(codes), scales, 0, 0};
    a.wide = d % 8 == 0 && aligned_to(x, 16) && aligned_to(codes, 8);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (x_dtype == SPEC_DTYPE_FP32) return launch_rows<float, float, float, false>(a, st);
    if (x_dtype == SPEC_DTYPE_BF16) return launch_rows<__nv_bfloat16, __nv_bfloat16, __nv_bfloat16, false>(a, st);
    return launch_rows<__half, __half, __half, false>(a, st);
}

extern "C" int spec_norm_fp8(const void* x, int x_dtype, const void* residual, void* h, int h_dtype, const float* gain, float eps,
                             int rows, int d, void* codes, float* scales, void* stream) {
    using namespace spec;
    if (!float_dtype(x_dtype)) return fail(SPEC_ERR_BAD_ARG, "spec_norm_fp8: dtype %d", x_dtype);
    const bool sum = residual || h;
    if (sum && h_dtype != SPEC_DTYPE_FP32 && h_dtype != x_dtype) return fail(SPEC_ERR_BAD_ARG, "spec_norm_fp8: h_dtype %d is neither fp32 nor x's", h_dtype);
    if (rows < 0 || d < 1 || d > kWidest) return fail(SPEC_ERR_BAD_ARG, "spec_norm_fp8: rows=%d d=%d (d in 1..%d)", rows, d, kWidest);
    if (!(eps > 0.0f) || eps > 3.0e38f) return fail(SPEC_ERR_BAD_ARG, "spec_norm_fp8: eps must be finite and above zero");
    if (rows == 0) return SPEC_OK;
    if (!x || !gain || !codes || !scales) return fail(SPEC_ERR_BAD_ARG, "spec_norm_fp8: null pointer");
    const int hb = sum ? dtype_bytes(h_dtype) : 1;
    if (!aligned_to(x, dtype_bytes(x_dtype)) || !aligned_to(residual, hb) || !aligned_to(h, hb) || !aligned_to(gain, 4) || !aligned_to(scales, 4))
        return fail(SPEC_ERR_BAD_ARG, "spec_norm_fp8: a pointer is not aligned to its elements");
    RowsArgs a{x, residual, h, gain, eps, rows, d, 0, static_cast<uint8_t*>(codes), scales, 0, 0};
    a.wide = d % 8 == 0 && aligned_to(x, 16) && aligned_to(residual, 16) && aligned_to(h, 16) && aligned_to(gain, 16) && aligned_to(codes, 8);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const auto go = [&](auto type) {
        using T = decltype(type);
        if (!sum) return launch_rows<T, T, T, true>(a, st);
        if (h_dtype == SPEC_DTYPE_FP32) return launch_rows<T, float, float, true>(a, st);
        if (!h) return launch_rows<T, T, float, true>(a, st);  // (a sum that is not stored is not rounded)
        return launch_rows<T, T, T, true>(a, st);
    };
    return x_dtype == SPEC_DTYPE_FP32 ? go(float{}) : x_dtype == SPEC_DTYPE_BF16 ? go(__nv_bfloat16{}) : go(__half{});
}
