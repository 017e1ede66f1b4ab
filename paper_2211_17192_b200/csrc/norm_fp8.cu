// Rows to e4m3 codes with a scale each, as they are or behind the residual's addition and a root-mean-square norm:
//   h = x + residual (stored in its own type; the norm is taken of what was stored)
//   y = (h * gain) * (mean(h^2) + eps)^(-1/2),  codes and scale of y (fp8_util.cuh).
// Bound by memory: every element is read once, held in registers across the row's one reduction (the sum of squares and the
// largest |h * gain| travel together: the row's factor is positive, so it moves in front of the maximum, and rounding is
// monotone), and written once.  A CTA has one row; a thread has up to four groups of eight neighbouring elements.
#include <algorithm>

#include "fp8_util.cuh"

namespace spec {
namespace {

constexpr int kWidest = 32768;  // 1024 threads of four groups of eight

template <typename TX, typename TH, int GROUPS, bool NORM>
__global__ void __launch_bounds__(1024)
rows_fp8_kernel(const TX* x, const TH* residual, TH* h, const float* __restrict__ gain, float eps, int d, int wide,
                uint8_t* __restrict__ codes, float* __restrict__ scales) {
    pdl_trigger();
    pdl_wait();
    const size_t row = blockIdx.x;
    x += row * d;
    codes += row * d;
    float y[GROUPS][8];
    float squares = 0.0f;
    uint32_t largest = 0u;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const int c0 = (g * blockDim.x + threadIdx.x) * 8;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            const int c = c0 + half * 4;
            if (wide ? c < d : c + 4 <= d) load4(x + c, wide, v);
            else
                for (int i = 0; i < 4; ++i)
                    if (c + i < d) v[i] = to_float(x[c + i]);
#pragma unroll
            for (int i = 0; i < 4; ++i) y[g][half * 4 + i] = v[i];
        }
    }
    if constexpr (NORM) {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const int c0 = (g * blockDim.x + threadIdx.x) * 8;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int c = c0 + half * 4;
                float r[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (residual) {
                    const TH* in = residual + row * d + c;
                    if (wide ? c < d : c + 4 <= d) load4(in, wide, r);
                    else
                        for (int i = 0; i < 4; ++i)
                            if (c + i < d) r[i] = to_float(in[i]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) r[i] += y[g][half * 4 + i];
                if (h) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) r[i] = to_float(from_float<TH>(r[i]));
                    TH* out = h + row * d + c;
                    if (wide ? c < d : c + 4 <= d) store4(out, wide, r);
                    else
                        for (int i = 0; i < 4; ++i)
                            if (c + i < d) out[i] = from_float<TH>(r[i]);
                }
                float w[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (wide ? c < d : c + 4 <= d) load4(gain + c, wide, w);
                else
                    for (int i = 0; i < 4; ++i)
                        if (c + i < d) w[i] = gain[c + i];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    squares += r[i] * r[i];
                    y[g][half * 4 + i] = r[i] * w[i];
                }
            }
        }
    }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int i = 0; i < 8; ++i) largest = max(largest, magnitude(y[g][i]));

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
    float factor = 1.0f;
    if constexpr (NORM) {
        factor = __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(squares, static_cast<float>(d)) + eps));
        largest = magnitude(__uint_as_float(largest) * factor);
    }
    const float scale = row_scale(largest, kE4m3Top), inverse = __fdiv_rn(1.0f, scale);
    if (threadIdx.x == 0) scales[row] = scale;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const int c0 = (g * blockDim.x + threadIdx.x) * 8;
        uint32_t packed[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) packed[i] = codes_e4m3(y[g][2 * i] * factor * inverse, y[g][2 * i + 1] * factor * inverse);
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
};

template <typename TX, typename TH, bool NORM>
int launch_rows(const RowsArgs& a, cudaStream_t stream) {
    const int eights = (a.d + 7) / 8;
    const int groups = eights <= 512 ? 1 : eights <= 1024 ? 2 : 4;
    const int threads = ((eights + groups - 1) / groups + 31) / 32 * 32;
    const auto go = [&](auto kernel) {
        return launch_pdl(kernel, dim3(a.rows), dim3(threads), 0, stream, static_cast<const TX*>(a.x), static_cast<const TH*>(a.residual),
                          static_cast<TH*>(a.h), a.gain, a.eps, a.d, a.wide, a.codes, a.scales);
    };
    if (groups == 1) return go(rows_fp8_kernel<TX, TH, 1, NORM>);
    if (groups == 2) return go(rows_fp8_kernel<TX, TH, 2, NORM>);
    return go(rows_fp8_kernel<TX, TH, 4, NORM>);
}

}  // namespace
}  // namespace spec

extern "C" int spec_quantize_fp8(const void* x, int x_dtype, int rows, int d, void* codes, float* scales, void* stream) {
    using namespace spec;
    if (!float_dtype(x_dtype)) return fail(SPEC_ERR_BAD_ARG, "spec_quantize_fp8: dtype %d", x_dtype);
    if (rows < 0 || d < 1 || d > kWidest) return fail(SPEC_ERR_BAD_ARG, "spec_quantize_fp8: rows=%d d=%d (d in 1..%d)", rows, d, kWidest);
    if (rows == 0) return SPEC_OK;
    if (!x || !codes || !scales) return fail(SPEC_ERR_BAD_ARG, "spec_quantize_fp8: null pointer");
    if (!aligned_to(x, dtype_bytes(x_dtype)) || !aligned_to(scales, 4)) return fail(SPEC_ERR_BAD_ARG, "spec_quantize_fp8: a pointer is not aligned to its elements");
    RowsArgs a{x, nullptr, nullptr, nullptr, 0.0f, rows, d, 0, static_cast<uint8_t*>(codes), scales};
    a.wide = d % 8 == 0 && aligned_to(x, 16) && aligned_to(codes, 8);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (x_dtype == SPEC_DTYPE_FP32) return launch_rows<float, float, false>(a, st);
    if (x_dtype == SPEC_DTYPE_BF16) return launch_rows<__nv_bfloat16, float, false>(a, st);
    return launch_rows<__half, float, false>(a, st);
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
    RowsArgs a{x, residual, h, gain, eps, rows, d, 0, static_cast<uint8_t*>(codes), scales};
    a.wide = d % 8 == 0 && aligned_to(x, 16) && aligned_to(residual, 16) && aligned_to(h, 16) && aligned_to(gain, 16) && aligned_to(codes, 8);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool same = sum && h_dtype == x_dtype;
    if (x_dtype == SPEC_DTYPE_FP32) return launch_rows<float, float, true>(a, st);
    if (x_dtype == SPEC_DTYPE_BF16) return same ? launch_rows<__nv_bfloat16, __nv_bfloat16, true>(a, st) : launch_rows<__nv_bfloat16, float, true>(a, st);
    return same ? launch_rows<__half, __half, true>(a, st) : launch_rows<__half, float, true>(a, st);
}
