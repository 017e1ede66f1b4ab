// New tokens' K and V rows into a paged cache in 16 or 8 bits (rotary positions on the way), and cached rows back out.
//
// Both kernels are bound by memory and, at a few rows, by the latency of one dependent chain (start -> page -> row).  A group
// of d_head / 8 lanes has one row of one head: eight elements to a lane, so that a pair of a rotation (j, j + d_head / 2) and the
// largest magnitude of the row never leave the group, and nothing goes through shared memory.
#include <algorithm>

#include "paged.cuh"

namespace spec {
namespace {

constexpr int kThreads = 256;

// Elements in the order that the rotation wants: four at 4 l, four at 4 l + d / 2.
template <typename T, int D, int KV>
__global__ void __launch_bounds__(kThreads)
kv_append_kernel(const T* q, const T* k, const T* v, long long q_stride, long long k_stride, long long v_stride, int n_heads,
                 const __grid_constant__ Paged cache, void* pool, float* scales, const int32_t* start, const int32_t* counts, int batch, int rows,
                 const float2* rope, int rope_positions, T* q_out, int wide) {
    pdl_trigger();
    pdl_wait();
    constexpr int kLanes = D / 8;
    const int items = n_heads + 2 * cache.n_kv;
    const long long group = (static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x) / kLanes;
    const int l = threadIdx.x % kLanes;
    const long long total = static_cast<long long>(batch) * rows * items;
    const long long token = min(group, total - 1) / items;  // (lanes past the end go along, for the exchanges below)
    const int item = static_cast<int>(min(group, total - 1) - token * items);
    const int b = static_cast<int>(token / rows), r = static_cast<int>(token - static_cast<long long>(b) * rows);
    const int first = start[b];
    bool live = group < total && r < (counts ? counts[b] : rows) && first >= 0 && first <= 0x7fffffff - rows;
    const int position = live ? first + r : 0;
    if (rope && position >= rope_positions) live = false;

    const bool is_q = item < n_heads;
    const int which = is_q ? 0 : (item - n_heads) / cache.n_kv;
    const int head = is_q ? item : (item - n_heads) - which * cache.n_kv;
    const T* src = is_q ? q + token * q_stride : which == 0 ? k + token * k_stride : v + token * v_stride;
    src += head * D + 4 * l;
    float lo[4] = {0.0f, 0.0f, 0.0f, 0.0f}, hi[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (live) {
        load4(src, wide, lo);
        load4(src + D / 2, wide, hi);
    }
    if (live && rope && (is_q || which == 0)) {
        const float2* cs = rope + static_cast<size_t>(position) * (D / 2) + 4 * l;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 t = cs[i];
            const float x = lo[i], y = hi[i];
            // (each product and the sum rounded by itself: the same bits as an elementwise program's, so that codes agree)
            lo[i] = __fsub_rn(__fmul_rn(x, t.x), __fmul_rn(y, t.y));
            hi[i] = __fadd_rn(__fmul_rn(y, t.x), __fmul_rn(x, t.y));
        }
    }
    if (is_q) {
        if (live) {
            T* out = q_out + (token * n_heads + head) * D + 4 * l;
            store4(out, wide, lo);
            store4(out + D / 2, wide, hi);
        }
    }
    const long long at = live && !is_q ? cache.row(b, which, head, position) : -1;
    if constexpr (KV == SPEC_DTYPE_E4M3 || KV == SPEC_DTYPE_INT8) {
        uint32_t largest = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) largest = max(largest, max(magnitude(lo[i]), magnitude(hi[i])));
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) largest = max(largest, __shfl_xor_sync(kFullMask, largest, o));
        if (at < 0) return;
        const float scale = row_scale(largest, KV == SPEC_DTYPE_E4M3 ? kE4m3Top : kInt8Top), inverse = __fdiv_rn(1.0f, scale);
        uint32_t c[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float(&y)[4] = h ? hi : lo;
            if constexpr (KV == SPEC_DTYPE_E4M3) c[h] = codes_e4m3(y[0] * inverse, y[1] * inverse) | codes_e4m3(y[2] * inverse, y[3] * inverse) << 16;
            else c[h] = codes_int8(y[0] * inverse, y[1] * inverse) | codes_int8(y[2] * inverse, y[3] * inverse) << 16;
        }
        uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(pool) + at * D) + l;
        out[0] = c[0];
        out[D / 8] = c[1];
        if (l == 0) scales[at] = scale;
    } else {
        if (at < 0) return;
        using E = std::conditional_t<KV == SPEC_DTYPE_BF16, __nv_bfloat16, __half>;
        if constexpr (KV == SPEC_DTYPE_FP16) {  // (finite values past the type's range are held as its largest, as in the engine's caches)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (fabsf(lo[i]) > 65504.0f) lo[i] = copysignf(65504.0f, lo[i]);
                if (fabsf(hi[i]) > 65504.0f) hi[i] = copysignf(65504.0f, hi[i]);
            }
        }
        E* out = static_cast<E*>(pool) + at * D + 4 * l;
        store4(out, true, lo);
        store4(out + D / 2, true, hi);
    }
}

template <typename T, int D, int KV>
__global__ void __launch_bounds__(kThreads)
kv_read_kernel(const __grid_constant__ Paged cache, const void* __restrict__ pool, const float* __restrict__ scales, const int32_t* start,
               const int32_t* counts, int batch, int rows, T* k, T* v, int wide) {
    pdl_trigger();
    pdl_wait();
    constexpr int kLanes = D / 8;
    const int items = 2 * cache.n_kv;
    const long long group = (static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x) / kLanes;
    const int l = threadIdx.x % kLanes;
    if (group >= static_cast<long long>(batch) * rows * items) return;
    const long long token = group / items;
    const int item = static_cast<int>(group - token * items);
    const int b = static_cast<int>(token / rows), r = static_cast<int>(token - static_cast<long long>(b) * rows);
    const int first = start[b];
    if (r >= (counts ? counts[b] : rows) || first < 0 || first > 0x7fffffff - rows) return;
    const int which = item / cache.n_kv, head = item - which * cache.n_kv;
    const long long at = cache.row(b, which, head, first + r);
    if (at < 0) return;
    float y[2][4];
    if constexpr (KV == SPEC_DTYPE_E4M3 || KV == SPEC_DTYPE_INT8) {
        const uint2 c = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(pool) + at * D + 8 * l);
        const float scale = scales[at];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t byte = (h ? c.y : c.x) >> (8 * i) & 0xffu;
                if constexpr (KV == SPEC_DTYPE_E4M3) {
                    __nv_fp8_e4m3 e;
                    e.__x = static_cast<__nv_fp8_storage_t>(byte);
                    y[h][i] = static_cast<float>(e) * scale;
                } else {
                    y[h][i] = static_cast<float>(static_cast<int8_t>(byte)) * scale;
                }
            }
        }
    } else {
        using E = std::conditional_t<KV == SPEC_DTYPE_BF16, __nv_bfloat16, __half>;
        const E* src = static_cast<const E*>(pool) + at * D + 8 * l;
        load4(src, true, y[0]);
        load4(src + 4, true, y[1]);
    }
    T* out = (which == 0 ? k : v) + (token * cache.n_kv + head) * D + 8 * l;
    store4(out, wide, y[0]);
    store4(out + 4, wide, y[1]);
}

bool grid_of(long long items, int lanes, unsigned* grid) {
    const long long blocks = (items * lanes + kThreads - 1) / kThreads;
    *grid = static_cast<unsigned>(blocks);
    return blocks <= 0x7fffffffll;
}

template <typename F>
int with_kv(int kv_dtype, F f) {
    switch (kv_dtype) {
        case SPEC_DTYPE_FP16: return f(std::integral_constant<int, SPEC_DTYPE_FP16>{});
        case SPEC_DTYPE_BF16: return f(std::integral_constant<int, SPEC_DTYPE_BF16>{});
        case SPEC_DTYPE_E4M3: return f(std::integral_constant<int, SPEC_DTYPE_E4M3>{});
        default: return f(std::integral_constant<int, SPEC_DTYPE_INT8>{});
    }
}
template <typename F>
int with_float(int dtype, F f) {
    if (dtype == SPEC_DTYPE_FP32) return f(float{});
    if (dtype == SPEC_DTYPE_BF16) return f(__nv_bfloat16{});
    return f(__half{});
}

}  // namespace

int check_paged(const char* who, const void* pool, const float* scales, int kv_dtype, int pages, int page_size, int n_kv_heads, int d_head,
                const int32_t* page_table, int max_pages, int batch, Paged* out) {
    const bool eight = kv_dtype == SPEC_DTYPE_E4M3 || kv_dtype == SPEC_DTYPE_INT8;
    if (!eight && kv_dtype != SPEC_DTYPE_FP16 && kv_dtype != SPEC_DTYPE_BF16) return fail(SPEC_ERR_BAD_ARG, "%s: kv_dtype %d", who, kv_dtype);
    if (d_head != 64 && d_head != 128) return fail(SPEC_ERR_BAD_ARG, "%s: d_head=%d (64 or 128)", who, d_head);
    if (page_size < 32 || page_size > 256 || (page_size & (page_size - 1))) return fail(SPEC_ERR_BAD_ARG, "%s: page_size=%d (a power of two in 32..256)", who, page_size);
    if (n_kv_heads < 1 || n_kv_heads > 1024 || pages < 1 || max_pages < 1 || max_pages > 0x7fffffff / page_size || batch < 0 || batch > 65535)
        return fail(SPEC_ERR_BAD_ARG, "%s: n_kv_heads=%d pages=%d max_pages=%d batch=%d", who, n_kv_heads, pages, max_pages, batch);
    if (!pool || !page_table || (eight && !scales)) return fail(SPEC_ERR_BAD_ARG, "%s: null pointer", who);
    if (!aligned_to(pool, 16) || !aligned_to(page_table, 4) || !aligned_to(scales, 4)) return fail(SPEC_ERR_BAD_ARG, "%s: a pointer is not aligned (the pool to 16 bytes)", who);
    int shift = 0;
    while ((1 << shift) < page_size) ++shift;
    *out = Paged{page_table, pages, max_pages, n_kv_heads, shift};
    return SPEC_OK;
}

}  // namespace spec

extern "C" int spec_kv_append(const void* q, const void* k, const void* v, int dtype, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                              int n_heads, int n_kv_heads, int d_head, int batch, int rows, const int32_t* start, const int32_t* counts,
                              const float* rope, int rope_positions, void* q_out, void* pool, float* scales, int kv_dtype, int pages, int page_size,
                              const int32_t* page_table, int max_pages, void* stream) {
    using namespace spec;
    const char* who = "spec_kv_append";
    if (!float_dtype(dtype)) return fail(SPEC_ERR_BAD_ARG, "%s: dtype %d", who, dtype);
    if (rows < 0 || batch < 0) return fail(SPEC_ERR_BAD_ARG, "%s: batch=%d rows=%d", who, batch, rows);
    if (rows == 0 || batch == 0) return SPEC_OK;
    Paged cache;
    const int status = check_paged(who, pool, scales, kv_dtype, pages, page_size, n_kv_heads, d_head, page_table, max_pages, batch, &cache);
    if (status != SPEC_OK) return status;
    if (!k || !v || !start) return fail(SPEC_ERR_BAD_ARG, "%s: null pointer", who);
    if ((q != nullptr) != (q_out != nullptr) || (q && n_heads < 1) || n_heads < 0 || n_heads > 65536) return fail(SPEC_ERR_BAD_ARG, "%s: q and q_out come together, with n_heads in 1..65536", who);
    if (rope && rope_positions < 1) return fail(SPEC_ERR_BAD_ARG, "%s: rope_positions=%d", who, rope_positions);
    const int heads = q ? n_heads : 0, bytes = dtype_bytes(dtype);
    if (k_stride < static_cast<int64_t>(n_kv_heads) * d_head || v_stride < static_cast<int64_t>(n_kv_heads) * d_head || (q && q_stride < static_cast<int64_t>(heads) * d_head))
        return fail(SPEC_ERR_BAD_ARG, "%s: a row stride is below the heads' elements", who);
    if (!aligned_to(q, bytes) || !aligned_to(k, bytes) || !aligned_to(v, bytes) || !aligned_to(q_out, bytes) || !aligned_to(rope, 8) || !aligned_to(start, 4) || !aligned_to(counts, 4))
        return fail(SPEC_ERR_BAD_ARG, "%s: a pointer is not aligned to its elements", who);
    const size_t vec = 4 * static_cast<size_t>(bytes);
    const int wide = aligned_to(q, vec) && aligned_to(k, vec) && aligned_to(v, vec) && aligned_to(q_out, vec) && k_stride % 4 == 0 && v_stride % 4 == 0 && (!q || q_stride % 4 == 0);
    unsigned grid;
    if (!grid_of(static_cast<long long>(batch) * rows * (heads + 2 * n_kv_heads), d_head / 8, &grid)) return fail(SPEC_ERR_BAD_ARG, "%s: too many rows for one call", who);
    return with_float(dtype, [&](auto t) {
        using T = decltype(t);
        return with_kv(kv_dtype, [&](auto kv) {
            constexpr int KV = decltype(kv)::value;
            const auto go = [&](auto kernel) {
                return launch_pdl(kernel, dim3(grid), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), static_cast<const T*>(q), static_cast<const T*>(k),
                                  static_cast<const T*>(v), static_cast<long long>(q_stride), static_cast<long long>(k_stride), static_cast<long long>(v_stride),
                                  heads, cache, pool, scales, start, counts, batch, rows, reinterpret_cast<const float2*>(rope), rope_positions, static_cast<T*>(q_out), wide);
            };
            return d_head == 64 ? go(kv_append_kernel<T, 64, KV>) : go(kv_append_kernel<T, 128, KV>);
        });
    });
}

extern "C" int spec_kv_read(const void* pool, const float* scales, int kv_dtype, int pages, int page_size, int n_kv_heads, int d_head,
                            const int32_t* page_table, int max_pages, int batch, int rows, const int32_t* start, const int32_t* counts,
                            void* k, void* v, int dtype, void* stream) {
    using namespace spec;
    const char* who = "spec_kv_read";
    if (!float_dtype(dtype)) return fail(SPEC_ERR_BAD_ARG, "%s: dtype %d", who, dtype);
    if (rows < 0 || batch < 0) return fail(SPEC_ERR_BAD_ARG, "%s: batch=%d rows=%d", who, batch, rows);
    if (rows == 0 || batch == 0) return SPEC_OK;
    Paged cache;
    const int status = check_paged(who, pool, scales, kv_dtype, pages, page_size, n_kv_heads, d_head, page_table, max_pages, batch, &cache);
    if (status != SPEC_OK) return status;
    if (!k || !v || !start) return fail(SPEC_ERR_BAD_ARG, "%s: null pointer", who);
    const int bytes = dtype_bytes(dtype);
    if (!aligned_to(k, bytes) || !aligned_to(v, bytes) || !aligned_to(start, 4) || !aligned_to(counts, 4)) return fail(SPEC_ERR_BAD_ARG, "%s: a pointer is not aligned to its elements", who);
    const int wide = aligned_to(k, 4 * static_cast<size_t>(bytes)) && aligned_to(v, 4 * static_cast<size_t>(bytes));
    unsigned grid;
    if (!grid_of(static_cast<long long>(batch) * rows * 2 * n_kv_heads, d_head / 8, &grid)) return fail(SPEC_ERR_BAD_ARG, "%s: too many rows for one call", who);
    return with_float(dtype, [&](auto t) {
        using T = decltype(t);
        return with_kv(kv_dtype, [&](auto kv) {
            constexpr int KV = decltype(kv)::value;
            const auto go = [&](auto kernel) {
                return launch_pdl(kernel, dim3(grid), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), cache, pool, scales, start, counts, batch, rows,
                                  static_cast<T*>(k), static_cast<T*>(v), wide);
            };
            return d_head == 64 ? go(kv_read_kernel<T, 64, KV>) : go(kv_read_kernel<T, 128, KV>);
        });
    });
}
