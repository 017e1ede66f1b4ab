// New tokens' K and V rows into a paged cache in 16 or 8 bits (rotary positions on the way), and cached rows back out.
//
// Both kernels are bound by memory and, at a few rows, by the latency of one dependent chain (start -> page -> row).  A CTA has one
// token, so that its place is found once per thread and its angles are loaded once; a group of d_head / 16 lanes has one row of
// one head at a time: sixteen elements to a lane, so that a pair of a rotation (j, j + d_head / 2) and the largest magnitude of the row
// never leave the group, and nothing goes through shared memory.  (A group of twice as many lanes for every row of every token, with
// divisions in 64 bits and the angles loaded for each row: 2 x 1024 tokens of 48 heads, append and read 21.1 us; so 14.5.)  The
// first row's loads go out beside the chain.
#include <algorithm>

#include "paged.cuh"

namespace spec {
namespace {

constexpr int kAppendThreads = 96;  // (2 x 1024 tokens of 48 heads: 10.8 us; 64 threads 12.7, 128 12.2, 256 16.1)
constexpr int kReadThreads = 128;   // (3.7 us; 96 threads 4.6)

// Elements in the order that the rotation wants: eight at 8 l, eight at 8 l + d / 2.  grid = (tokens, shares of a token's heads).
template <typename T, int D, int KV>
__global__ void __launch_bounds__(kAppendThreads)
kv_append_kernel(const T* q, const T* k, const T* v, long long q_stride, long long k_stride, long long v_stride, int n_heads,
                 const __grid_constant__ Paged cache, void* pool, float* scales, const int32_t* start, const int32_t* counts, int rows,
                 const float2* rope, int rope_positions, T* q_out, int wide) {
    pdl_trigger();
    pdl_wait();
    constexpr int kLanes = D / 16, kGroups = kAppendThreads / kLanes;
    const int items = n_heads + 2 * cache.n_kv;
    const int l = threadIdx.x % kLanes;
    const size_t token = blockIdx.x;
    const int b = blockIdx.x / static_cast<unsigned>(rows), r = blockIdx.x - b * rows;
    // (the lanes of a warp stay together, for the exchanges below: a group past the end goes along with the last item)
    int mine = blockIdx.y * kGroups + threadIdx.x / kLanes;
    float lo[8], hi[8];
    const auto fetch = [&]() {
        const int item = min(mine, items - 1), which = item < n_heads ? 0 : (item - n_heads) / cache.n_kv;
        const T* src = item < n_heads ? q + token * q_stride + item * D
                                      : (which == 0 ? k + token * k_stride : v + token * v_stride) + (item - n_heads - which * cache.n_kv) * D;
        load_row(src + 8 * l, wide, lo);
        load_row(src + 8 * l + D / 2, wide, hi);
    };
    fetch();  // (beside the chain that finds the token's place)
    const int first = start[b];
    if (r >= (counts ? counts[b] : rows) || first < 0 || first > 0x7fffffff - rows) return;
    const int position = first + r;
    if (rope && position >= rope_positions) return;
    const long long at0 = cache.row(b, 0, 0, position);  // of K's first head; its other heads and V lie at fixed distances
    float cosine[8], sine[8];
    if (rope) {
        const float2* cs = rope + static_cast<size_t>(position) * (D / 2) + 8 * l;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 t = cs[i];
            cosine[i] = t.x;
            sine[i] = t.y;
        }
    }
    while (true) {
        const int item = min(mine, items - 1);
        const bool live = mine < items, is_q = item < n_heads;
        const int which = is_q ? 0 : (item - n_heads) / cache.n_kv;
        const int head = is_q ? item : (item - n_heads) - which * cache.n_kv;
        if (rope && (is_q || which == 0)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = lo[i], y = hi[i];
                // (each product and the sum rounded by itself: the same bits as an elementwise program's, so that codes agree)
                lo[i] = __fsub_rn(__fmul_rn(x, cosine[i]), __fmul_rn(y, sine[i]));
                hi[i] = __fadd_rn(__fmul_rn(y, cosine[i]), __fmul_rn(x, sine[i]));
            }
        }
        if (is_q && live) {
            T* out = q_out + (token * n_heads + head) * D + 8 * l;
            store_row(out, wide, lo);
            store_row(out + D / 2, wide, hi);
        }
        const bool write = live && !is_q && at0 >= 0;
        const long long at = at0 + ((static_cast<long long>(which) * cache.n_kv + head) << cache.page_shift);
        if constexpr (KV == SPEC_DTYPE_E4M3 || KV == SPEC_DTYPE_INT8) {
            uint32_t largest = 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) largest = max(largest, max(magnitude(lo[i]), magnitude(hi[i])));
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) largest = max(largest, __shfl_xor_sync(kFullMask, largest, o));
            if (write) {
            const float scale = row_scale(largest, KV == SPEC_DTYPE_E4M3 ? kE4m3Top : kInt8Top), inverse = __fdiv_rn(1.0f, scale);
            const auto codes = [&](const float(&y)[8], int i) {
                if constexpr (KV == SPEC_DTYPE_E4M3) return codes_e4m3(y[i] * inverse, y[i + 1] * inverse) | codes_e4m3(y[i + 2] * inverse, y[i + 3] * inverse) << 16;
                else return codes_int8(y[i] * inverse, y[i + 1] * inverse) | codes_int8(y[i + 2] * inverse, y[i + 3] * inverse) << 16;
            };
            uint2* out = reinterpret_cast<uint2*>(static_cast<uint8_t*>(pool) + at * D) + l;
            out[0] = make_uint2(codes(lo, 0), codes(lo, 4));
            out[D / 16] = make_uint2(codes(hi, 0), codes(hi, 4));
            if (l == 0) scales[at] = scale;
            }
        } else if (write) {
            using E = std::conditional_t<KV == SPEC_DTYPE_BF16, __nv_bfloat16, __half>;
            if constexpr (KV == SPEC_DTYPE_FP16) {  // (finite values past the type's range are held as its largest; infinities stay what they are)
                const auto held = [](float& x) {
                    if (fabsf(x) > 65504.0f && fabsf(x) < INFINITY) x = copysignf(65504.0f, x);
                };
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    held(lo[i]);
                    held(hi[i]);
                }
            }
            E* out = static_cast<E*>(pool) + at * D + 8 * l;
            store_row(out, true, lo);
            store_row(out + D / 2, true, hi);
        }
        mine += gridDim.y * kGroups;
        if (mine - static_cast<int>(threadIdx.x) / kLanes >= items) break;  // (for the whole block)
        fetch();
    }
}

template <typename T, int D, int KV>
__global__ void __launch_bounds__(kReadThreads)
kv_read_kernel(const __grid_constant__ Paged cache, const void* pool, const float* scales, const int32_t* start,
               const int32_t* counts, int rows, T* k, T* v, int wide) {
    pdl_trigger();
    pdl_wait();
    constexpr int kLanes = D / 16, kGroups = kReadThreads / kLanes;
    const int l = threadIdx.x % kLanes;
    const size_t token = blockIdx.x;
    const int b = blockIdx.x / static_cast<unsigned>(rows), r = blockIdx.x - b * rows;
    const int first = start[b];
    if (r >= (counts ? counts[b] : rows) || first < 0 || first > 0x7fffffff - rows) return;
    const long long at0 = cache.row(b, 0, 0, first + r);
    if (at0 < 0) return;
    for (int item = blockIdx.y * kGroups + threadIdx.x / kLanes; item < 2 * cache.n_kv; item += gridDim.y * kGroups) {
        const int which = item / cache.n_kv, head = item - which * cache.n_kv;
        const long long at = at0 + (static_cast<long long>(item) << cache.page_shift);
        T* out = (which == 0 ? k : v) + (token * cache.n_kv + head) * D + 16 * l;
        float y[16];
        if constexpr (KV == SPEC_DTYPE_E4M3 || KV == SPEC_DTYPE_INT8) {
            const uint4 c = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(pool) + at * D)[l];
            const uint32_t words[4] = {c.x, c.y, c.z, c.w};
            const float scale = scales[at];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t byte = words[i / 4] >> (8 * (i % 4)) & 0xffu;
                if constexpr (KV == SPEC_DTYPE_E4M3) {
                    __nv_fp8_e4m3 e;
                    e.__x = static_cast<__nv_fp8_storage_t>(byte);
                    y[i] = static_cast<float>(e) * scale;
                } else {
                    y[i] = static_cast<float>(static_cast<int8_t>(byte)) * scale;
                }
            }
        } else {
            using E = std::conditional_t<KV == SPEC_DTYPE_BF16, __nv_bfloat16, __half>;
            load_row(static_cast<const E*>(pool) + at * D + 16 * l, true, y);
        }
        store_row(out, wide, y);
    }
}

// A token to a CTA; its heads are shared by several where there are few tokens.
dim3 grid_of(int tokens, int items, int lanes, int threads) {
    const int rounds = (items * lanes + threads - 1) / threads;
    return dim3(tokens, std::min(rounds, std::max(1, 1184 / tokens)));
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
    if (n_kv_heads < 1 || n_kv_heads > 1024 || pages < 1 || max_pages < 1 || max_pages > 0x7fffff00 / page_size || batch < 0 || batch > 65535)
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
    const int wide = aligned_to(q, 16) && aligned_to(k, 16) && aligned_to(v, 16) && aligned_to(q_out, 16) && k_stride % 8 == 0 && v_stride % 8 == 0 && (!q || q_stride % 8 == 0);
    if (static_cast<long long>(batch) * rows > 0x7fffffffll) return fail(SPEC_ERR_BAD_ARG, "%s: too many rows for one call", who);
    const dim3 grid = grid_of(batch * rows, heads + 2 * n_kv_heads, d_head / 16, kAppendThreads);
    return with_float(dtype, [&](auto t) {
        using T = decltype(t);
        return with_kv(kv_dtype, [&](auto kv) {
            constexpr int KV = decltype(kv)::value;
            const auto go = [&](auto kernel) {
                return launch_pdl(kernel, grid, dim3(kAppendThreads), 0, static_cast<cudaStream_t>(stream), static_cast<const T*>(q), static_cast<const T*>(k),
                                  static_cast<const T*>(v), static_cast<long long>(q_stride), static_cast<long long>(k_stride), static_cast<long long>(v_stride),
                                  heads, cache, pool, scales, start, counts, rows, reinterpret_cast<const float2*>(rope), rope_positions, static_cast<T*>(q_out), wide);
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
    const int wide = aligned_to(k, 16) && aligned_to(v, 16);
    if (static_cast<long long>(batch) * rows > 0x7fffffffll) return fail(SPEC_ERR_BAD_ARG, "%s: too many rows for one call", who);
    const dim3 grid = grid_of(batch * rows, 2 * n_kv_heads, d_head / 16, kReadThreads);
    return with_float(dtype, [&](auto t) {
        using T = decltype(t);
        return with_kv(kv_dtype, [&](auto kv) {
            constexpr int KV = decltype(kv)::value;
            const auto go = [&](auto kernel) {
                return launch_pdl(kernel, grid, dim3(kReadThreads), 0, static_cast<cudaStream_t>(stream), cache, pool, scales, start, counts, rows,
                                  static_cast<T*>(k), static_cast<T*>(v), wide);
            };
            return d_head == 64 ? go(kv_read_kernel<T, 64, KV>) : go(kv_read_kernel<T, 128, KV>);
        });
    });
}
