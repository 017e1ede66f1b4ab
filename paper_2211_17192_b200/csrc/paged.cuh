// The paged K,V rows that spec_kv_append writes and spec_kv_read and spec_paged_attention read:
// pool [pages][K, V][kv head][page_size][d_head], scales [pages][K, V][kv head][page_size] fp32 beside 8-bit pools.
#pragma once

#include "fp8_util.cuh"

namespace spec {

struct Paged {
    const int32_t* table;  // [batch][width]: page of every page_size tokens of a sequence
    int pages, width, n_kv, page_shift;
    // Index of a (token, head) row among the pool's rows; negative where the table leads to no page.
    __device__ __forceinline__ long long row(int b, int which, int head, int position) const {
        const int slot = position >> page_shift;
        if (position < 0 || slot >= width) return -1;
        const int page = table[static_cast<size_t>(b) * width + slot];
        if (page < 0 || page >= pages) return -1;
        return (((static_cast<long long>(page) * 2 + which) * n_kv + head) << page_shift) + (position & ((1 << page_shift) - 1));
    }
};

// Checks what all three entry points are given alike; SPEC_OK or a failure.
int check_paged(const char* who, const void* pool, const float* scales, int kv_dtype, int pages, int page_size, int n_kv_heads, int d_head,
                const int32_t* page_table, int max_pages, int batch, Paged* out);

}  // namespace spec
