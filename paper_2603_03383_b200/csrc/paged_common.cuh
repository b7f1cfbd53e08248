// Pages of a K/V cache as the kernels see them.
#pragma once
#include "common.cuh"

namespace mtv {

struct PagedRef {
    const int32_t *table;      // [B][max_pages]
    int64_t stride_page, stride_h, stride_t;   // elements
    int max_pages, n_pages, page_shift;

    // n rows behind L fit what the table holds
    __device__ __forceinline__ bool fits(int L, int n) const {
        return L >= 0 && n >= 0 && (int64_t)L + n <= ((int64_t)max_pages << page_shift);
    }
    // Offset of slot s (head 0) in a pool, for a slot that fits; -1 where the table holds no page of the pool.
    __device__ __forceinline__ int64_t row(int b, int s) const {
        const int page = table[(int64_t)b * max_pages + (s >> page_shift)];
        if (page < 0 || page >= n_pages) return -1;
        return page * stride_page + (s & ((1 << page_shift) - 1)) * stride_t;
    }
    // One warp: MTV_OK, or why rows [L, L + n) of sequence b cannot all be reached.
    __device__ __forceinline__ int check(int b, int L, int n, int lane) const {
        if (!fits(L, n)) return MTV_ERR_CAPACITY;
        bool ok = true;
        const int end = n ? (int)(((int64_t)L + n - 1) >> page_shift) + 1 : 0;
        for (int i = (L >> page_shift) + lane; i < end; i += 32) {
            const int page = table[(int64_t)b * max_pages + i];
            ok = ok && page >= 0 && page < n_pages;
        }
        return __all_sync(0xffffffffu, ok) ? MTV_OK : MTV_ERR_BOUNDS;
    }
};

// MTV_OK, or what such pages are refused with.
static inline int paged_ref(PagedRef &r, const mtv_pool_layout *pool, const int32_t *page_table, int max_pages, int D) {
    if (!pool || !page_table || max_pages < 1 || pool->n_pages < 1) return MTV_ERR_INVALID_ARG;
    if (pool->page_size < 16 || pool->page_size > 65536 || (pool->page_size & (pool->page_size - 1))) return MTV_ERR_UNSUPPORTED_SHAPE;
    if (pool->stride_page % 8 || pool->stride_h % 8 || pool->stride_t % 8 || pool->stride_t < D || pool->stride_h < D || pool->stride_page < D)
        return MTV_ERR_INVALID_ARG;
    r.table = page_table;
    r.stride_page = pool->stride_page; r.stride_h = pool->stride_h; r.stride_t = pool->stride_t;
    r.max_pages = max_pages; r.n_pages = pool->n_pages;
    r.page_shift = 0;
    while ((1 << r.page_shift) < pool->page_size) ++r.page_shift;
    // slots are counted in 32 bits
    if (((int64_t)max_pages << r.page_shift) > 0x7fffff00ll) return MTV_ERR_UNSUPPORTED_SHAPE;
    return MTV_OK;
}

}  // namespace mtv
