// The paged KV cache: K and V pools of one layer, [n_pages][page_size][Hkv][128] bf16, and a table that says which page holds which
// positions of a request.  A row of a pool is a token of a page, laid out like a row of the contiguous caches, so a contiguous cache is a
// pool whose table counts upwards.
#pragma once

#include "flux_internal.h"

namespace flux {

struct PageArgs {
    unsigned char *pool[2];          // K, V
    const int32_t *table;            // [B][cols]
    int n_pages, shift, cols;        // page_size = 1 << shift
    // page of position p of request b as the table has it
    __device__ __forceinline__ int entry(int b, int p) const { return table[(size_t)b * cols + (p >> shift)]; }
    __device__ __forceinline__ size_t row(int page, int p) const { return ((size_t)page << shift) + (p & ((1 << shift) - 1)); }
    __device__ __forceinline__ int64_t room() const { return (int64_t)cols << shift; }
};

inline PageArgs page_args(const flux_pages &pg)
{
    PageArgs a;
    a.pool[0] = (unsigned char *)pg.k;
    a.pool[1] = (unsigned char *)pg.v;
    a.table = pg.table;
    a.n_pages = pg.n_pages;
    a.cols = pg.max_pages;
    a.shift = 0;
    while ((1 << a.shift) < pg.page_size) ++a.shift;
    return a;
}

}  // namespace flux
