// A paged key-value cache as the kernels see it (psf_cache.hip, psf_paged.hip).
#ifndef PSF_CACHE_H
#define PSF_CACHE_H

#include "psf_internal.h"

namespace psf {

struct Cache {
    int pages, page, kv_heads, d, seqs, cols;
    bool bf16;
    size_t row_bytes() const { return (size_t)d * (bf16 ? 2 : 4); }
    size_t page_bytes() const { return (size_t)kv_heads * page * row_bytes(); }
};

psf_status make_cache(const psf_cache_desc *desc, Cache *out);

// x / by for 0 <= x < 2^31 by one multiplication: with 2^(l-1) < by <= 2^l and m = ceil(2^(31+l) / by) < 2^32 the
// product x m / 2^(31+l) exceeds x / by by less than 2^31 (m - 2^(31+l) / by) / 2^(31+l) < 1 / by.
struct FastDiv {
    uint32_t by, mul, shift;
    __device__ __forceinline__ uint32_t div(uint32_t x) const { return by == 1 ? x : __umulhi(x, mul) >> shift; }
};
inline FastDiv fast_div(uint32_t by)
{
    FastDiv f{by, 0, 0};
    if (by <= 1) return f;
    uint32_t l = 0;
    while ((1ull << l) < by) ++l;                         // l >= 1
    f.mul = (uint32_t)(((1ull << (31 + l)) + by - 1) / by);
    f.shift = l - 1;
    return f;
}

// Page of position `at` of a sequence, -1 where the table has none that lies in the pool.
__device__ __forceinline__ int page_of(const int32_t *table_row, int col, int cols, int pages)
{
    if ((unsigned)col >= (unsigned)cols) return -1;
    const int p = table_row[col];
    return (unsigned)p < (unsigned)pages ? p : -1;
}

}  // namespace psf
#endif
