// What the calls on a paged cache share: the cache and a batch of entries as kernels take them, and how an entry is read.
#pragma once
#include "dsla_internal.h"

namespace dsla {

struct CacheArgs {
    int32_t *table, *lens, *refs, *status;
    int n_pages, page_log2, H_kv, d, n_seqs, max_pages;
};
struct BatchArgs {
    const int32_t *cu, *row;
    int32_t *start;
    int B, total;
};

// One entry as the batch describes it: its tokens cu .. cu + n - 1 and its row of the cache.  ok = false: out of range.
struct Entry {
    int cu, n, row;
    bool ok;
};

namespace {

__device__ __forceinline__ Entry read_entry(const BatchArgs &x, const CacheArgs &c, int b)
{
    Entry e;
    e.cu = x.cu ? x.cu[b] : b;
    const int end = x.cu ? x.cu[b + 1] : b + 1;
    e.row = x.row ? x.row[b] : b;
    e.ok = e.cu >= 0 && end >= e.cu && end <= x.total && e.row >= 0 && e.row < c.n_seqs;
    e.n = e.ok ? end - e.cu : 0;
    return e;
}

// Tokens that a row of the table has columns for.
__device__ __forceinline__ long long row_room(const CacheArgs &c) { return static_cast<long long>(c.max_pages) << c.page_log2; }

__device__ __forceinline__ void report(int32_t *status, int bits)
{
    if (status) atomicOr(status, bits);
}

__device__ __forceinline__ int pages_of(long long tokens, int page_log2)
{
    return static_cast<int>((tokens + (1 << page_log2) - 1) >> page_log2);
}

// The page of token t of a row, or -1 where the table gives none that exists.
__device__ __forceinline__ int page_of(const CacheArgs &c, int row, int t)
{
    const int p = c.table[static_cast<size_t>(row) * c.max_pages + (t >> c.page_log2)];
    return p >= 0 && p < c.n_pages ? p : -1;
}

inline CacheArgs args_of(const dsla_cache &c)
{
    return CacheArgs{c.table, c.lens, c.refs, c.status, c.n_pages, __builtin_ctz(c.page), c.H_kv, c.d, c.n_seqs, c.max_pages};
}
inline BatchArgs args_of(const dsla_batch &x) { return BatchArgs{x.cu, x.row, x.start, x.B, static_cast<int>(x.total)}; }

}  // namespace
}  // namespace dsla
