// The book-keeping of a paged key/value cache (include/dsla.h: dsla_cache) and the moves of pages and rows that follow from it.
//
// State is the table, the lengths and the reference counts only; a page is free where its count is zero, and new pages are
// the lowest free ones in ascending order.  The free set has no order of its own, so ends, forks and copies may go through
// atomics in any order and every call still has one result.  What has to be in order (which entry gets which page) is done
// by one workgroup with prefix sums; what moves bytes is done by the whole chip, from lists that this workgroup leaves in
// the workspace.  The host knows none of the numbers: lists have their lengths beside them on the device.
#include "paged_common.h"

namespace dsla {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;

// A page (or its first rows) to copy, in every pool.
struct Move {
    int32_t src, dst, rows, pad;
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
struct Pools {
    char *p[DSLA_MAX_POOLS];
};

__global__ __launch_bounds__(256) void cache_init_kernel(CacheArgs c)
{
    const size_t entries = static_cast<size_t>(c.n_seqs) * c.max_pages, step = static_cast<size_t>(gridDim.x) * 256;
    const size_t at = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x;
    for (size_t i = at; i < entries; i += step) c.table[i] = -1;
    for (size_t i = at; i < static_cast<size_t>(c.n_pages); i += step) c.refs[i] = 0;
    for (size_t i = at; i < static_cast<size_t>(c.n_seqs); i += step) c.lens[i] = 0;
}

// Exclusive sum over the workgroup; *total: of all.  Called by every thread.
__device__ __forceinline__ long long block_prefix(long long x, long long *s_wave, long long *total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    long long sum = x;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const long long y = __shfl_up(sum, off);
        if (lane >= off) sum += y;
    }
    __syncthreads();   // (the last call's sums are read)
    if (lane == 63) s_wave[wave] = sum;
    __syncthreads();
    long long before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) {
        if (w < wave) before += s_wave[w];
        all += s_wave[w];
    }
    *total = all;
    return before + sum - x;
}

// Where a wavefront of the planning workgroup looks for pages: a run of whole wavefronts' worth; the first `idle` look for none.
__device__ __forceinline__ void wave_pages(int n_pages, int idle, int *from, int *to)
{
    const int rows = (n_pages + 63) / 64, waves = kPlanWaves - idle, wave = static_cast<int>(threadIdx.x >> 6) - idle;
    const long long per = (rows + waves - 1) / waves * 64ll, a = per * wave, b = a + per;
    *from = wave < 0 ? 0 : static_cast<int>(a < n_pages ? a : n_pages);
    *to = wave < 0 ? 0 : static_cast<int>(b < n_pages ? b : n_pages);
}
// f(first page, the reference count of page first + lane or -1 past the end) for 64 pages after 64; until f returns false.  The loads of kBatch
// of them stand together, but each is conditional and the compiler waits for each in its branch: one is in flight, and long pools are bound by
// that (64 new pages, the last ones of 20000 / 131072 / 2^20: 14 / 55 / 414 us, events around the launch, of which about 4 are there without any work).
constexpr int kBatch = 4;
template <class F>
__device__ __forceinline__ void each_page(const int32_t *refs, int from, int to, F &&f)
{
    const int lane = threadIdx.x & 63;
    for (int p = from; p < to; p += 64 * kBatch) {
        int r[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) r[u] = p + 64 * u + lane < to ? refs[p + 64 * u + lane] : -1;
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (p + 64 * u < to && !f(p + 64 * u, r[u])) return;
    }
}

// What an entry asks for: its row's length, the first column that gets a new page, and how many.  at = -1: it is left out.
struct Need {
    int len, at;
    long long pages;
};
__device__ __forceinline__ Need need_of(const CacheArgs &c, const Entry &e, bool again, int *bits)
{
    Need w{e.ok ? c.lens[e.row] : -1, -1, 0};
    if (!e.ok || again || w.len < 0 || w.len > row_room(c)) {
        *bits |= DSLA_STATUS_CACHE_ENTRY;
    } else if (static_cast<long long>(w.len) + e.n > row_room(c)) {
        *bits |= DSLA_STATUS_CACHE_FULL;
    } else {
        const bool partial = (w.len & ((1 << c.page_log2) - 1)) != 0 && e.n > 0;
        const int last = partial ? page_of(c, e.row, w.len - 1) : 0;
        if (last < 0) {
            *bits |= DSLA_STATUS_CACHE_ENTRY;
        } else {
            w.at = pages_of(w.len, c.page_log2) - (partial && c.refs[last] > 1);
            w.pages = pages_of(static_cast<long long>(w.len) + e.n, c.page_log2) - w.at;
        }
    }
    return w;
}
// An entry that is served, with `before` pages ahead of it: its length, and its shared page that is not full onto the list.
__device__ __forceinline__ void serve(const CacheArgs &c, const Entry &e, const Need &w, int before, const int32_t *fresh, Move *moves, int *s_moves)
{
    if (w.pages > 0 && w.at < pages_of(w.len, c.page_log2)) {
        const int old = page_of(c, e.row, w.len - 1);
        moves[atomicAdd(s_moves, 1)] = Move{old, fresh[before], w.len & ((1 << c.page_log2) - 1), 0};
        atomicSub(&c.refs[old], 1);
    }
    c.lens[e.row] = w.len + e.n;
}
// The new pages into the table: page number r of all belongs to the last entry that has at most r pages ahead of it.
__device__ __forceinline__ void place(const CacheArgs &c, const BatchArgs &x, const int32_t *before, const int32_t *first, const int32_t *fresh, int granted)
{
    for (int r = threadIdx.x; r < granted; r += kPlanThreads) {
        int lo = 0, hi = x.B;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (before[mid] <= r) lo = mid;
            else hi = mid;
        }
        const int row = x.row ? x.row[lo] : lo;
        c.table[static_cast<size_t>(row) * c.max_pages + first[lo] + (r - before[lo])] = fresh[r];
        c.refs[fresh[r]] = 1;
    }
}

// Room for the entries' tokens.  Workspace: claim[n_seqs], the first entry that names a row; before[B], the pages that the entries ahead
// need; first[B], the first column that gets a new page; fresh[n_pages], the free pages in ascending order; moves[B] and their number.
__global__ __launch_bounds__(kPlanThreads) void cache_extend_kernel(CacheArgs c, BatchArgs x, int32_t *claim, int32_t *before, int32_t *first,
                                                                    int32_t *fresh, Move *moves, int32_t *n_moves)
{
    __shared__ long long s_wave[kPlanWaves];
    __shared__ int s_found[kPlanWaves], s_granted, s_moves;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (tid == 0) s_granted = s_moves = 0;
    for (int b = tid; b < x.B; b += kPlanThreads) {
        const Entry e = read_entry(x, c, b);
        if (e.ok) claim[e.row] = 0x7fffffff;
    }
    __syncthreads();
    for (int b = tid; b < x.B; b += kPlanThreads) {
        const Entry e = read_entry(x, c, b);
        if (e.ok) atomicMin(&claim[e.row], b);
    }
    __syncthreads();

    long long wanted = 0;
    int bits = 0;
    for (int b0 = 0; b0 < x.B; b0 += kPlanThreads) {
        const int b = b0 + tid;
        Need w{0, -1, 0};
        if (b < x.B) {
            const Entry e = read_entry(x, c, b);
            w = need_of(c, e, e.ok && claim[e.row] != b, &bits);
        }
        long long sum;
        const long long mine = wanted + block_prefix(w.pages, s_wave, &sum);
        if (b < x.B) {
            before[b] = static_cast<int32_t>(mine < 0x7fffffff ? mine : 0x7fffffff);
            first[b] = w.at;
        }
        wanted += sum;
    }

    // the lowest free pages, as many as are wanted
    int from, to, found = 0;
    wave_pages(c.n_pages, 0, &from, &to);
    if (wanted > 0)
        each_page(c.refs, from, to, [&](int, int r) {
            found += __popcll(__ballot(r == 0));
            return true;
        });
    if (lane == 0) s_found[wave] = found;
    __syncthreads();
    int rank = 0, all = 0;
    for (int w = 0; w < kPlanWaves; ++w) {
        if (w < wave) rank += s_found[w];
        all += s_found[w];
    }
    if (found > 0 && rank < wanted)
        each_page(c.refs, from, to, [&](int p, int r) {
            const unsigned long long m = __ballot(r == 0);
            if (r == 0) fresh[rank + __popcll(m & ((1ull << lane) - 1))] = p + lane;
            rank += __popcll(m);
            return rank < wanted;
        });
    __syncthreads();

    for (int b = tid; b < x.B; b += kPlanThreads) {
        int start = -1;
        if (first[b] >= 0) {
            const Entry e = read_entry(x, c, b);
            Need w{c.lens[e.row], first[b], 0};
            w.pages = pages_of(static_cast<long long>(w.len) + e.n, c.page_log2) - w.at;
            if (w.pages > 0 && before[b] + w.pages > all) {
                bits |= DSLA_STATUS_CACHE_FULL;
            } else {
                start = w.len;
                if (w.pages > 0) atomicMax(&s_granted, static_cast<int>(before[b] + w.pages));
                serve(c, e, w, before[b], fresh, moves, &s_moves);
            }
        }
        x.start[b] = start;
    }
    if (bits) report(c.status, bits);
    __syncthreads();
    place(c, x, before, first, fresh, s_granted);
    if (tid == 0) *n_moves = s_moves;
}

// The same for up to kFew entries and kFewPages pages, as decoding has them: bound by the chain of dependent reads, which is cut short, and by the
// scan of the counts.  The
// first wavefronts look at the entries while the others look for free pages (once: which are free stays in LDS as bits), an
// entry's thread keeps what it read, and one that names a row again finds out by looking at the rows of those ahead.  The kernel above
// and this one (us): 64 requests of which some need one of 20000 pages 9.2 / 8.7, 56 branches that all copy 10.4 / 8.2, 16 requests of up
// to 15 new pages 7.8 / 5.1.
constexpr int kFew = 256, kFewWaves = kFew / 64, kFewPages = 131072;
__global__ __launch_bounds__(kPlanThreads) void cache_extend_few_kernel(CacheArgs c, BatchArgs x, int32_t *fresh, Move *moves, int32_t *n_moves)
{
    __shared__ unsigned long long s_free[kFewPages / 64];
    __shared__ __align__(16) int32_t s_row[kFew];
    __shared__ int32_t s_before[kFew], s_first[kFew];
    __shared__ __align__(16) int s_need[kFewWaves];
    __shared__ int s_found[kPlanWaves], s_granted, s_moves;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (tid == 0) s_granted = s_moves = 0;
    Entry e{0, 0, 0, false};
    Need w{0, -1, 0};
    int bits = 0, from = 0, to = 0, found = 0;
    if (wave < kFewWaves) {
        if (tid < x.B) e = read_entry(x, c, tid);
        s_row[tid] = e.ok ? e.row : -1;
    } else {
        wave_pages(c.n_pages, kFewWaves, &from, &to);
        each_page(c.refs, from, to, [&](int p, int r) {
            const unsigned long long m = __ballot(r == 0);
            if (lane == 0) s_free[p / 64] = m;
            found += __popcll(m);
            return true;
        });
    }
    if (lane == 0) s_found[wave] = found;
    __syncthreads();
    if (tid < x.B) {
        int same = 0;
        if (x.row)
#pragma unroll 2
            for (int o = 0; o < x.B; o += 4) {   // (rows behind the last entry are -1)
                const int4 r = *reinterpret_cast<const int4 *>(s_row + o);
                same |= ((r.x == e.row) & (o < tid)) | ((r.y == e.row) & (o + 1 < tid)) | ((r.z == e.row) & (o + 2 < tid)) | ((r.w == e.row) & (o + 3 < tid));
            }
        w = need_of(c, e, same != 0, &bits);
    }
    // sums in 32 bits: what no pool has counts as a page more than there are
    const int pages = w.pages <= c.n_pages ? static_cast<int>(w.pages) : c.n_pages + 1;
    int sum = pages;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(sum, off);
        sum += lane >= off ? y : 0;
    }
    if (lane == 63 && wave < kFewWaves) s_need[wave] = sum;
    __syncthreads();
    const int4 need = *reinterpret_cast<const int4 *>(s_need);
    const int before = sum - pages + (wave > 0 ? need.x : 0) + (wave > 1 ? need.y : 0) + (wave > 2 ? need.z : 0), wanted = need.x + need.y + need.z + need.w;
    if (tid < x.B) {
        s_before[tid] = before;
        s_first[tid] = w.at;
    }
    int rank = lane < kPlanWaves ? s_found[lane] : 0;
#pragma unroll
    for (int off = 1; off < kPlanWaves; off <<= 1) {
        const int y = __shfl_up(rank, off);
        rank += lane >= off ? y : 0;
    }
    const int all = __builtin_amdgcn_readlane(rank, kPlanWaves - 1);
    rank = __builtin_amdgcn_readlane(rank, __builtin_amdgcn_readfirstlane(wave)) - found;
    for (int p = from; p < to && rank < wanted; p += 64) {
        const unsigned long long m = s_free[p / 64];
        if (m >> lane & 1) fresh[rank + __popcll(m & ((1ull << lane) - 1))] = p + lane;
        rank += __popcll(m);
    }
    __syncthreads();
    if (tid < x.B) {
        const bool served = w.at >= 0 && (pages == 0 || before + pages <= all);
        if (w.at >= 0 && !served) bits |= DSLA_STATUS_CACHE_FULL;
        if (served && pages > 0) atomicMax(&s_granted, before + pages);
        if (served) serve(c, e, w, before, fresh, moves, &s_moves);
        x.start[tid] = served ? w.len : -1;
    }
    if (bits) report(c.status, bits);
    __syncthreads();
    place(c, x, s_before, s_first, fresh, s_granted);
    if (tid == 0) *n_moves = s_moves;
}

// The pages of a list, or their first rows, in every pool.  A wavefront takes one head of one page in one pool: its rows are
// consecutive bytes.  Bound by memory; stores carry the non-temporal hint, loads do not, since branches of one request copy the same
// rows: 56 branches of 8 requests in 32 pools (293 MB) 65 us without a hint, 65 with it on the loads, 44 on the stores, 61 on both;
// half of 160 pages to the front of 32 pools, twice (1.07 GB) 249, 217, 221, 231.
__global__ __launch_bounds__(1024) void cache_copy_kernel(const Move *moves, const int32_t *n_moves, int n_pools, int H_kv, int page, int row_bytes,
                                                          Pools pools)
{
    const int lane = threadIdx.x & 63;
    const long long items = static_cast<long long>(*n_moves) * n_pools * H_kv;
    const size_t head_bytes = static_cast<size_t>(page) * row_bytes;
    for (long long i = static_cast<long long>(blockIdx.x) * 16 + (threadIdx.x >> 6); i < items; i += static_cast<long long>(gridDim.x) * 16) {
        const int h = static_cast<int>(i % H_kv);
        const long long j = i / H_kv;
        const Move m = moves[j / n_pools];
        char *pool = pools.p[j % n_pools];
        const u32x4 *src = reinterpret_cast<const u32x4 *>(pool + (static_cast<size_t>(m.src) * H_kv + h) * head_bytes);
        u32x4 *dst = reinterpret_cast<u32x4 *>(pool + (static_cast<size_t>(m.dst) * H_kv + h) * head_bytes);
        const int n = m.rows * row_bytes / 16;
        int t = lane;
        for (; t + 3 * 64 < n; t += 4 * 64) {
            u32x4 x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = src[t + 64 * u];
#pragma unroll
            for (int u = 0; u < 4; ++u) __builtin_nontemporal_store(x[u], dst + t + 64 * u);
        }
        for (; t < n; t += 64) dst[t] = src[t];
    }
}

// A sequence is cut to `keep` tokens: by one wavefront, which waits for the numbers of 64 pages before it asks for the next.  (Ends, forks and cuts of up
// to some hundred pages are a launch and two dependent reads, 2 to 5 us; rows of 8192 pages are ended or forked in 42.)
__device__ __forceinline__ void cut_row(const CacheArgs &c, int row, int len, int keep)
{
    const int have = pages_of(len, c.page_log2);
    for (int col = pages_of(keep, c.page_log2) + static_cast<int>(threadIdx.x & 63); col < have; col += 64) {
        int32_t *entry = c.table + static_cast<size_t>(row) * c.max_pages + col;
        const int p = *entry;
        if (p >= 0 && p < c.n_pages) atomicSub(&c.refs[p], 1);
        else report(c.status, DSLA_STATUS_CACHE_ENTRY);
        *entry = -1;
    }
    if ((threadIdx.x & 63) == 0) c.lens[row] = keep;
}

__global__ __launch_bounds__(64) void cache_truncate_kernel(CacheArgs c, const int32_t *new_lens)
{
    const int s = blockIdx.x, keep = new_lens[s], len = c.lens[s];
    if (keep < 0 || keep >= len) return;
    if (len > row_room(c)) {
        if (threadIdx.x == 0) report(c.status, DSLA_STATUS_CACHE_ENTRY);
        return;
    }
    cut_row(c, s, len, keep);
}

__global__ __launch_bounds__(64) void cache_fork_kernel(CacheArgs c, const int32_t *parent)
{
    const int s = blockIdx.x, from = parent[s];
    if (from < 0) return;
    const int len = from < c.n_seqs && parent[from] < 0 ? c.lens[from] : -1;   // (a parent that is no child: its row is not written)
    if (len < 0 || len > row_room(c) || c.lens[s] != 0) {
        if (threadIdx.x == 0) report(c.status, DSLA_STATUS_CACHE_ENTRY);
        return;
    }
    const int have = pages_of(len, c.page_log2);
    for (int col = threadIdx.x; col < have; col += 64) {
        const int p = c.table[static_cast<size_t>(from) * c.max_pages + col];
        if (p >= 0 && p < c.n_pages) atomicAdd(&c.refs[p], 1);
        else report(c.status, DSLA_STATUS_CACHE_ENTRY);
        c.table[static_cast<size_t>(s) * c.max_pages + col] = p;
    }
    if (threadIdx.x == 0) c.lens[s] = len;
}

// The length that entry b is cut to once its accepted tokens are at the front, or -1: it stays as it is.  By a wavefront; nothing that it
// reads is changed before cache_accept_cut_kernel.
__device__ __forceinline__ int accepted_length(const CacheArgs &c, const BatchArgs &x, const Entry &e, int b, const int32_t *path, const int32_t *n_accepted, bool tell)
{
    const int start = x.start[b], n = n_accepted[b], lane = threadIdx.x & 63;
    const bool asked = n >= 0 && !(e.ok && start < 0);
    bool again = false;
    if (x.row)
        for (int o = lane; o < b; o += 64)
            if (x.row[o] == e.row && x.start[o] >= 0) again |= read_entry(x, c, o).ok;
    again = __ballot(again) != 0;
    bool good = asked && e.ok && !again && n <= e.n && static_cast<long long>(start) + e.n <= row_room(c) && c.lens[e.row] == start + e.n;
    if (good) {
        for (int i = lane; i < n; i += 64) {
            const int p = path[e.cu + i];
            if (p < 0 || p >= e.n || (i > 0 && path[e.cu + i - 1] >= p)) {
                good = false;
            } else if (p != i) {
                const int from = page_of(c, e.row, start + p), to = page_of(c, e.row, start + i);
                if (from < 0 || to < 0 || c.refs[to] != 1) good = false;
            }
        }
        good = __ballot(!good) == 0;
    }
    if (tell && lane == 0 && asked && !good) report(c.status, DSLA_STATUS_CACHE_ENTRY);
    return good ? start + n : -1;
}

// Accepted tokens to the front.  A wavefront takes one head of one entry in one pool; the first of an entry's leaves the verdict.
// path[i] >= i and ascending, so no row is written that a later one of the path still has to be read from: groups of rows go in order,
// and within a group all are read before any is written.
__global__ __launch_bounds__(256) void cache_accept_rows_kernel(CacheArgs c, BatchArgs x, const int32_t *path, const int32_t *n_accepted, int32_t *verdict,
                                                                int n_pools, int row_bytes, Pools pools)
{
    const int lane = threadIdx.x & 63, heads = n_pools > 0 ? n_pools * c.H_kv : 1;   // wavefronts of an entry
    const long long item = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (item >= static_cast<long long>(x.B) * heads) return;
    const int b = static_cast<int>(item / heads), which = static_cast<int>(item % heads);
    const Entry e = read_entry(x, c, b);
    const int length = accepted_length(c, x, e, b, path, n_accepted, which == 0);
    if (which == 0 && lane == 0) verdict[b] = length;
    if (length < 0 || n_pools == 0) return;
    const int h = which % c.H_kv, start = x.start[b], n = length - start, page = 1 << c.page_log2;
    char *pool = pools.p[which / c.H_kv];
    const int lanes = row_bytes / 16, rows = 64 / lanes;   // lanes of a row; rows of a group
    for (int i0 = 0; i0 < n; i0 += rows) {
        const int i = i0 + lane / lanes;
        const int p = i < n ? path[e.cu + i] : i;
        if (p != i) {
            const int t = start + p, u = start + i;
            const uint4 row = reinterpret_cast<const uint4 *>(pool + ((static_cast<size_t>(page_of(c, e.row, t)) * c.H_kv + h) * page + (t & (page - 1))) * row_bytes)[lane % lanes];
            reinterpret_cast<uint4 *>(pool + ((static_cast<size_t>(page_of(c, e.row, u)) * c.H_kv + h) * page + (u & (page - 1))) * row_bytes)[lane % lanes] = row;
        }
    }
}

__global__ __launch_bounds__(64) void cache_accept_cut_kernel(CacheArgs c, BatchArgs x, const int32_t *verdict)
{
    const int b = blockIdx.x;
    if (verdict[b] < 0) return;
    const Entry e = read_entry(x, c, b);
    cut_row(c, e.row, x.start[b] + e.n, verdict[b]);
}

// Pages in use to the front: the list of moves and where every page goes.  One workgroup reads the counts three times, 3.4 to 5 us for some
// hundred pages, beside the copy of what moves.
__global__ __launch_bounds__(kPlanThreads) void cache_compact_kernel(CacheArgs c, int32_t *to_page, Move *moves, int32_t *n_moves, int32_t *n_live)
{
    __shared__ int s_live[kPlanWaves], s_src[kPlanWaves], s_dst[kPlanWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int from, to, live = 0;
    wave_pages(c.n_pages, 0, &from, &to);
    each_page(c.refs, from, to, [&](int, int r) {
        live += __popcll(__ballot(r > 0));
        return true;
    });
    if (lane == 0) s_live[wave] = live;
    __syncthreads();
    int L = 0;
    for (int w = 0; w < kPlanWaves; ++w) L += s_live[w];
    // in use from page L on, and free below it: as many of the ones as of the others
    int src = 0, dst = 0;
    each_page(c.refs, from, to, [&](int p, int r) {
        const bool in = p + lane < to, used = r > 0;
        src += __popcll(__ballot(used && p + lane >= L));
        dst += __popcll(__ballot(in && !used && p + lane < L));
        return true;
    });
    if (lane == 0) {
        s_src[wave] = src;
        s_dst[wave] = dst;
    }
    __syncthreads();
    src = dst = 0;
    int n = 0;
    for (int w = 0; w < kPlanWaves; ++w) {
        if (w < wave) {
            src += s_src[w];
            dst += s_dst[w];
        }
        n += s_src[w];
    }
    each_page(c.refs, from, to, [&](int p, int r) {
        const bool in = p + lane < to, used = r > 0;
        const bool moves_away = used && p + lane >= L, hole = in && !used && p + lane < L;
        const unsigned long long ms = __ballot(moves_away), md = __ballot(hole), low = (1ull << lane) - 1;
        if (in && !used && p + lane >= L) to_page[p + lane] = p + lane;   // (a table that names a page no one counts keeps its number)
        if (moves_away) moves[src + __popcll(ms & low)].src = p + lane;
        if (hole) {
            Move &m = moves[dst + __popcll(md & low)];
            m.dst = p + lane;
            m.rows = 1 << c.page_log2;
        }
        src += __popcll(ms);
        dst += __popcll(md);
        return true;
    });
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        const Move m = moves[i];
        to_page[m.src] = m.dst;
        c.refs[m.dst] = c.refs[m.src];
        c.refs[m.src] = 0;
    }
    if (threadIdx.x == 0) {
        *n_moves = n;
        *n_live = L;
    }
}

__global__ __launch_bounds__(256) void cache_rename_kernel(CacheArgs c, const int32_t *to_page, const int32_t *n_live)
{
    const int s = blockIdx.x, len = c.lens[s], L = *n_live;
    const int have = len > 0 && len <= row_room(c) ? pages_of(len, c.page_log2) : 0;
    for (int col = threadIdx.x; col < have; col += 256) {
        int32_t *entry = c.table + static_cast<size_t>(s) * c.max_pages + col;
        if (*entry >= L && *entry < c.n_pages) *entry = to_page[*entry];
    }
}

size_t up16(size_t n) { return (n + 15) / 16 * 16; }

// Where the parts of the workspace are.
struct Scratch {
    int32_t *n_moves, *claim, *before, *first, *fresh;
    Move *moves;
    size_t bytes;
};
Scratch scratch_of(const dsla_cache &c, int B, void *workspace)
{
    char *at = static_cast<char *>(workspace);
    const auto take = [&](size_t n) {
        char *p = at;
        at += up16(n);
        return p;
    };
    Scratch s;
    s.n_moves = reinterpret_cast<int32_t *>(take(sizeof(int32_t)));
    s.claim = reinterpret_cast<int32_t *>(take(sizeof(int32_t) * c.n_seqs));
    s.before = reinterpret_cast<int32_t *>(take(sizeof(int32_t) * B));
    s.first = reinterpret_cast<int32_t *>(take(sizeof(int32_t) * B));
    s.fresh = reinterpret_cast<int32_t *>(take(sizeof(int32_t) * c.n_pages));
    const int most = c.n_pages > B ? c.n_pages : B;
    s.moves = reinterpret_cast<Move *>(take(sizeof(Move) * most));
    s.bytes = static_cast<size_t>(at - static_cast<char *>(workspace));
    return s;
}

Pools pools_of(int n, void *const *pools)
{
    Pools p;
    for (int i = 0; i < DSLA_MAX_POOLS; ++i) p.p[i] = i < n ? static_cast<char *>(pools[i]) : nullptr;
    return p;
}
int row_bytes(const dsla_cache &c) { return c.d * (c.dtype == DSLA_BF16 ? 2 : 4); }

// Copies run with the chip full; the number of workgroups does not depend on the number of moves, which the host does not know.
constexpr int kCopyGroups = 512;

hipError_t launch_moves(const dsla_cache &c, const Scratch &s, int n_pools, void *const *pools, hipStream_t stream)
{
    if (n_pools == 0) return hipSuccess;
    ProfileScope ps(DSLA_KERNEL_CACHE, stream);
    DSLA_LAUNCH(ps, cache_copy_kernel, dim3(kCopyGroups), dim3(1024), 0, stream, static_cast<const Move *>(s.moves),
                static_cast<const int32_t *>(s.n_moves), n_pools, c.H_kv, c.page, row_bytes(c), pools_of(n_pools, pools));
    return hipGetLastError();
}

}  // namespace

size_t cache_workspace_bytes(const dsla_cache &c, int B) { return scratch_of(c, B, nullptr).bytes; }

hipError_t launch_cache_init(const dsla_cache &c, hipStream_t stream)
{
    const size_t entries = static_cast<size_t>(c.n_seqs) * c.max_pages, most = entries > static_cast<size_t>(c.n_pages) ? entries : c.n_pages;
    const size_t groups = (most + 255) / 256;
    ProfileScope ps(DSLA_KERNEL_CACHE, stream);
    DSLA_LAUNCH(ps, cache_init_kernel, dim3(static_cast<unsigned>(groups < 2048 ? groups : 2048)), dim3(256), 0, stream, args_of(c));
    return hipGetLastError();
}

hipError_t launch_cache_extend(const dsla_cache &c, const dsla_batch &x, int n_pools, void *const *pools, void *workspace, hipStream_t stream)
{
    const Scratch s = scratch_of(c, x.B, workspace);
    {
        ProfileScope ps(DSLA_KERNEL_CACHE, stream);
        if (x.B <= kFew && c.n_pages <= kFewPages)
            DSLA_LAUNCH(ps, cache_extend_few_kernel, dim3(1), dim3(kPlanThreads), 0, stream, args_of(c), args_of(x), s.fresh, s.moves, s.n_moves);
        else
            DSLA_LAUNCH(ps, cache_extend_kernel, dim3(1), dim3(kPlanThreads), 0, stream, args_of(c), args_of(x), s.claim, s.before, s.first, s.fresh,
                        s.moves, s.n_moves);
    }
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_moves(c, s, n_pools, pools, stream);
}

hipError_t launch_cache_fork(const dsla_cache &c, const int32_t *parent, hipStream_t stream)
{
    ProfileScope ps(DSLA_KERNEL_CACHE, stream);
    DSLA_LAUNCH(ps, cache_fork_kernel, dim3(c.n_seqs), dim3(64), 0, stream, args_of(c), parent);
    return hipGetLastError();
}

hipError_t launch_cache_truncate(const dsla_cache &c, const int32_t *new_lens, hipStream_t stream)
{
    ProfileScope ps(DSLA_KERNEL_CACHE, stream);
    DSLA_LAUNCH(ps, cache_truncate_kernel, dim3(c.n_seqs), dim3(64), 0, stream, args_of(c), new_lens);
    return hipGetLastError();
}

hipError_t launch_cache_accept(const dsla_cache &c, const dsla_batch &x, const int32_t *path, const int32_t *n_accepted, int n_pools,
                               void *const *pools, void *workspace, hipStream_t stream)
{
    int32_t *verdict = scratch_of(c, x.B, workspace).before;
    const size_t items = static_cast<size_t>(x.B) * (n_pools > 0 ? n_pools * c.H_kv : 1);
    {
        ProfileScope ps(DSLA_KERNEL_CACHE, stream);
        DSLA_LAUNCH(ps, cache_accept_rows_kernel, dim3(static_cast<unsigned>((items + 3) / 4)), dim3(256), 0, stream, args_of(c), args_of(x), path, n_accepted,
                    verdict, n_pools, row_bytes(c), pools_of(n_pools, pools));
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    ProfileScope ps(DSLA_KERNEL_CACHE, stream);
    DSLA_LAUNCH(ps, cache_accept_cut_kernel, dim3(x.B), dim3(64), 0, stream, args_of(c), args_of(x), static_cast<const int32_t *>(verdict));
    return hipGetLastError();
}

hipError_t launch_cache_compact(const dsla_cache &c, int32_t *n_live, int n_pools, void *const *pools, void *workspace, hipStream_t stream)
{
    const Scratch s = scratch_of(c, 1, workspace);
    {
        ProfileScope ps(DSLA_KERNEL_CACHE, stream);
        DSLA_LAUNCH(ps, cache_compact_kernel, dim3(1), dim3(kPlanThreads), 0, stream, args_of(c), s.fresh, s.moves, s.n_moves, n_live);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    e = launch_moves(c, s, n_pools, pools, stream);
    if (e != hipSuccess) return e;
    ProfileScope ps(DSLA_KERNEL_CACHE, stream);
    DSLA_LAUNCH(ps, cache_rename_kernel, dim3(c.n_seqs), dim3(256), 0, stream, args_of(c), static_cast<const int32_t *>(s.fresh), static_cast<const int32_t *>(n_live));
    return hipGetLastError();
}

}  // namespace dsla
