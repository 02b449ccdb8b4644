// What the kernels of attention over a paged cache share: their arguments, and how the work of a call is laid out.
//
// The query heads of a key/value head and the entry's tokens are the rows of one matrix of queries (row = token * G + head of
// the group), cut into tiles.  A tile against all keys of its sequence is a unit of work; units lie one after another on a line of
// granules of kGranule keys, and every workgroup takes an equal stretch of that line, whatever the lengths are (the host does not
// know them).  The one or two units that a stretch only has a part of leave a record there; the workgroup that begins such a unit
// also leaves word of it, and a last kernel merges the records of each.
#pragma once
#include <cfloat>

#include "attention_tiles.h"
#include "paged_common.h"

namespace dsla {

// A unit that goes on behind the stretch it begins in: `rows` rows from row `row` of the queries of entry and head (its first token's
// number in the packed tensors: cu), in the records of `parts` workgroups.  parts = 0: none.
struct OpenUnit {
    int32_t parts, cu, kv, row, rows, pad[3];
};

struct PagedArgs {
    CacheArgs c;
    BatchArgs x;
    const void *q, *k, *v;
    const uint64_t *tree;
    void *o;
    float *sums;           // [2 groups][tile_rows][D]: sums of the parts that the workgroups leave
    float2 *stats;         // [2 groups][tile_rows]: their reference and the sum of their weights
    OpenUnit *open;        // [groups]
    int H, G, max_n, tile_rows, log2_tile, groups;
    uint32_t G_inverse;    // 2^32 / G, rounded up
    float scale_log2e;
    __device__ __forceinline__ int token(int row) const { return G == 1 ? row : static_cast<int>(__umulhi(row, G_inverse)); }   // row / G (G <= 4096, row < 64 G)
};

// Tiles of kRowsTile rows (attention_paged_rows.hip), 16 bits.
constexpr int kRowsTile = 128;
hipError_t launch_attention_paged_rows(const PagedArgs &a, ProfileScope &ps, hipStream_t stream);

namespace {

constexpr int kWaves = 4;       // of a workgroup

// The stretch of a workgroup, one of `count` (of one that merges: whose open unit is its): those of one XCD (workgroups go round the 8 of them) lie
// next to each other, so that the tiles of one head's rows find each other's keys in its L2, and the merge the records.  8 requests of 8192
// tokens, 64 drafted, 32 heads on 8 of 128: 115 -> 106 us; with one token each neither gains nor loses.
__device__ __forceinline__ int stretch_of(int count)
{
    const int xcd = blockIdx.x % 8, more = count % 8;
    return xcd * (count / 8) + (xcd < more ? xcd : more) + blockIdx.x / 8;
}
// The reference of a query's exponentials is raised only when a score exceeds it by more than this (log2): weights stay below 2^8.
constexpr float kSlack = 8.f;

constexpr int kGranule = 128;   // keys
// What beginning and ending a unit costs, in granules.  0 / 1 / 2 / 3 (us, 16 bits, one token each, 32 heads on 8 of 128): 64 requests of 100 to
// 8192 tokens 156 / 91 / 85 / 88, 8 of 500 to 2000 18.0 / 16.8 / 15.2 / 15.6, 16 of 8192 84 / 86 / 85 / 87.
constexpr int kAhead = 2;

__device__ __forceinline__ bool not_finite(float f) { return (__float_as_uint(f) & 0x7f800000u) == 0x7f800000u; }

// What is needed of an entry; units = 0: it takes no part.  On the line a granule has 1 << log2_weight places and lies at the first of them; a unit is
// its granules and kAhead granules' places ahead of them, about what it costs to begin and to end one.  In the kernel for many rows a granule
// has two, so that stretches differ by no more than a block of keys; tiles with few rows have no fewer, since what a block of keys costs hardly
// depends on them: 32 requests of 500 to 4000 tokens, 1 to 64 drafted, 98 us with half for tiles of up to 64 rows, 82 so.
struct Work {
    int cu, n, row, start, L, tiles, granules, units, log2_weight;
    __device__ __forceinline__ int unit() const { return (granules + kAhead) << log2_weight; }
    __device__ __forceinline__ int size() const { return units * unit(); }   // (fits: the host refuses what could not)
    // Of the places at .. at + len - 1 of a unit: its first granule there (or the first one behind), and how many.
    __device__ __forceinline__ int granule(int at) const
    {
        const int place = at - (kAhead << log2_weight);
        return place <= 0 ? 0 : (place + (1 << log2_weight) - 1) >> log2_weight;
    }
    __device__ __forceinline__ int first() const { return kAhead << log2_weight; }   // the first granule's place in a unit
};
__device__ __forceinline__ Work work_of(const PagedArgs &a, int cu, int n, int row, int start)
{
    Work w{cu, n, row, start, start + n, (n * a.G + a.tile_rows - 1) >> a.log2_tile, 0, 0, a.tile_rows == kRowsTile};
    w.granules = (w.L + kGranule - 1) / kGranule;
    w.units = w.tiles * a.c.H_kv;
    return w;
}
__device__ __forceinline__ Work read_work(const PagedArgs &a, int b, bool tell)
{
    const Entry e = read_entry(a.x, a.c, b);
    const int start = a.x.start[b];
    const bool fits = e.ok & (e.n <= a.max_n) & (static_cast<long long>(start) + e.n <= row_room(a.c)), live = fits & (start >= 0);
    if (tell && !fits && (!e.ok || start >= 0)) report(a.c.status, DSLA_STATUS_CACHE_ENTRY);
    return work_of(a, e.cu, live ? e.n : 0, e.row, live ? start : 0);
}

// The same of an entry that is the whole wavefront's, in scalar registers.
__device__ __forceinline__ Work read_work_scalar(const PagedArgs &a, int b)
{
    const Work w = read_work(a, b, false);
    return work_of(a, __builtin_amdgcn_readfirstlane(w.cu), __builtin_amdgcn_readfirstlane(w.n), __builtin_amdgcn_readfirstlane(w.row), __builtin_amdgcn_readfirstlane(w.start));
}

// Inclusive sum over the wavefront: within rows of 16 lanes, then the rows' last lanes handed on.  (Through LDS instead, like the divisions that
// are multiplications here, it is part of about 1 us in front of the first keys, most of a short call being what happens once.)
__device__ __forceinline__ int wave_prefix(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // from 1, 2, 4, 8 lanes below
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // lane 15 of a row to the next one
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // lane 31 to the upper half
    return x;
}

// The line as every wavefront finds it for itself: how much there is of it and a workgroup takes, and the entry that a stretch begins in, with what
// lies ahead of it.
struct Line {
    int total, per, b, before;
    Work w;
};
__device__ __forceinline__ Line read_line(const PagedArgs &a, int stretch, bool tell)
{
    const int lane = threadIdx.x & 63;
    Line l;
    Work w = read_work(a, lane < a.x.B ? lane : 0, tell && lane < a.x.B);
    int n = lane < a.x.B ? w.size() : 0, sum = wave_prefix(n);
    l.total = __builtin_amdgcn_readlane(sum, 63);
    for (int b0 = 64; b0 < a.x.B; b0 += 64) {
        const Work v = read_work(a, b0 + lane < a.x.B ? b0 + lane : 0, tell && b0 + lane < a.x.B);
        l.total += __builtin_amdgcn_readlane(wave_prefix(b0 + lane < a.x.B ? v.size() : 0), 63);
    }
    l.per = (l.total + a.groups - 1) / a.groups;
    if (l.per < (a.tile_rows == kRowsTile ? 2 : 1)) l.per = a.tile_rows == kRowsTile ? 2 : 1;   // (a granule's places: no stretch inside a unit without one)
    const long long x = static_cast<long long>(l.per) * stretch;
    int ahead = 0;
    l.b = l.before = 0;
    for (int b0 = 0;;) {
        const unsigned long long hit = __ballot((x >= ahead + sum - n) & (x < ahead + sum));
        if (hit) {
            const int at = __builtin_ctzll(hit);
            l.b = b0 + at;
            l.before = ahead + __builtin_amdgcn_readlane(sum - n, at);
            l.w = work_of(a, __builtin_amdgcn_readlane(w.cu, at), __builtin_amdgcn_readlane(w.n, at), __builtin_amdgcn_readlane(w.row, at),
                          __builtin_amdgcn_readlane(w.start, at));
            return l;
        }
        ahead += __builtin_amdgcn_readlane(sum, 63);
        b0 += 64;
        if (b0 >= a.x.B) break;
        w = read_work(a, b0 + lane < a.x.B ? b0 + lane : 0, false);
        n = b0 + lane < a.x.B ? w.size() : 0;
        sum = wave_prefix(n);
    }
    l.total = 0;   // a stretch past the end
    l.w = work_of(a, 0, 0, 0, 0);
    return l;
}

}  // namespace
}  // namespace dsla
