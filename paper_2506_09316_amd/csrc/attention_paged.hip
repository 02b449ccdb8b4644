// Softmax attention of the last tokens of every sequence over a paged cache (include/dsla.h: dsla_attention_paged).
//
// A workgroup takes tiles of 16 NT rows; its four wavefronts take blocks of keys in turn, each with a running maximum m, sum z and
// output tiles of its own, and merge at the end of a unit (attention_paged.h: how the work is laid out).
//
// Keys and values go from memory to the matrix instructions' operands without passing through LDS.  Transposed score tiles
// S^T[key][query] = K Q^T take rows of K as they lie; a result tile has the query in the lane's column and four keys in its
// registers, and the second product O^T[feature][query] = V^T P^T may take the keys of its contraction in any order, so the
// exponentials are its right operand as they are.  The left one, V^T, has a feature per row: a lane loads D/16 adjacent features of
// the keys whose weights it holds (whole rows of V, 16 lanes to a row), and row i of tile t is feature i * D/16 + t, so that a lane's own
// loads hold all that it needs: in 32 bits as they are, in 16 bits after exchanging halves between the registers of two keys.
//
// Bound by reading: 64 requests of 100 to 8192 tokens, one token each, 32 heads on 8 of 128 in 16 bits, 492 MB in 84 us (5.9 TB/s), one of
// 131072 tokens 537 MB in 89 us (6.0 TB/s; non-temporal loads made 93 of 120).  A short call is bound by what happens once, one wait after
// another (entries, queries, numbers of pages, keys) and code that is fetched: one request of 1000 tokens, 32 heads of 128, 11.5 us, the
// first kernel 9.8 in a profile.
#include "attention_paged.h"

namespace dsla {
namespace {

// A block of keys and values as a wavefront holds it.  Lane = 16 g + i.  KEYS keys in NS tiles of 16; slot j of a lane in the second
// product is key 16 (j / 4) + 4 g + j % 4, whose weight the score tiles leave in that lane.
template <class T, int D>
struct Block;

template <int D>
struct Block<bf16_t, D> {
    static constexpr int NS = 2, KEYS = 32, SLOTS = 8, NK = D / 32, TF = D / 16;
    u32x4 k[NS][NK];
    uint32_t v[SLOTS][TF / 2];
    struct Query {
        bf16x8 q[NK];
        __device__ __forceinline__ void load(const bf16_t *p, int lane)
        {
#pragma unroll
            for (int c = 0; c < NK; ++c) q[c] = *reinterpret_cast<const bf16x8 *>(p + 32 * c + 8 * (lane >> 4));
        }
        __device__ __forceinline__ void zero()
        {
#pragma unroll
            for (int c = 0; c < NK; ++c) q[c] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
        }
    };
    __device__ __forceinline__ void load_k(int s, const bf16_t *rows, int lane)
    {
#pragma unroll
        for (int c = 0; c < NK; ++c) k[s][c] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(rows + (lane & 15) * D + 8 * (lane >> 4) + 32 * c));
    }
    __device__ __forceinline__ void load_v(int s, const bf16_t *rows, int lane)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bf16_t *p = rows + (4 * (lane >> 4) + j) * D + (lane & 15) * TF;
            if constexpr (TF == 8) {
                const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
#pragma unroll
                for (int w = 0; w < 4; ++w) v[4 * s + j][w] = x[w];
            } else {
                const u32x2 x = *reinterpret_cast<const u32x2 *>(p);
                v[4 * s + j][0] = x[0];
                v[4 * s + j][1] = x[1];
            }
        }
    }
    __device__ __forceinline__ f32x4 scores(int s, const Query &q) const
    {
        f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NK; ++c) a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[s][c]), q.q[c], a, 0, 0, 0);
        return a;
    }
    __device__ __forceinline__ void clear_v(int j)
    {
#pragma unroll
        for (int w = 0; w < TF / 2; ++w) v[j][w] = 0;
    }
    // infinities and NaN to zero; whether there were any
    __device__ __forceinline__ bool tame_v(int j)
    {
        uint32_t any = 0;
#pragma unroll
        for (int w = 0; w < TF / 2; ++w) {
            const uint32_t lo = (v[j][w] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, hi = (v[j][w] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
            v[j][w] &= ~(lo | hi);
            any |= lo | hi;
        }
        return any != 0;
    }
    // exchanges halves so that vt(t) is the operand of feature tile t
    struct Operand {
        bf16x8 a[TF];
    };
    __device__ __forceinline__ Operand operand() const
    {
        Operand r;
#pragma unroll
        for (int t = 0; t < TF; ++t) {
            u32x4 x;
#pragma unroll
            for (int w = 0; w < 4; ++w) x[w] = __builtin_amdgcn_perm(v[2 * w + 1][t / 2], v[2 * w][t / 2], t % 2 ? 0x07060302u : 0x05040100u);
            r.a[t] = __builtin_bit_cast(bf16x8, x);
        }
        return r;
    }
    // With SPLIT the second product takes a weight in two parts of 16 bits, its upper bits and the rest of p (1 + 2^-20), which keeps it to 2^-15; without,
    // it is rounded, by at most 2^-8.  The sum is that of the parts as they are, so that what the roundings have in common (weights that are
    // nearly alike) cancels; neither part of a weight is zero or negative, so an infinite value reaches its sum as what it is.  A tile of 16 rows
    // is bound by reading and splits, rounded / split (us, 32 heads on 8 of 128): 64 requests of 100 to 8192 tokens 83.7 / 83.9, one of
    // 131072 88.6 / 89.0, one of 1000, 32 heads, 11.3 / 11.5 (11.6 with the rest on the chain of z).  Two tiles do not: 32 requests of 2000,
    // 8 tokens each, 46.3 / 47.6, in heads of 64 27.9 / 29.9.
    template <bool SPLIT>
    static __device__ __forceinline__ void accumulate(const Operand &v, const float (&p)[SLOTS], float &z, f32x4 (&acc)[TF])
    {
        const bf16x2 one = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
        u32x4 upper, rest;
        float zr = 0.f;
#pragma unroll
        for (int j = 0; j < SLOTS; j += 2) {
            const uint32_t a = __float_as_uint(p[j]), b = __float_as_uint(p[j + 1]), u = SPLIT ? __builtin_amdgcn_perm(b, a, 0x07060302u) : pack2(p[j], p[j + 1]);
            z = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, u), one, z, false);
            upper[j / 2] = u;
            if (SPLIT) {
                const uint32_t r = pack2(fmaf(p[j], 1.f + 0x1p-20f, -__uint_as_float(a & 0xffff0000u)), fmaf(p[j + 1], 1.f + 0x1p-20f, -__uint_as_float(b & 0xffff0000u)));
                zr = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, r), one, zr, false);
                rest[j / 2] = r;
            }
        }
#pragma unroll
        for (int t = 0; t < TF; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.a[t], __builtin_bit_cast(bf16x8, upper), acc[t], 0, 0, 0);
        if (SPLIT) {
            z += zr;
#pragma unroll
            for (int t = 0; t < TF; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.a[t], __builtin_bit_cast(bf16x8, rest), acc[t], 0, 0, 0);
        }
    }
};

template <int D>
struct Block<float, D> {
    static constexpr int NS = 1, KEYS = 16, SLOTS = 4, NK = D / 16, TF = D / 16;
    f32x4 k[NS][NK];
    float v[SLOTS][TF];
    struct Query {
        f32x4 q[NK];
        __device__ __forceinline__ void load(const float *p, int lane)
        {
#pragma unroll
            for (int c = 0; c < NK; ++c) q[c] = *reinterpret_cast<const f32x4 *>(p + 16 * c + 4 * (lane >> 4));
        }
        __device__ __forceinline__ void zero()
        {
#pragma unroll
            for (int c = 0; c < NK; ++c) q[c] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    __device__ __forceinline__ void load_k(int s, const float *rows, int lane)
    {
#pragma unroll
        for (int c = 0; c < NK; ++c) k[s][c] = *reinterpret_cast<const f32x4 *>(rows + (lane & 15) * D + 4 * (lane >> 4) + 16 * c);
    }
    __device__ __forceinline__ void load_v(int, const float *rows, int lane)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int w = 0; w < TF; w += 4) {
                const f32x4 x = *reinterpret_cast<const f32x4 *>(rows + (4 * (lane >> 4) + j) * D + (lane & 15) * TF + w);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[j][w + e] = x[e];
            }
    }
    __device__ __forceinline__ f32x4 scores(int s, const Query &q) const
    {
        f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NK; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) a = __builtin_amdgcn_mfma_f32_16x16x4f32(k[s][c][e], q.q[c][e], a, 0, 0, 0);
        return a;
    }
    __device__ __forceinline__ void clear_v(int j)
    {
#pragma unroll
        for (int t = 0; t < TF; ++t) v[j][t] = 0.f;
    }
    __device__ __forceinline__ bool tame_v(int j)
    {
        bool any = false;
#pragma unroll
        for (int t = 0; t < TF; ++t) {
            const bool bad = not_finite(v[j][t]);
            any |= bad;
            v[j][t] = bad ? 0.f : v[j][t];
        }
        return any;
    }
    typedef Block<float, D> Operand;
    __device__ __forceinline__ const Operand &operand() const { return *this; }
    template <bool>
    static __device__ __forceinline__ void accumulate(const Operand &b, const float (&p)[SLOTS], float &z, f32x4 (&acc)[TF])
    {
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) z += p[j];
#pragma unroll
        for (int j = 0; j < SLOTS; ++j)
#pragma unroll
            for (int t = 0; t < TF; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(b.v[j][t], p[j], acc[t], 0, 0, 0);
    }
};

template <class T, int D, int NT>
__global__ __launch_bounds__(64 * kWaves, NT == 4 ? 1 : 2) void attention_paged_kernel(PagedArgs a)
{
    using B = Block<T, D>;
    constexpr int TF = B::TF, SLOTS = B::SLOTS, KEYS = B::KEYS, NS = B::NS;
    __shared__ f32x4 s_acc[kWaves / 2][NT * TF][64];
    __shared__ float s_m[kWaves / 2][NT][64], s_z[kWaves / 2][NT][64];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
    const int plog = a.c.page_log2, page = 1 << plog;
    const int stretch = stretch_of(a.groups);
    const Line line = read_line(a, stretch, blockIdx.x == 0 && wave == 0);
    if (threadIdx.x == 0) a.open[stretch].parts = 0;
    if (line.total == 0) return;
    int x0 = line.per * stretch, before = line.before, b = line.b;   // (no more than the total)
    const int x1 = line.total - x0 < line.per ? line.total : x0 + line.per;
    Work w = line.w;

    while (x0 < x1) {
        while (x0 - before >= w.size()) {   // (also over entries that take no part)
            before += w.size();
            w = read_work_scalar(a, ++b);
        }
        // the unit at x0, and the granules of it that are the workgroup's
        const int unit = (x0 - before) / w.unit(), at = x0 - before - unit * w.unit();
        const int len = w.unit() - at < x1 - x0 ? w.unit() - at : x1 - x0;
        const int g0 = w.granule(at), take = w.granule(at + len) - g0;
        const int kv = w.tiles == 1 ? unit : unit / w.tiles, tile = unit - kv * w.tiles;
        if (threadIdx.x == 0 && g0 == 0 && take < w.granules) {
            const int first = x0 - at + w.first();   // the place of the unit's first granule (the workgroup's)
            const int rows = w.n * a.G - tile * a.tile_rows;
            a.open[stretch] = OpenUnit{take > 0 ? (first + ((w.granules - 1) << w.log2_weight)) / line.per - stretch + 1 : 0, w.cu, kv, tile * a.tile_rows, rows < a.tile_rows ? rows : a.tile_rows, {}};
        }
        x0 += len;
        if (take <= 0) continue;
        __syncthreads();   // (the last unit's merge)

        typename B::Query q[NT];
        uint64_t mask[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r = (tile * NT + n) * 16 + i, j = a.token(r);
            const bool is = j < w.n;
            mask[n] = a.tree ? a.tree[w.cu + (is ? j : 0)] : ~0ull >> (63 - (is ? j : 0));
            q[n].load(static_cast<const T *>(a.q) + (static_cast<size_t>(w.cu + (is ? j : 0)) * a.H + kv * a.G + r - j * a.G) * D, lane);
            if (!is) q[n].zero();
        }

        f32x4 acc[NT][TF];
        float m[NT], z[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n] = -FLT_MAX;
            z[n] = 0.f;
#pragma unroll
            for (int t = 0; t < TF; ++t) acc[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        const int from = g0 * kGranule, to = w.granules - g0 == take ? w.L : from + take * kGranule;
        const T *kp = static_cast<const T *>(a.k) + ((static_cast<size_t>(kv) << plog) * D);
        const T *vp = static_cast<const T *>(a.v) + ((static_cast<size_t>(kv) << plog) * D);
        const size_t pitch = (static_cast<size_t>(a.c.H_kv) << plog) * D;
        const int32_t *table = a.c.table + static_cast<size_t>(w.row) * a.c.max_pages;
        const int pages = pages_of(w.L, plog);
        int window = -64, ids = 0;
        unsigned long long none = 0;   // pages of the window that the table gives no number for

        for (int t0 = from + wave * KEYS; t0 < to; t0 += kWaves * KEYS) {
            if (((t0 >> plog) & ~63) != window) {   // the numbers of 64 pages, one in a lane
                window = (t0 >> plog) & ~63;
                ids = window + lane < pages ? table[window + lane] : 0;
                none = __ballot((ids < 0) | (ids >= a.c.n_pages));
                if (none) {
                    if (lane == 0) report(a.c.status, DSLA_STATUS_CACHE_ENTRY);
                    ids = none >> lane & 1 ? 0 : ids;
                }
            }
            B x;
            int gap = 0;   // bit s: tile s has no page
            const T *rows[NS];
#pragma unroll
            for (int s = 0; s < NS; ++s) {   // (a tile of 16 keys lies in one page; past the end page 0 of the pool is read and nothing is made of it)
                const int t = t0 + 16 * s, p = (t >> plog) - window;
                gap |= static_cast<int>(none >> p & 1) << s;
                const size_t off = static_cast<size_t>(__builtin_amdgcn_readlane(ids, p)) * pitch + static_cast<size_t>(t & (page - 1)) * D;
                x.load_k(s, kp + off, lane);
                rows[s] = vp + off;
            }
#pragma unroll
            for (int s = 0; s < NS; ++s) x.load_v(s, rows[s], lane);

            // Past start, and where pages are missing: which keys exist and which a query sees, as bits counted from key t0 + 4 g (a lane's
            // keys are 0 .. 3 and 16 .. 19 from there).
            const bool edge = (t0 + KEYS > w.start) | (gap != 0);   // (uniform)
            const int left = to - t0 - 4 * g, past = w.start - t0 - 4 * g;
            uint32_t there = ~0u;
            if (edge) {
                there = left >= 32 ? ~0u : left > 0 ? (1u << left) - 1 : 0u;
                if (gap & 1) there &= 0xffff0000u;
                if (gap & 2) there &= 0x0000ffffu;
            }
            float p[NT][SLOTS];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    const f32x4 sc = x.scores(s, q[n]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) p[n][4 * s + r] = sc[r] * a.scale_log2e;
                }
                if (edge) {
                    const uint32_t drafted = past >= 32 ? ~0u : past > 0 ? static_cast<uint32_t>(mask[n]) << past | ((1u << past) - 1) : static_cast<uint32_t>(mask[n] >> (-past & 63));
                    const uint32_t seen = drafted & there;
#pragma unroll
                    for (int j = 0; j < SLOTS; ++j) p[n][j] = seen & 1u << (16 * (j / 4) + j % 4) ? p[n][j] : -INFINITY;
                }
                float top = -FLT_MAX;
#pragma unroll
                for (int j = 0; j < SLOTS; ++j) top = fmaxf(top, p[n][j]);
                if (__ballot(top > m[n] + kSlack)) {   // the reference of some query is raised: for all of the tile, and the four lanes of each alike
                    top = fmaxf(top, __shfl_xor(top, 16));
                    top = fmaxf(fmaxf(top, __shfl_xor(top, 32)), m[n]);
                    const float c0 = __builtin_amdgcn_exp2f(m[n] - top);
                    m[n] = top;
                    z[n] *= c0;
#pragma unroll
                    for (int t = 0; t < TF; ++t) acc[n][t] *= c0;
                }
#pragma unroll
                for (int j = 0; j < SLOTS; ++j) p[n][j] = __builtin_amdgcn_exp2f(p[n][j] - m[n]);
            }
            if (edge) {
                // What does not exist is zero, and where queries see different tokens an infinity or NaN among them too: zero times it would reach
                // the queries that do not see it.  Those that do get their products one by one.
#pragma unroll
                for (int j = 0; j < SLOTS; ++j)
                    if (!(there & 1u << (16 * (j / 4) + j % 4))) x.clear_v(j);
                if ((w.n > 1) | (a.tree != nullptr)) {
                    bool wild = false;
#pragma unroll
                    for (int j = 0; j < SLOTS; ++j)
                        if (16 * (j / 4) + j % 4 >= past) wild |= x.tame_v(j);
                    if (__builtin_expect(__ballot(wild) != 0, 0)) {
                        float *s_p = reinterpret_cast<float *>(&s_acc[0][0][0]) + wave * (NT * SLOTS * 64);   // (no more than the merge uses)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int j = 0; j < SLOTS; ++j) s_p[(n * SLOTS + j) * 64 + lane] = p[n][j];
                        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
                        for (int c = 0; c < KEYS; ++c) {
                            const int t = t0 + c;
                            if (t < w.start || t >= to || (gap >> (c >> 4) & 1)) continue;
                            const T *row = (NS > 1 && c >= 16 ? rows[NS - 1] : rows[0]) + (c & 15) * D;
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                const float weight = s_p[(n * SLOTS + (c >> 4) * 4 + (c & 3)) * 64 + ((c & 15) >> 2) * 16 + i];
                                const bool seen = mask[n] >> (t - w.start) & 1;
#pragma unroll
                                for (int e = 0; e < 4 * TF; ++e) {
                                    const float f = to_f32(row[4 * g * TF + e]);
                                    acc[n][e % TF][e / TF] += seen && not_finite(f) ? f * weight : 0.f;
                                }
                            }
                        }
                    }
                }
            }
            const auto &v = x.operand();
#pragma unroll
            for (int n = 0; n < NT; ++n) B::template accumulate<NT == 1>(v, p[n], z[n], acc[n]);
        }

        // the sums of a query's four lanes; then wavefronts 2 and 3 into 0 and 1, and 1 into 0
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            z[n] += __shfl_xor(z[n], 16);
            z[n] += __shfl_xor(z[n], 32);
        }
#pragma unroll 1
        for (int half = kWaves / 2; half > 0; half >>= 1) {
            __syncthreads();
            if (wave >= half && wave < 2 * half) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    s_m[wave - half][n][lane] = m[n];
                    s_z[wave - half][n][lane] = z[n];
#pragma unroll
                    for (int t = 0; t < TF; ++t) s_acc[wave - half][n * TF + t][lane] = acc[n][t];
                }
            }
            __syncthreads();
            if (wave < half) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float mo = s_m[wave][n][lane], top = fmaxf(m[n], mo), c0 = __builtin_amdgcn_exp2f(m[n] - top), c1 = __builtin_amdgcn_exp2f(mo - top);
                    m[n] = top;
                    z[n] = c0 * z[n] + c1 * s_z[wave][n][lane];
#pragma unroll
                    for (int t = 0; t < TF; ++t) acc[n][t] = c0 * acc[n][t] + c1 * s_acc[wave][n * TF + t][lane];
                }
            }
        }
        if (wave != 0) continue;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r = (tile * NT + n) * 16 + i, j = a.token(r);
            if (j >= w.n) continue;
            if (take == w.granules) {
                T *o = static_cast<T *>(a.o) + (static_cast<size_t>(w.cu + j) * a.H + kv * a.G + r - j * a.G) * D + 4 * g * TF;
                const float inv = z[n] == 0.f ? 0.f : 1.f / z[n];   // (a query that sees nothing: zeros)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int t = 0; t < TF; ++t) o[e * TF + t] = from_f32<T>(acc[n][t][e] * inv);
            } else {
                // a stretch has no more than one unit that began before it (record 0) and one that goes on after it (record 1)
                const size_t rec = (2 * static_cast<size_t>(stretch) + (g0 == 0)) * a.tile_rows + n * 16 + i;
                if (g == 0) a.stats[rec] = make_float2(m[n], z[n]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int t = 0; t < TF; t += 4)
                        *reinterpret_cast<f32x4 *>(a.sums + rec * D + (4 * g + e) * TF + t) = f32x4{acc[n][t][e], acc[n][t + 1][e], acc[n][t + 2][e], acc[n][t + 3][e]};
            }
        }
    }
}

// Merges the records of the units that lie in several stretches: workgroup (x, y) takes rows of the one that stretch x begins and does
// not end.  D / 4 lanes hold a row, kMergeRows rows are a workgroup's; with SPLIT it has one row, whose records its groups of lanes
// share.  Bound by its launch and the records' way through memory: 2 to 5 us with one token each, 9 where the tiles have 128 rows.  (Four or
// eight stretches to a workgroup, so that fewer have nothing to do: the same.)
constexpr int kMergeRows = 8;
template <class T, int D, bool SPLIT>
__global__ __launch_bounds__(256) void attention_paged_merge_kernel(PagedArgs a)
{
    constexpr int LPR = D / 4, GROUPS = 256 / LPR, U = 4, STEP = SPLIT ? GROUPS : 1;
    __shared__ f32x4 s_part[GROUPS][LPR];
    __shared__ float2 s_stat[GROUPS];
    const int stretch = stretch_of(a.groups);
    const OpenUnit open = a.open[stretch];
    const int group = threadIdx.x / LPR, f = threadIdx.x % LPR;
    const int row0 = blockIdx.y * (SPLIT ? 1 : kMergeRows), row1 = row0 + (SPLIT ? 1 : kMergeRows);
    if (open.parts == 0 || row0 >= open.rows) return;
    for (int row = row0 + (SPLIT ? 0 : group); row < (row1 < open.rows ? row1 : open.rows); row += SPLIT ? 1 : GROUPS) {
        const size_t rec = 2 * static_cast<size_t>(stretch) * a.tile_rows + row;   // of part p: record 1 of the first workgroup, record 0 of the others
        float M = -FLT_MAX, Z = 0.f;
        f32x4 A = {0.f, 0.f, 0.f, 0.f};
        for (int p0 = SPLIT ? group : 0; p0 < open.parts; p0 += STEP * U) {   // U records are requested before the first is used
            float2 s[U];
            f32x4 x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int p = p0 + u * STEP < open.parts ? p0 + u * STEP : p0;
                const size_t at = rec + static_cast<size_t>(p == 0 ? 1 : 2 * p) * a.tile_rows;
                s[u] = a.stats[at];
                x[u] = *reinterpret_cast<const f32x4 *>(a.sums + at * D + 4 * f);
            }
            float top = M;
#pragma unroll
            for (int u = 0; u < U; ++u) top = fmaxf(top, s[u].x);
            const float c0 = __builtin_amdgcn_exp2f(M - top);
            Z *= c0;
            A *= c0;
            M = top;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (p0 + u * STEP < open.parts) {
                    const float c = __builtin_amdgcn_exp2f(s[u].x - M);
                    Z = fmaf(c, s[u].y, Z);
                    A += c * x[u];
                }
        }
        if (SPLIT) {
            s_part[group][f] = A;
            if (f == 0) s_stat[group] = make_float2(M, Z);
            __syncthreads();
            if (group != 0) return;
            for (int o = 1; o < GROUPS; ++o) {
                const float top = fmaxf(M, s_stat[o].x), c0 = __builtin_amdgcn_exp2f(M - top), c1 = __builtin_amdgcn_exp2f(s_stat[o].x - top);
                Z = c0 * Z + c1 * s_stat[o].y;
                A = c0 * A + c1 * s_part[o][f];
                M = top;
            }
        }
        const float inv = Z == 0.f ? 0.f : 1.f / Z;
        const int r = open.row + row, j = a.token(r);
        T *o = static_cast<T *>(a.o) + (static_cast<size_t>(open.cu + j) * a.H + open.kv * a.G + r - j * a.G) * D + 4 * f;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = from_f32<T>(A[e] * inv);
    }
}

// Stretches of the line: one workgroup to a compute unit.  256 / 384 / 512 / 768 / 1024 of them (us, with kAhead = 1; 16 bits, one token
// each): 64 requests of 100 to 8192 tokens, 32 heads on 8 of 128, 88 / 101 / 87 / 87 / 93; one of 131072 89 / 107 / 92 / 91 / 97; 16 of 8192
// 86 / 104 / 90 / 89 / 94; 64 of 300 to 700 33 / 35 / 32 / 32 / 36; 8 of 500 to 2000 17.2 / 19.1 / 19.2 / 16.9 / 17.0.
// (The kernel for many rows: two workgroups to a unit.)
constexpr int kStretches = 256, kRowsStretches = 512;

// How the work is cut: tiles of 16 NT rows, and how many workgroups share the line.
struct PagedPlan {
    int NT, tile_rows, groups;   // NT = 0: attention_paged_rows.hip
    bool split_merge;
    size_t records;
};
PagedPlan plan_of(const dsla_cache &c, const dsla_batch &x, int H, int64_t max_len)
{
    PagedPlan p;
    const int G = H / c.H_kv;
    const int64_t rows = static_cast<int64_t>(x.max_n) * G, heads = static_cast<int64_t>(x.B) * c.H_kv;
    // Beyond 32 rows the kernel for many rows, 16 bits; this one with 2 (4) tiles of 16 / that one (us, 32 heads on 8 of 128): 20 to 32 rows of 8
    // requests of 8192 tokens 50 to 54 / 64, 32 of 2000 46 to 49 / 60, 8 of 1000 17 to 19 / 20, 64 of 512 33 to 35 / 31; 36 to 64 rows 62 to 66 /
    // 65 to 70, 52 to 55 / 62 to 65, 24 to 26 / 21 to 24, 45 to 49 / 32 to 34: no side wins there, and that one is built for the rows above anyway.
    p.NT = rows <= 16 ? 1 : rows <= 32 ? 2 : c.dtype == DSLA_BF16 ? 0 : 4;
    p.tile_rows = p.NT ? 16 * p.NT : kRowsTile;
    const int64_t units = heads * ((rows + p.tile_rows - 1) / p.tile_rows);
    const int64_t room = static_cast<int64_t>(c.max_pages) * c.page, longest = max_len < 1 ? 1 : max_len < room ? max_len : room;
    const int64_t granules = units * ((longest + kGranule - 1) / kGranule);
    const int stretches = p.NT ? kStretches : kRowsStretches;
    p.groups = static_cast<int>(granules < stretches ? granules : stretches);
    // A workgroup to a row where units have many records / eight rows to one (us, 32 heads on 8 of 128): one request of 131072 tokens 86 / 89, of
    // 20000 20 / 24, two 32 / 33, four of 8000 the same; tiles of 128 rows, two of 20000 tokens 85 / 76, four of 8000 76 / 65.
    p.split_merge = p.NT && p.groups > 8 * units;
    p.records = 2 * static_cast<size_t>(p.groups) * p.tile_rows;
    return p;
}

template <class T, int D>
hipError_t launch_t(const PagedPlan &p, const PagedArgs &a, hipStream_t stream)
{
    ProfileScope ps(DSLA_KERNEL_ATTENTION_PAGED, stream);
    hipError_t err = hipSuccess;
    if constexpr (sizeof(T) == 2)
        if (p.NT == 0) err = launch_attention_paged_rows(a, ps, stream);
    if (p.NT) {
        auto kernel = p.NT == 1 ? attention_paged_kernel<T, D, 1> : attention_paged_kernel<T, D, 2>;
        if constexpr (sizeof(T) == 4)
            if (p.NT == 4) kernel = attention_paged_kernel<T, D, 4>;
        DSLA_LAUNCH_FIRST(ps, kernel, dim3(static_cast<unsigned>(p.groups)), dim3(64 * kWaves), 0, stream, a);
        err = hipGetLastError();
    }
    if (err != hipSuccess) return err;
    const unsigned rows = a.max_n * a.G < a.tile_rows ? a.max_n * a.G : a.tile_rows;
    if (p.split_merge) DSLA_LAUNCH_LAST(ps, (attention_paged_merge_kernel<T, D, true>), dim3(p.groups, rows), dim3(256), 0, stream, a);
    else DSLA_LAUNCH_LAST(ps, (attention_paged_merge_kernel<T, D, false>), dim3(p.groups, (rows + kMergeRows - 1) / kMergeRows), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

// The line's places, two to a granule in the kernel for many rows, are 32-bit numbers.
bool attention_paged_fits(const dsla_cache &c, const dsla_batch &x, int H)
{
    const int64_t rows = static_cast<int64_t>(x.max_n) * (H / c.H_kv), room = static_cast<int64_t>(c.max_pages) * c.page;
    const int tile_rows = plan_of(c, x, H, 1).tile_rows;
    return static_cast<double>(x.B) * c.H_kv * ((rows + tile_rows - 1) / tile_rows) * static_cast<double>(room / kGranule + 1 + kAhead) < 1.0e9;
}

size_t attention_paged_workspace_bytes(const dsla_cache &c, const dsla_batch &x, int H, int64_t max_len)
{
    const PagedPlan p = plan_of(c, x, H, max_len);
    return p.records * (2 + c.d) * sizeof(float) + p.groups * sizeof(OpenUnit);
}

hipError_t launch_attention_paged(const dsla_cache &c, const dsla_batch &x, int H, int64_t max_len, float scale, const void *q, const void *k_pages,
                                  const void *v_pages, const uint64_t *tree, void *o, void *workspace, hipStream_t stream)
{
    const PagedPlan p = plan_of(c, x, H, max_len);
    PagedArgs a;
    a.c = args_of(c);
    a.x = args_of(x);
    a.q = q;
    a.k = k_pages;
    a.v = v_pages;
    a.tree = tree;
    a.o = o;
    a.sums = static_cast<float *>(workspace);
    a.stats = reinterpret_cast<float2 *>(a.sums + p.records * c.d);
    a.open = reinterpret_cast<OpenUnit *>(a.stats + p.records);
    a.H = H;
    a.G = H / c.H_kv;
    a.max_n = x.max_n;
    a.tile_rows = p.tile_rows;
    a.log2_tile = __builtin_ctz(p.tile_rows);
    a.G_inverse = static_cast<uint32_t>(((1ull << 32) + a.G - 1) / a.G);
    a.groups = p.groups;
    a.scale_log2e = scale * 1.44269504088896341f;
    if (c.dtype == DSLA_BF16) return c.d == 128 ? launch_t<bf16_t, 128>(p, a, stream) : launch_t<bf16_t, 64>(p, a, stream);
    return c.d == 128 ? launch_t<float, 128>(p, a, stream) : launch_t<float, 64>(p, a, stream);
}

}  // namespace dsla
