// Softmax attention of the last tokens of every sequence over a paged cache (include/dsla.h: dsla_attention_paged).
//
// The query heads of a key/value head and the entry's tokens are the rows of one matrix of queries (row = token * G + head of
// the group), cut into tiles of 16 NT rows.  A workgroup takes a tile against a part of the sequence's keys; its four wavefronts
// take blocks of keys in turn, each with a running maximum m, sum z and output tiles of its own, and merge at the end; parts leave
// records that a second kernel merges.
//
// Keys and values go from memory to the matrix instructions' operands without passing through LDS.  Transposed score tiles
// S^T[key][query] = K Q^T take rows of K as they lie; a result tile has the query in the lane's column and four keys in its
// registers, and the second product O^T[feature][query] = V^T P^T may take the keys of its contraction in any order, so the
// exponentials are its right operand as they are.  The left one, V^T, has a feature per row: a lane loads D/16 adjacent features of
// the keys whose weights it holds (whole rows of V, 16 lanes to a row), and row i of tile t is feature i * D/16 + t, so that a lane's own
// loads hold all that it needs: in 32 bits as they are, in 16 bits after exchanging halves between the registers of two keys.
#include <cfloat>

#include "paged_common.h"

namespace dsla {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;
// The reference of a query's exponentials is raised only when a score exceeds it by more than this (log2): weights stay below 2^8.
constexpr float kSlack = 8.f;

struct PagedArgs {
    CacheArgs c;
    BatchArgs x;
    const void *q, *k, *v;
    const uint64_t *tree;
    void *o;
    float *parts;          // [B][H_kv][P][max_n G][2 + D]: m, z, sums; where P > 1
    int H, G, max_n, tiles, P, part_keys, units;
    float scale_log2e;
};

__device__ __forceinline__ bool not_finite(float f) { return (__float_as_uint(f) & 0x7f800000u) == 0x7f800000u; }

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
        for (int c = 0; c < NK; ++c) k[s][c] = *reinterpret_cast<const u32x4 *>(rows + (lane & 15) * D + 8 * (lane >> 4) + 32 * c);
    }
    __device__ __forceinline__ void load_v(int s, const bf16_t *rows, int lane)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bf16_t *p = rows + (4 * (lane >> 4) + j) * D + (lane & 15) * TF;
            if constexpr (TF == 8) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(p);
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
    // The weights are rounded to 16 bits for the second product (they are at most 2^8 and positive: 2^-9 of each, of either sign); their sum
    // is taken before.
    static __device__ __forceinline__ void accumulate(const Operand &v, const float (&p)[SLOTS], f32x4 (&acc)[TF])
    {
        bf16x8 b;
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) b[j] = static_cast<__bf16>(p[j]);
#pragma unroll
        for (int t = 0; t < TF; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.a[t], b, acc[t], 0, 0, 0);
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
    static __device__ __forceinline__ void accumulate(const Operand &b, const float (&p)[SLOTS], f32x4 (&acc)[TF])
    {
#pragma unroll
        for (int j = 0; j < SLOTS; ++j)
#pragma unroll
            for (int t = 0; t < TF; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(b.v[j][t], p[j], acc[t], 0, 0, 0);
    }
};

// What the workgroups of an entry need to know about it; live = false: it takes no part.
struct Work {
    Entry e;
    int start, L, parts;
    bool live;
};
__device__ __forceinline__ Work read_work(const PagedArgs &a, int b)
{
    Work w;
    w.e = read_entry(a.x, a.c, b);
    w.start = a.x.start[b];
    const bool fits = w.e.ok && w.e.n <= a.max_n && static_cast<long long>(w.start) + w.e.n <= row_room(a.c);
    w.live = fits && w.start >= 0 && w.e.n > 0;
    w.L = w.live ? w.start + w.e.n : 0;
    const int parts = static_cast<int>((static_cast<long long>(w.L) + a.part_keys - 1) / a.part_keys);
    w.parts = parts < a.P ? parts : a.P;   // (the last part takes what is left, also of a sequence that is longer than was announced)
    if (!fits && (!w.e.ok || w.start >= 0) && threadIdx.x == 0) report(a.c.status, DSLA_STATUS_CACHE_ENTRY);
    return w;
}

template <class T, int D, int NT>
__global__ __launch_bounds__(64 * kWaves, NT == 4 ? 1 : 2) void attention_paged_kernel(PagedArgs a)
{
    using B = Block<T, D>;
    constexpr int TF = B::TF, SLOTS = B::SLOTS, KEYS = B::KEYS;
    __shared__ f32x4 s_acc[kWaves / 2][NT * TF][64];
    __shared__ float s_m[kWaves / 2][NT][64], s_z[kWaves / 2][NT][64];

    // Workgroups go round-robin over the 8 XCDs: the tiles of one part of one sequence's head come 8 apart, so that one L2 serves them
    const int id = blockIdx.x, unit = id / (8 * a.tiles) * 8 + id % 8, tile = id / 8 % a.tiles;
    if (unit >= a.units) return;
    const int part = unit % a.P, kv = unit / a.P % a.c.H_kv, b = unit / a.P / a.c.H_kv;
    const Work w = read_work(a, b);
    if (!w.live || part >= w.parts || tile * 16 * NT >= w.e.n * a.G) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
    const int plog = a.c.page_log2, page = 1 << plog;

    typename B::Query q[NT];
    uint64_t mask[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = (tile * NT + n) * 16 + i, j = r / a.G;
        mask[n] = 0;
        if (j < w.e.n) {
            mask[n] = a.tree ? a.tree[w.e.cu + j] : ~0ull >> (63 - j);
            q[n].load(static_cast<const T *>(a.q) + (static_cast<size_t>(w.e.cu + j) * a.H + kv * a.G + r % a.G) * D, lane);
        } else {
            q[n].zero();
        }
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

    const int from = part * a.part_keys, to = part == a.P - 1 || w.L - from < a.part_keys ? w.L : from + a.part_keys;
    const T *kp = static_cast<const T *>(a.k) + ((static_cast<size_t>(kv) << plog) * D);
    const T *vp = static_cast<const T *>(a.v) + ((static_cast<size_t>(kv) << plog) * D);
    const size_t pitch = (static_cast<size_t>(a.c.H_kv) << plog) * D;
    const int32_t *table = a.c.table + static_cast<size_t>(w.e.row) * a.c.max_pages;
    const int pages = pages_of(w.L, plog);
    int window = -64, ids = 0;
    unsigned long long none = 0;   // pages of the window that the table gives no number for

    for (int t0 = from + wave * KEYS; t0 < to; t0 += kWaves * KEYS) {
        if (((t0 >> plog) & ~63) != window) {   // the numbers of 64 pages, one in a lane
            window = (t0 >> plog) & ~63;
            ids = window + lane < pages ? table[window + lane] : 0;
            none = __ballot(ids < 0 || ids >= a.c.n_pages);
            if (none) {
                if (lane == 0) report(a.c.status, DSLA_STATUS_CACHE_ENTRY);
                if (none >> lane & 1) ids = 0;
            }
        }
        B x;
        bool gap = false;
        const T *rows[B::NS];
#pragma unroll
        for (int s = 0; s < B::NS; ++s) {   // (a tile of 16 keys lies in one page; past the end page 0 of the pool is read and nothing is made of it)
            const int t = t0 + 16 * s, p = (t >> plog) - window;
            gap |= none >> p & 1;
            const int number = __builtin_amdgcn_readlane(ids, p);
            const size_t at = static_cast<size_t>(number) * pitch + static_cast<size_t>(t & (page - 1)) * D;
            x.load_k(s, kp + at, lane);
            rows[s] = vp + at;
        }
#pragma unroll
        for (int s = 0; s < B::NS; ++s) x.load_v(s, rows[s], lane);

        const bool edge = t0 + KEYS > w.start || gap;   // (uniform)
        uint32_t there = ~0u;                           // bit j: the key of slot j exists
        float p[NT][SLOTS];
        if (edge) {
            there = 0;
#pragma unroll
            for (int j = 0; j < SLOTS; ++j) {
                const int t = t0 + 16 * (j / 4) + 4 * g + j % 4;
                if (t < to && !(none >> (((t0 + 16 * (j / 4)) >> plog) - window) & 1)) there |= 1u << j;
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float top = -FLT_MAX;
#pragma unroll
            for (int s = 0; s < B::NS; ++s) {
                const f32x4 sc = x.scores(s, q[n]);
#pragma unroll
                for (int r = 0; r < 4; ++r) p[n][4 * s + r] = sc[r] * a.scale_log2e;
            }
            if (edge) {
#pragma unroll
                for (int j = 0; j < SLOTS; ++j) {
                    const int t = t0 + 16 * (j / 4) + 4 * g + j % 4;
                    const bool seen = (there >> j & 1) && (t < w.start || (mask[n] >> ((t - w.start) & 63) & 1));
                    p[n][j] = seen ? p[n][j] : -INFINITY;
                }
            }
#pragma unroll
            for (int j = 0; j < SLOTS; ++j) top = fmaxf(top, p[n][j]);
            if (__ballot(top > m[n] + kSlack)) {   // the reference of some query is raised: for all of the tile, and the four lanes of each alike
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(fmaxf(top, __shfl_xor(top, 32)), m[n]);
                const float c0 = exp2f(m[n] - top);
                m[n] = top;
                z[n] *= c0;
#pragma unroll
                for (int t = 0; t < TF; ++t) acc[n][t] *= c0;
            }
#pragma unroll
            for (int j = 0; j < SLOTS; ++j) {
                p[n][j] = __builtin_amdgcn_exp2f(p[n][j] - m[n]);
                z[n] += p[n][j];
            }
        }
        if (edge) {
            // What does not exist is zero, and an infinity or NaN among the drafted tokens too: zero times it would reach the queries that do not
            // see it.  Those that do get their products one by one.
            bool wild = false;
#pragma unroll
            for (int j = 0; j < SLOTS; ++j) {
                if (!(there >> j & 1)) x.clear_v(j);
                else if (t0 + 16 * (j / 4) + 4 * g + j % 4 >= w.start) wild |= x.tame_v(j);
            }
            if (__ballot(wild)) {
                float *s_p = reinterpret_cast<float *>(&s_acc[0][0][0]) + wave * (NT * SLOTS * 64);   // (a quarter of what the merge uses, at most)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < SLOTS; ++j) s_p[(n * SLOTS + j) * 64 + lane] = p[n][j];
                __builtin_amdgcn_wave_barrier();
#pragma unroll 1
                for (int c = 0; c < KEYS; ++c) {
                    const int t = t0 + c;
                    if (t < w.start || t >= to || (none >> ((t >> plog) - window) & 1)) continue;
                    const T *row = rows[0] + (c & 15) * D;
                    if constexpr (B::NS > 1) row = c < 16 ? row : rows[1] + (c & 15) * D;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const float weight = s_p[(n * SLOTS + (c >> 4) * 4 + (c & 3)) * 64 + ((c & 15) >> 2) * 16 + i];
                        const bool seen = (mask[n] >> (t - w.start)) & 1;
#pragma unroll
                        for (int e = 0; e < 4 * TF; ++e) {
                            const float f = to_f32(row[4 * g * TF + e]);
                            acc[n][e % TF][e / TF] += seen && not_finite(f) ? f * weight : 0.f;
                        }
                    }
                }
            }
        }
        const auto &v = x.operand();
#pragma unroll
        for (int n = 0; n < NT; ++n) B::accumulate(v, p[n], acc[n]);
    }

    // the sums of a query's four lanes; then wavefronts 2 and 3 into 0 and 1, and 1 into 0
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        z[n] += __shfl_xor(z[n], 16);
        z[n] += __shfl_xor(z[n], 32);
    }
#pragma unroll
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
                const float mo = s_m[wave][n][lane], top = fmaxf(m[n], mo), c0 = exp2f(m[n] - top), c1 = exp2f(mo - top);
                m[n] = top;
                z[n] = c0 * z[n] + c1 * s_z[wave][n][lane];
#pragma unroll
                for (int t = 0; t < TF; ++t) acc[n][t] = c0 * acc[n][t] + c1 * s_acc[wave][n * TF + t][lane];
            }
        }
    }
    if (wave != 0) return;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = (tile * NT + n) * 16 + i, j = r / a.G;
        if (j >= w.e.n) continue;
        if (w.parts == 1) {
            T *o = static_cast<T *>(a.o) + (static_cast<size_t>(w.e.cu + j) * a.H + kv * a.G + r % a.G) * D + 4 * g * TF;
            const float inv = z[n] == 0.f ? 0.f : 1.f / z[n];   // (a query that sees nothing: zeros)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int t = 0; t < TF; ++t) o[e * TF + t] = from_f32<T>(acc[n][t][e] * inv);
        } else {
            float *rec = a.parts + (static_cast<size_t>(unit) * a.max_n * a.G + r) * (2 + D);
            if (g == 0) {
                rec[0] = m[n];
                rec[1] = z[n];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int t = 0; t < TF; ++t) rec[2 + (4 * g + e) * TF + t] = acc[n][t][e];
        }
    }
}

// Merges the records of a row's parts.
template <class T, int D>
__global__ __launch_bounds__(D) void attention_paged_merge_kernel(PagedArgs a)
{
    const int rows = a.max_n * a.G, r = blockIdx.x % rows, kv = blockIdx.x / rows % a.c.H_kv, b = blockIdx.x / rows / a.c.H_kv, f = threadIdx.x;
    const Work w = read_work(a, b);
    const int j = r / a.G;
    if (!w.live || w.parts == 1 || j >= w.e.n) return;
    const float *rec = a.parts + ((static_cast<size_t>(b) * a.c.H_kv + kv) * a.P * rows + r) * (2 + D);
    const size_t pitch = static_cast<size_t>(rows) * (2 + D);
    float M = -FLT_MAX, Z = 0.f, A = 0.f;
    constexpr int U = 8;
    for (int p0 = 0; p0 < w.parts; p0 += U) {   // eight records are requested before the first is used
        float m[U], z[U], s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float *x = rec + (p0 + u < w.parts ? p0 + u : w.parts - 1) * pitch;
            m[u] = x[0];
            z[u] = x[1];
            s[u] = x[2 + f];
        }
        float top = M;
#pragma unroll
        for (int u = 0; u < U; ++u) top = fmaxf(top, m[u]);
        const float c0 = exp2f(M - top);
        Z *= c0;
        A *= c0;
        M = top;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float c = exp2f(m[u] - M);
            Z = p0 + u < w.parts ? fmaf(c, z[u], Z) : Z;
            A = p0 + u < w.parts ? fmaf(c, s[u], A) : A;
        }
    }
    static_cast<T *>(a.o)[(static_cast<size_t>(w.e.cu + j) * a.H + kv * a.G + r % a.G) * D + f] = from_f32<T>(Z == 0.f ? 0.f : A / Z);
}

// How the work is cut: tiles of 16 NT rows, P parts of part_keys keys.
struct PagedPlan {
    int NT, tiles, P, part_keys;
    size_t ws_bytes;
};
PagedPlan plan_of(const dsla_cache &c, const dsla_batch &x, int H, int64_t max_len)
{
    PagedPlan p;
    const int G = H / c.H_kv;
    const int64_t rows = static_cast<int64_t>(x.max_n) * G, heads = static_cast<int64_t>(x.B) * c.H_kv;
    p.NT = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    p.tiles = static_cast<int>((rows + 16 * p.NT - 1) / (16 * p.NT));
    const int64_t room = static_cast<int64_t>(c.max_pages) * c.page, longest = max_len < 1 ? 1 : max_len < room ? max_len : room;
    int64_t P = (1024 + heads * p.tiles - 1) / (heads * p.tiles);
    const int64_t most = (longest + 255) / 256;
    if (P > most) P = most;
    p.part_keys = static_cast<int>(((longest + P - 1) / P + 127) / 128 * 128);
    p.P = static_cast<int>((longest + p.part_keys - 1) / p.part_keys);
    p.ws_bytes = p.P > 1 ? static_cast<size_t>(heads) * p.P * rows * (2 + c.d) * sizeof(float) : 0;
    return p;
}

template <class T, int D>
hipError_t launch_t(const PagedPlan &p, const PagedArgs &a, hipStream_t stream)
{
    ProfileScope ps(DSLA_KERNEL_ATTENTION_PAGED, stream);
    if (p.P == 1) ps.e1_first = ps.e1;   // no merge kernel follows: the first launch closes the record too
    auto kernel = p.NT == 1 ? attention_paged_kernel<T, D, 1> : p.NT == 2 ? attention_paged_kernel<T, D, 2> : attention_paged_kernel<T, D, 4>;
    const int64_t groups = (static_cast<int64_t>(a.units) + 7) / 8 * 8 * p.tiles;
    DSLA_LAUNCH_FIRST(ps, kernel, dim3(static_cast<unsigned>(groups)), dim3(64 * kWaves), 0, stream, a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess || p.P == 1) return err;
    DSLA_LAUNCH_LAST(ps, (attention_paged_merge_kernel<T, D>), dim3(static_cast<unsigned>(a.x.B) * a.c.H_kv * a.max_n * a.G), dim3(D), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

size_t attention_paged_workspace_bytes(const dsla_cache &c, const dsla_batch &x, int H, int64_t max_len) { return plan_of(c, x, H, max_len).ws_bytes; }

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
    a.parts = static_cast<float *>(workspace);
    a.H = H;
    a.G = H / c.H_kv;
    a.max_n = x.max_n;
    a.tiles = p.tiles;
    a.P = p.P;
    a.part_keys = p.part_keys;
    a.units = x.B * c.H_kv * p.P;
    a.scale_log2e = scale * 1.44269504088896341f;
    if (c.dtype == DSLA_BF16) return c.d == 128 ? launch_t<bf16_t, 128>(p, a, stream) : launch_t<bf16_t, 64>(p, a, stream);
    return c.d == 128 ? launch_t<float, 128>(p, a, stream) : launch_t<float, 64>(p, a, stream);
}

}  // namespace dsla
