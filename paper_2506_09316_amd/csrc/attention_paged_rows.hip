// Attention over a paged cache with many queries to a key/value head: trees and chains of drafted tokens, 16 bits.
//
// Beyond 32 rows (queries times heads of a group) a wavefront's operands straight from memory would mean reading the same keys for
// every tile of rows.  Here a workgroup of four wavefronts takes tiles of 128 rows, 32 to a wavefront, and streams the keys and values
// through LDS, 64 at a time, read once for all of them: by loads that go from the pages straight to LDS, one block ahead
// (attention_tiles.h: the image that keeps the reads free of conflicts).  Where no more than 64 rows are there, two wavefronts share
// 32 of them and take half of the keys of a block each.
//
// Bound by the vector and matrix instructions, which overlap as far as the two workgroups of a compute unit are at different steps: 8 requests
// of 8192 tokens, 64 drafted, 32 heads on 8 of 128, 106 to 110 us for 68.7 GFLOP (640 TFLOP/s; 6.9 vector instructions to a matrix one, matrix pipes
// busy a third of the cycles, 274 MB read), of which 10 to 17 are the merge of 38 MB of records.  For heads of 128 all 256 vector registers are taken and
// two more lie in scratch memory.
//
// Score tiles S^T[key][query] = K Q^T and the second product O^T[feature][query] = V^T P^T, whose right operand are the exponentiated
// tiles as the first product leaves them.
#include <type_traits>

#include "attention_paged.h"

namespace dsla {
namespace {

// 16 bytes a lane from `base` (uniform) + `voff` (per lane) into LDS at `lds` (uniform) + 16 * lane.  The compiler does not know these
// loads: whoever reads the bytes waits with loads_landed_barrier() first.  (The five states in front are what a vector memory
// instruction needs behind a vector instruction that wrote its scalar address.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void page_to_lds16(const char *lds, uint32_t voff, const char *base)
{
    const uint32_t at = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char *)lds)));
    const uint64_t p = reinterpret_cast<uint64_t>(base);
    const uint64_t u = static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(p >> 32)))) << 32 | static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(p)));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at), "v"(voff), "s"(u) : "m0", "memory");
}
#pragma clang diagnostic pop

constexpr int kRowsWaves = kRowsTile / 32;

// The arguments, to be read anew: kept over a unit's blocks they would take the registers from what the blocks need.
__device__ __forceinline__ const PagedArgs &arguments()
{
    auto at = __builtin_amdgcn_kernarg_segment_ptr();
    asm("" : "+s"(at));
    return *(const PagedArgs *)at;
}

template <int D>
__global__ __launch_bounds__(64 * kRowsWaves, 2) void attention_paged_rows_kernel(PagedArgs)
{
    const PagedArgs &a = arguments();
    using L = AttnTiles<D>;
    constexpr int NKB = D / 16, CT = D / 32;           // contraction blocks over the features; output tiles of 32 features
    constexpr int RPI = 1024 / L::RB;                  // rows that one load of a wavefront fills
    constexpr int NI = kKeys / RPI / kRowsWaves;          // loads of a wavefront for a block's keys
    __shared__ __attribute__((aligned(1024))) char buf[2 * L::BUF_BYTES];
    __shared__ int s_wild;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ln = lane & 31, g = lane >> 5;
    const int plog = a.c.page_log2, page = 1 << plog;
    const int stretch = stretch_of(a.groups);
    const Line line = read_line(a, stretch, blockIdx.x == 0 && wave == 0);
    if (threadIdx.x == 0) a.open[stretch].parts = 0;
    if (line.total == 0) return;
    int x0 = line.per * stretch, before = line.before, b = line.b;   // (no more than the total)
    const int x1 = line.total - x0 < line.per ? line.total : x0 + line.per;
    Work w = line.w;

    // this lane's place in a load: row lr of its RPI rows, piece position lp
    const uint32_t lr = static_cast<uint32_t>(lane) / L::NC, lp = static_cast<uint32_t>(lane) % L::NC, row0 = RPI * wave + lr;
    const uint32_t goff_k = lr * L::RB + 16 * (lp ^ L::swz_k(row0));
    const uint32_t goff_v = lr * L::RB + 16 * ((((lp >> 2) ^ L::swz_v(row0)) << 2) | (lp & 3u));
    // fragment reads: keys, row 32 t + ln, logical piece 2 kb + g; values, row 4 g + l16 / 4 of 16 keys (+ 8 for the second read)
    const uint32_t sk = L::swz_k(ln), kf_off = ln * L::RB + 16 * ((g ^ sk) & 1u), kf_s1 = sk >> 1;
    const uint32_t l16 = lane & 15, vrow = 4 * g + (l16 >> 2), sv = L::swz_v(vrow), vt_off = vrow * L::RB + 32 * ((lane >> 4) & 1) + 8 * (l16 & 3);
    // the sign of the scale goes into the queries
    const float scale = fabsf(a.scale_log2e);
    const uint32_t flip = a.scale_log2e < 0.f ? 0x80008000u : 0u;

    while (x0 < x1) {
        const PagedArgs &a = arguments();
        while (x0 - before >= w.size()) {   // (also over entries that take no part)
            before += w.size();
            w = read_work(a, ++b, false);
        }
        // the unit at x0, and the granules of it that are the workgroup's
        const int unit = (x0 - before) / w.unit(), at = x0 - before - unit * w.unit();
        const int len = w.unit() - at < x1 - x0 ? w.unit() - at : x1 - x0;
        const int g0 = w.granule(at), take = w.granule(at + len) - g0;
        const int tile = unit % w.tiles, kv = unit / w.tiles;
        if (threadIdx.x == 0 && g0 == 0 && take < w.granules) {
            const int first = x0 - at + w.first();   // the place of the unit's first granule (the workgroup's)
            const int rows = w.n * a.G - tile * a.tile_rows;
            a.open[stretch] = OpenUnit{take > 0 ? (first + ((w.granules - 1) << w.log2_weight)) / line.per - stretch + 1 : 0, w.cu, kv, tile * a.tile_rows, rows < a.tile_rows ? rows : a.tile_rows, {}};
        }
        x0 += len;
        if (take <= 0) continue;
        __syncthreads();   // (the last unit's merge)

        const int live = w.n * a.G - tile * kRowsTile;              // rows
        const bool halves = live <= kRowsTile / 2;                  // (uniform) the first wavefronts the first half of a block's keys, the others the second
        const int my = halves ? wave & (kRowsWaves / 2 - 1) : wave, r = tile * kRowsTile + 32 * my + ln, j = a.token(r);
        const bool works = 32 * my < live, is = j < w.n;
        const uint64_t mask = a.tree ? a.tree[w.cu + (is ? j : 0)] : ~0ull >> (63 - (is ? j : 0));
        bf16x8 qf[NKB];
        {
            const bf16_t *q = static_cast<const bf16_t *>(a.q) + (static_cast<size_t>(w.cu + (is ? j : 0)) * a.H + kv * a.G + r - j * a.G) * D + 8 * g;
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb) {
                u32x4 u = *reinterpret_cast<const u32x4 *>(q + 16 * kb);
#pragma unroll
                for (int e = 0; e < 4; ++e) u[e] = is ? u[e] ^ flip : 0u;
                qf[kb] = __builtin_bit_cast(bf16x8, u);
            }
        }
        f32x16 oacc[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int e = 0; e < 16; ++e) oacc[ct][e] = 0.f;
        float m = -FLT_MAX, z = 0.f;   // z: this lane's share (the other half of the keys is with lane + 32)

        const int from = g0 * kGranule, to = w.granules - g0 == take ? w.L : from + take * kGranule;
        const char *kp = static_cast<const char *>(a.k) + ((static_cast<size_t>(kv) << plog) * L::RB);
        const char *vp = static_cast<const char *>(a.v) + ((static_cast<size_t>(kv) << plog) * L::RB);
        const size_t pitch = (static_cast<size_t>(a.c.H_kv) << plog) * L::RB;
        const int32_t *table = a.c.table + static_cast<size_t>(w.row) * a.c.max_pages;
        const int pages = pages_of(w.L, plog);
        int window = -64, ids = 0;
        unsigned long long none = 0;   // pages of the window that the table gives no number for

        // Starts the loads of the block at t0; which of its four tiles of 16 keys have no page.  (Past the end page 0 of the pool is read.)
        const auto stage = [&](char *to_lds, int t0) {
            if (((t0 >> plog) & ~63) != window) {   // the numbers of 64 pages, one in a lane
                window = (t0 >> plog) & ~63;
                ids = window + lane < pages ? table[window + lane] : 0;
                none = __ballot((ids < 0) | (ids >= a.c.n_pages));
                if (none) {
                    if (tid == 0) report(a.c.status, DSLA_STATUS_CACHE_ENTRY);
                    ids = none >> lane & 1 ? 0 : ids;
                }
            }
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                const int load = wave + kRowsWaves * n, t = t0 + RPI * load;
                const size_t off = static_cast<size_t>(__builtin_amdgcn_readlane(ids, (t >> plog) - window)) * pitch + static_cast<size_t>(t & (page - 1)) * L::RB;
                page_to_lds16(to_lds + load * 1024, goff_k, kp + off);
                page_to_lds16(to_lds + L::K_BYTES + load * 1024, goff_v, vp + off);
            }
            int gap = 0;
#pragma unroll
            for (int s = 0; s < 4; ++s) gap |= static_cast<int>(none >> (((t0 + 16 * s) >> plog) - window) & 1) << s;
            return gap;
        };

        // The block at t0 against this wavefront's rows: NH tiles of 32 keys from tile `half`.
        const auto products = [&](auto tiles, const char *kb_, const char *vb_, int t0, int gap, bool edge, bool wild, int half) {
            constexpr int NH = decltype(tiles)::value;
            const int k0 = t0 + 32 * half;
            f32x16 sc[NH];
#pragma unroll
            for (int t = 0; t < NH; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) sc[t][e] = 0.f;
            // The fragments of keys are asked for kReads products ahead, in an order that is kept: with one ahead, as the compiler has it, every
            // product waits for its own.
            constexpr int kReads = 6;
            bf16x8 kf[kReads];
            const auto read_k = [&](int i) {   // product i: tile i % NH, features 16 (i / NH) and on
                kf[i % kReads] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(kb_ + 32 * (half + i % NH) * L::RB + kf_off + 32 * (i / NH ^ kf_s1)));
            };
#pragma unroll
            for (int i = 0; i < kReads; ++i) read_k(i);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < NH * NKB; ++i) {
                sc[i % NH] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i % kReads], qf[i / NH], sc[i % NH], 0, 0, 0);
                if (i + kReads < NH * NKB) read_k(i + kReads);
                __builtin_amdgcn_sched_barrier(0);
            }
            float factor = scale;
            if (edge) {   // bits counted from key first: a lane's keys are first + 8 (e / 4) + e % 4
#pragma unroll
                for (int t = 0; t < NH; ++t) {
                    const int first = k0 + 32 * t + 4 * g, left = to - first, past = w.start - first;
                    uint32_t there = left >= 32 ? ~0u : left > 0 ? (1u << left) - 1 : 0u;
                    if (gap >> (2 * (half + t)) & 1) there &= 0xffff0000u;
                    if (gap >> (2 * (half + t) + 1) & 1) there &= 0x0000ffffu;
                    const uint32_t drafted = past >= 32 ? ~0u : past > 0 ? static_cast<uint32_t>(mask) << past | ((1u << past) - 1) : static_cast<uint32_t>(mask >> (-past & 63));
                    const uint32_t seen = drafted & there;
#pragma unroll
                    for (int e = 0; e < 16; ++e) sc[t][e] = seen & 1u << (8 * (e / 4) + e % 4) ? sc[t][e] * scale : -INFINITY;
                }
                factor = 1.f;
            }
            float top = sc[0][0];
#pragma unroll
            for (int t = 0; t < NH; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, sc[t][e]);
            top *= factor;
            if (__ballot(top > m + kSlack)) {   // the reference of some query is raised: both lanes of each alike
                top = fmaxf(fmaxf(top, __shfl_xor(top, 32)), m);
                const float c0 = __builtin_amdgcn_exp2f(m - top);
                m = top;
                z *= c0;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int e = 0; e < 16; ++e) oacc[ct][e] *= c0;
            }
            if (__builtin_expect(wild, 0)) {
#pragma unroll
                for (int t = 0; t < NH; ++t)
#pragma unroll 1
                    for (int c = 0; c < 32; ++c) {
                        const int key = k0 + 32 * t + c;
                        if (key < w.start || key >= to || (gap >> (2 * (half + t) + (c >> 4)) & 1)) continue;
                        const int number = page_of(a.c, w.row, key);
                        const bf16_t *row = reinterpret_cast<const bf16_t *>(vp + static_cast<size_t>(number) * pitch) + (key & (page - 1)) * D + 4 * g;
                        float weight = 0.f;
#pragma unroll
                        for (int e = 0; e < 16; ++e) weight = e == 4 * (c >> 3) + (c & 3) ? sc[t][e] : weight;
                        weight = __builtin_amdgcn_exp2f(fmaf(__shfl(weight, ln + 32 * (c >> 2 & 1)), factor, -m));
                        const bool seen = mask >> (key - w.start) & 1;
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                const float f = to_f32(row[32 * ct + 8 * (e / 4) + e % 4]);
                                oacc[ct][e] += seen && not_finite(f) ? f * weight : 0.f;
                            }
                    }
            }
            // 16 keys at a time: the exponentials and the packing of the next ones and the reads of their values run under the products of
            // these.  The weights are rounded to 16 bits for the second product; their sum is that of the rounded ones, so that what the
            // roundings have in common cancels.
            bf16x8 pf[2], vf[2][CT];
            const auto weights = [&](int s, int h) {
                u32x4 pw;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = __builtin_amdgcn_exp2f(fmaf(sc[h / 2][8 * (h % 2) + 2 * e], factor, -m)), y = __builtin_amdgcn_exp2f(fmaf(sc[h / 2][8 * (h % 2) + 2 * e + 1], factor, -m));
                    const uint32_t pair = pack2(x, y);
                    z = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3f803f80u), z, false);
                    pw[e] = pair;
                }
                pf[s] = __builtin_bit_cast(bf16x8, pw);
            };
            const auto read_v = [&](int s, int h) {
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) vf[s][ct] = load_vt_frag(vb_ + vt_off + 16 * (2 * half + h) * L::RB + 64 * (ct ^ sv), 8 * L::RB);
            };
            read_v(0, 0);
            weights(0, 0);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int h = 0; h < 2 * NH; ++h) {
                if (h + 1 < 2 * NH) {
                    read_v((h + 1) & 1, h + 1);
                    weights((h + 1) & 1, h + 1);
                }
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) oacc[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[h & 1][ct], pf[h & 1], oacc[ct], 0, 0, 0);
                if (h + 1 < 2 * NH) {
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) {
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                        __builtin_amdgcn_sched_group_barrier(0x400, 8 / CT, 0);
                        __builtin_amdgcn_sched_group_barrier(0x002, 16 / CT, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            __builtin_amdgcn_s_setprio(0);
        };

        const auto compute = [&](char *at_lds, int t0, int gap) {
            const bool edge = (t0 + kKeys > w.start) | (gap != 0);   // (uniform)
            char *kb_ = at_lds, *vb_ = at_lds + L::K_BYTES;
            bool wild = false;
            if (edge) {
                // What does not exist is zero, and where queries see different tokens an infinity or NaN among them too: zero times it would reach
                // the queries that do not see it.  Those that do get their products one by one.
                const bool tame = (w.n > 1) | (a.tree != nullptr);
                if (tid == 0) s_wild = 0;
                __syncthreads();
                for (int piece = tid; piece < kKeys * L::NC; piece += 64 * kRowsWaves) {
                    const int row = piece / L::NC, t = t0 + row;
                    u32x4 *p = reinterpret_cast<u32x4 *>(vb_) + piece;
                    if (t >= to || (gap >> (row >> 4) & 1)) {
                        *p = u32x4{0, 0, 0, 0};
                    } else if (tame && t >= w.start) {
                        u32x4 x = *p;
                        uint32_t any = 0;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t bad = ((x[e] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((x[e] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
                            x[e] &= ~bad;
                            any |= bad;
                        }
                        if (any) {
                            *p = x;
                            s_wild = 1;
                        }
                    }
                }
                __syncthreads();
                wild = s_wild != 0;
            }
            if (!works) return;
            if (halves) products(std::integral_constant<int, 1>(), kb_, vb_, t0, gap, edge, wild, wave / (kRowsWaves / 2));
            else products(std::integral_constant<int, 2>(), kb_, vb_, t0, gap, edge, wild, 0);
        };

        // Block n lives in buffer n % 2; its loads are issued one block ahead, right after the barrier that frees the buffer.  (Its lines asked for
        // yet a block earlier, so that the loads find them in the L2: 106 -> 118 us; what bounds the loop is not their latency.)
        const int blocks = (to - from + kKeys - 1) / kKeys;
        int gaps = stage(buf, from);   // four bits of each block that is staged
        for (int n = 0; n < blocks; ++n) {
            loads_landed_barrier();   // the block is there; every wavefront is done with the one before
            if (n + 1 < blocks) gaps |= stage(buf + (n + 1) % 2 * L::BUF_BYTES, from + (n + 1) * kKeys) << 4;
            compute(buf + n % 2 * L::BUF_BYTES, from + n * kKeys, gaps & 15);
            gaps >>= 4;
        }

        z += __shfl_xor(z, 32);
        if (halves) {   // the second half's wavefronts into the first's
            float *s = reinterpret_cast<float *>(buf) + (wave & (kRowsWaves / 2 - 1)) * (CT * 16 + 2) * 64 + lane;
            __syncthreads();
            if (wave >= kRowsWaves / 2) {
                s[0] = m;
                s[64] = z;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[(2 + 16 * ct + e) * 64] = oacc[ct][e];
            }
            __syncthreads();
            if (wave >= kRowsWaves / 2) continue;
            const float mo = s[0], top = fmaxf(m, mo), c0 = __builtin_amdgcn_exp2f(m - top), c1 = __builtin_amdgcn_exp2f(mo - top);
            m = top;
            z = c0 * z + c1 * s[64];
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int e = 0; e < 16; ++e) oacc[ct][e] = c0 * oacc[ct][e] + c1 * s[(2 + 16 * ct + e) * 64];
        }
        if (!is) continue;
        const PagedArgs &out = arguments();
        int at_row = lane & 31;
        asm("" : "+v"(at_row));
        at_row += tile * kRowsTile + 32 * my;
        const int at_token = out.token(at_row);
        if (take == w.granules) {
            uint32_t *o = reinterpret_cast<uint32_t *>(static_cast<bf16_t *>(out.o) + (static_cast<size_t>(w.cu + at_token) * out.H + kv * out.G + at_row - at_token * out.G) * D + 4 * g);
            const float inv = z == 0.f ? 0.f : 1.f / z;   // (a query that sees nothing: zeros)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *reinterpret_cast<u32x2 *>(o + 16 * ct + 4 * e) = u32x2{pack2(oacc[ct][4 * e] * inv, oacc[ct][4 * e + 1] * inv), pack2(oacc[ct][4 * e + 2] * inv, oacc[ct][4 * e + 3] * inv)};
        } else {
            // a stretch has no more than one unit that began before it (record 0) and one that goes on after it (record 1)
            const size_t rec = (2 * static_cast<size_t>(stretch) + (g0 == 0)) * kRowsTile + 32 * my + ln;
            if (g == 0) out.stats[rec] = make_float2(m, z);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *reinterpret_cast<f32x4 *>(out.sums + rec * D + 32 * ct + 8 * e + 4 * g) = f32x4{oacc[ct][4 * e], oacc[ct][4 * e + 1], oacc[ct][4 * e + 2], oacc[ct][4 * e + 3]};
        }
    }
}

}  // namespace

hipError_t launch_attention_paged_rows(const PagedArgs &a, ProfileScope &ps, hipStream_t stream)
{
    auto kernel = a.c.d == 128 ? attention_paged_rows_kernel<128> : attention_paged_rows_kernel<64>;
    DSLA_LAUNCH_FIRST(ps, kernel, dim3(static_cast<unsigned>(a.groups)), dim3(64 * kRowsWaves), 0, stream, a);
    return hipGetLastError();
}

}  // namespace dsla
