// The projections with e4m3 operands and a scale for each block of 128 (include/dsla.h: dsla_project_fp8):
//     out_j[m][c] = sum_b sx[m][b] sw[c / 128][b] sum_{k in block b} x[m][k] W_j[c][k] (+ bias_j[c])
// One MFMA of 16 x 16 x 128 covers a block of K.  E8M0 scales ride in the instruction; with fp32 scales it starts from zero and the
// block's sum is added times sx sw.  Columns are counted in blocks of 128 that never cross an output, as the scales of W are.
//
// Kernels (choose() has the rule): 256 x 256 tiles here, for outputs that fill the chip with them; tiles of 16 to 128 rows and columns with K
// shared by the wavefronts (project_fp8_rows.h) for everything smaller and for results in fp32.
#include "project_fp8.h"

#include <type_traits>

namespace dsla {
namespace {

// 16 bytes per lane from a buffer (lane offset `voff`, uniform offset `soff`) into LDS at `lds` (uniform) + 16 * lane
__device__ __forceinline__ void buffer_load_lds16(__amdgpu_buffer_rsrc_t res, char *lds, uint32_t voff, int soff)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(res, (__attribute__((address_space(3))) void *)(lds), 16, voff, soff, 0, 0);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const uint8_t *p, size_t offset, long long bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p + offset), 0, static_cast<int>(bytes), 0x00020000);
}

// ---------------------------------------------------------------------------------------------------------------
// 256 x 256 tiles
// ---------------------------------------------------------------------------------------------------------------
// A workgroup has 256 rows of x and 256 of W, and K in steps of 128 through two LDS buffers of 64 KB, filled by buffer loads that write LDS directly.
// E8M0: four wavefronts, one to a SIMD, with 128 x 128 results in 256 accumulation registers: 64 MFMAs a step for 32 LDS reads of 16 bytes.  fp32
// scales: the sums take vector instructions, which have no access to those registers: eight wavefronts with 128 x 64 results each.
// 16 x 16 x 128 products: registers only, random operands, they sustain 4.45 PFLOP/s, 32 x 32 x 64 4.1.
// M = 16384, K = 4096, N = 20480, E8M0: 0.99 to 1.05 ms from box to box (2620 to 2790 TFLOP/s; a library product of that shape without block scales 0.96);
// with fp32 scales 1.22.  Bound by power: the chip runs it at 1.72 GHz with the matrix pipes 67 % busy.  On the way: loads of a step in one go behind a barrier 1.24 ms (they keep the address unit busy for
// longer than the products they stand among, and the wavefront with them), spread over two thirds of the step 1.14, results 16 rows at a time through LDS
// without checks in whole tiles 1.07, scales through LDS by 16 bytes of a row instead of one at a time from memory 1.01 (with fp32 scales 1.93 -> 1.23 ms:
// an instruction that asks for one scale of 16 rows costs as much as two that fill 8 rows), read in front of the loads 1.23.  One barrier a step instead of
// two, which gives a load 1.4 steps instead of one to arrive, is the same: latency is not what bounds it.  K = 128: 10 us a tile, of which 6 are the start.
// The product of two fragments added to what stands in the accumulation registers, with scales from byte B of two registers.  (The
// compiler gives the result registers of its own and copies, which 256 accumulators leave no room for.)
template <int B>
__device__ __forceinline__ void product_in_place(f32x4 &acc, const i32x8 &w, const i32x8 &x, uint32_t scale_w, uint32_t scale_x)
{
    if (B) asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[0,0,0]" : "+a"(acc) : "v"(w), "v"(x), "v"(scale_w), "v"(scale_x));
    else asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]" : "+a"(acc) : "v"(w), "v"(x), "v"(scale_w), "v"(scale_x));
}

template <bool E8M0>
__global__ __launch_bounds__(E8M0 ? 256 : 512) void project_fp8_tile_kernel(Fp8Args a, int tiles_m, int tiles_n, int blocks, int group, long long per_xcd)
{
    constexpr int WN = E8M0 ? 2 : 4, NW = 2 * WN;    // wavefronts along the columns, in all
    constexpr int NJ = 16 / WN;                       // 16 x 16 tiles of a wavefront along the columns; 8 along the rows
    constexpr int OPB = 256 * 128;                    // bytes of an operand's tile and step
    constexpr int LOADS = 32 / NW;                    // instructions of a wavefront per operand and step
    __shared__ __attribute__((aligned(1024))) char st0[2 * OPB];
    __shared__ __attribute__((aligned(1024))) char st1[2 * OPB];
    int tm, tn;
    if (!tile_here(tiles_m, tiles_n, group, per_xcd, tm, tn)) return;
    const long long m0 = 256LL * tm;
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
    const int second = 2 * tn + 1 < blocks ? 2 * tn + 1 : 2 * tn;
    const Columns cb0 = columns_of(a, 2 * tn);
    Columns cb1 = columns_of(a, second);
    if (second == 2 * tn) cb1.count = 0;

    // ---- loading: an instruction fills 8 rows of 128 bytes; lane l fills position l % 8 of row l / 8, where piece c of a row R sits at
    // c ^ (R / 2 % 8).  The pieces behind K are asked for nowhere, and come as zeros, as rows that do not exist do. ----
    const long long rows_a = a.M - m0 < 256 ? a.M - m0 : 256;
    const __amdgpu_buffer_rsrc_t res_x = buffer_of(a.x, static_cast<size_t>(m0) * a.K, rows_a * a.K);
    const __amdgpu_buffer_rsrc_t res_w0 = buffer_of(a.w, static_cast<size_t>(cb0.row) * a.K, static_cast<long long>(cb0.count) * a.K);
    const __amdgpu_buffer_rsrc_t res_w1 = buffer_of(a.w, static_cast<size_t>(cb1.row) * a.K, static_cast<long long>(cb1.count) * a.K);
    const int piece = (lane & 7) ^ (((8 * wave + (lane >> 3)) >> 1) & 7);   // (the same for all of its rows: they are 8 NW apart)
    uint32_t voff[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) voff[i] = static_cast<uint32_t>(8 * (wave + NW * i) + (lane >> 3)) * static_cast<uint32_t>(a.K) + 16 * piece;
    auto fetch_x = [&](char *st, int ks, int i) {   // instruction i of an operand
        const int k0 = 128 * ks;
        buffer_load_lds16(res_x, st + (wave + NW * i) * 1024, 16 * piece < a.K - k0 ? voff[i] : kNowhere, k0);
    };
    auto fetch_w = [&](char *st, int ks, int i) {
        const int k0 = 128 * ks;
        const bool there = 16 * piece < a.K - k0;
        if (i < LOADS / 2) buffer_load_lds16(res_w0, st + OPB + (wave + NW * i) * 1024, there ? voff[i] : kNowhere, k0);
        else buffer_load_lds16(res_w1, st + OPB + (wave + NW * i) * 1024, there ? voff[i - LOADS / 2] : kNowhere, k0);
    };
    auto fetch = [&](char *st, int ks) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            fetch_x(st, ks, i);
            fetch_w(st, ks, i);
        }
    };

    // ---- scales: 16 bytes of every row at a time, for CHUNK steps, through LDS (an instruction that asks for one scale of 16 rows asks for as
    // many lines as two that fill 8 rows: with fp32 scales these were two thirds of all) ----
    const int nk = (a.K + 127) / 128;
    constexpr int SB = E8M0 ? 1 : 4, CHUNK = 16 / SB, SLOT = 4096 + 1024;
    __shared__ __attribute__((aligned(16))) char scales[3 * SLOT];
    const uint32_t row_scales = static_cast<uint32_t>(a.pitch) * SB;
    const __amdgpu_buffer_rsrc_t res_xs = buffer_of(static_cast<const uint8_t *>(a.xs), static_cast<size_t>(m0) * row_scales, rows_a * row_scales);
    const __amdgpu_buffer_rsrc_t res_ws = buffer_of(static_cast<const uint8_t *>(a.ws), static_cast<size_t>(2 * tn) * row_scales, (second - 2 * tn + 1) * row_scales);
    const uint32_t xs_from = static_cast<uint32_t>(64 * (wave & 3) + lane) * row_scales;
    const uint32_t ws_from = lane < 2 ? (lane ? (second - 2 * tn) * row_scales : 0u) : kNowhere;
    auto fetch_scales = [&](int ks, bool now = true) {   // of steps ks .. ks + CHUNK - 1; not now: nothing, to where nobody reads
        char *to = scales + (now ? ks / CHUNK & 1 : 2) * SLOT;
        buffer_load_lds16(res_xs, to + (wave & 3) * 1024, now ? xs_from : kNowhere, ks * SB);
        buffer_load_lds16(res_ws, to + 4096, now ? ws_from : kNowhere, ks * SB);
    };
    struct Scales {
        uint32_t x[8], w;
    };
    const uint32_t xs_at = static_cast<uint32_t>(128 * wm + r) * 16, ws_at = 4096u + static_cast<uint32_t>(wn / (WN / 2)) * 16;
    auto read_scales = [&](Scales &s, int ks) {   // E8M0: of steps ks and ks + 1 (ks even)
        const char *from = scales + (ks / CHUNK & 1) * SLOT + ks % CHUNK * SB;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (E8M0) s.x[i] = *reinterpret_cast<const uint16_t *>(from + xs_at + i * 256);
            else s.x[i] = *reinterpret_cast<const uint32_t *>(from + xs_at + i * 256);
        }
        s.w = E8M0 ? *reinterpret_cast<const uint16_t *>(from + ws_at) : *reinterpret_cast<const uint32_t *>(from + ws_at);
    };
    // What stands behind a row's last scale may be anything, and its products are of zeros: one.
    auto close_scales = [&](Scales &s, int ks) {
        const uint32_t keep = ks + 1 < nk ? 0xffffu : 0xffu, put = ks + 1 < nk ? 0u : 0x7f00u;
#pragma unroll
        for (int i = 0; i < 8; ++i) s.x[i] = (s.x[i] & keep) | put;
        s.w = (s.w & keep) | put;
    };

    // ---- fragments: lane (r, g) holds row r, pieces g and 4 + g ----
    const uint32_t pos = static_cast<uint32_t>(g ^ ((r >> 1) & 7)) << 4;
    const uint32_t fx = static_cast<uint32_t>(128 * wm + r) * 128, fw = OPB + static_cast<uint32_t>(16 * NJ * wn + r) * 128;
    auto fragment = [&](const char *st, uint32_t row) {
        return join(*reinterpret_cast<const u32x4 *>(st + row + pos), *reinterpret_cast<const u32x4 *>(st + row + (pos ^ 64)));
    };
    f32x4 acc[8][NJ];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if constexpr (E8M0) {
        // A step multiplies rows of tiles 0 and 1 column by column, then rows 2 .. 4, then 5 .. 7 column by column.  On entry the fragments of the
        // columns and of rows 0 and 1 are in registers or on their way; the other rows' are read under the first products.  Then everybody
        // has all it needs of `cur`, says so at a barrier, and the loads of step ks + 2 go there.  In front of the last rows a second barrier
        // says that step ks + 1 has landed in `nxt`: as these rows are done with a column, the next step's fragment takes its registers.
        // So a load has 1.4 steps to arrive; with one barrier for both it has one.
        i32x8 w[NJ], x[8];
        auto product = [&](int i, int j, const Scales &s, auto odd) {
            product_in_place<decltype(odd)::value>(acc[i][j], w[j], x[i], s.w, s.x[i]);
        };
        auto step = [&](const Scales &s, Scales &ns, char *cur, char *nxt, int ks, auto odd) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                if (j < 6) x[2 + j] = fragment(cur, fx + (2 + j) * 2048);
#pragma unroll
                for (int i = 0; i < 2; ++i) product(i, j, s, odd);
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                fetch_x(cur, ks + 2, j);
#pragma unroll
                for (int i = 2; i < 5; ++i) product(i, j, s, odd);
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_waitcnt(0x0f78);   // vmcnt(8): all but what this step has asked for
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
            if (decltype(odd)::value == 0 && (ks + 2) % CHUNK == 0) fetch_scales(ks + 2);
            if (decltype(odd)::value) read_scales(ns, ks + 1);
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                fetch_w(cur, ks + 2, j);
#pragma unroll
                for (int i = 5; i < 8; ++i) product(i, j, s, odd);
                w[j] = fragment(nxt, fw + j * 2048);
                if (j < 2) x[j] = fragment(nxt, fx + j * 2048);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        Scales s0, s1;
        fetch_scales(0);
        fetch(st0, 0);
        fetch(st1, 1);
        __builtin_amdgcn_s_waitcnt(0x0070);
        __builtin_amdgcn_s_barrier();
        read_scales(s0, 0);
#pragma unroll
        for (int i = 0; i < 2; ++i) x[i] = fragment(st0, fx + i * 2048);
#pragma unroll
        for (int j = 0; j < NJ; ++j) w[j] = fragment(st0, fw + j * 2048);
        for (int ks = 0; ks < nk; ks += 2) {
            close_scales(s0, ks);
            asm volatile("s_nop 1" : "+v"(s0.w), "+v"(s0.x[0]), "+v"(s0.x[1]), "+v"(s0.x[2]), "+v"(s0.x[3]), "+v"(s0.x[4]), "+v"(s0.x[5]), "+v"(s0.x[6]), "+v"(s0.x[7]));
            step(s0, s1, st0, st1, ks, std::integral_constant<int, 0>{});
            step(s0, s1, st1, st0, ks + 1, std::integral_constant<int, 1>{});
            s0 = s1;
        }
        asm volatile("s_nop 15");
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j) asm volatile("" : "+a"(acc[i][j]));
    } else {
        // Two wavefronts to a SIMD, one buffer read while the other fills; a row of tiles' sums are added under the next row's products.
        auto step = [&](char *cur, char *nxt, int ks) {
            __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
            __builtin_amdgcn_s_barrier();         // step ks has landed, and everybody is done with the other buffer
            __builtin_amdgcn_sched_barrier(0);
            Scales s;
            read_scales(s, ks);   // (ahead of the loads: behind them it would wait for them)
            __builtin_amdgcn_sched_barrier(0);
            fetch(nxt, ks + 1);
            fetch_scales(ks + 1, (ks + 1) % CHUNK == 0);   // (a branch here, and the accumulators do not stay where they are)
            i32x8 w[NJ], x[2];
            x[0] = fragment(cur, fx);
#pragma unroll
            for (int j = 0; j < NJ; ++j) w[j] = fragment(cur, fw + j * 2048);
            // product n starts from zero, and its sums are added three products later
            constexpr int BEHIND = 3;
            f32x4 t[BEHIND + 1];
            float scale[8];
#pragma unroll
            for (int n = 0; n < 8 * NJ + BEHIND; ++n) {
                const int i = n / NJ, j = n % NJ, k = n - BEHIND;
                if (j == 0 && i < 7) x[(i + 1) & 1] = fragment(cur, fx + (i + 1) * 2048);
                if (j == 0 && i < 8) scale[i] = __uint_as_float(s.x[i]) * __uint_as_float(s.w);
                if (n < 8 * NJ) t[n % (BEHIND + 1)] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[j], x[i & 1], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, kOne, 0, kOne);
                if (k >= 0)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[k / NJ][k % NJ][e] += t[k % (BEHIND + 1)][e] * scale[k / NJ];
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        fetch_scales(0);
        fetch(st0, 0);
        int ks = 0;
        for (; ks + 1 < nk; ks += 2) {
            step(st0, st1, ks);
            step(st1, st0, ks + 1);
        }
        if (ks < nk) step(st0, st1, ks);
    }
    __builtin_amdgcn_s_waitcnt(0x0070);
    __builtin_amdgcn_s_barrier();   // nothing in flight; everybody is done reading

    // ---- results: each wavefront turns a row of tiles at a time round in LDS, 16 rows of 16 NJ columns in bf16, the 16-byte piece c of row R
    // at position c ^ (R % pieces), so that they leave as whole rows.  (A wavefront's LDS instructions keep their order: it waits for nobody.) ----
    constexpr int PPR = 2 * NJ, ROWB = 32 * NJ, READS = 16 * PPR / 64;
    const Columns c = wn / (WN / 2) ? cb1 : cb0;
    const int first = (16 * NJ * wn) % 128;   // the wavefront's first column in its block
    char *epi = st0 + wave * 2 * 16 * ROWB;
    const int width = a.width[c.j], at = lane % PPR, sub = lane / PPR;
    const bool there = first + 8 * at < c.count;
    const long long left = a.M - m0 - 128 * wm;   // rows of the wavefront's that exist
    bf16_t *out = static_cast<bf16_t *>(a.out[c.j]) + static_cast<size_t>(m0 + 128 * wm + sub) * width + c.c0 + first + 8 * at;
    auto leave = [&](auto with_bias, auto whole) {
        constexpr bool BIAS = decltype(with_bias)::value, WHOLE = decltype(whole)::value;
        f32x4 bias[NJ];
        if (BIAS) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int col = first + 16 * j + 4 * g;
                bias[j] = a.bias && col < c.count ? *reinterpret_cast<const f32x4 *>(a.bias + c.row + col) : f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            char *turn = epi + (i & 1) * 16 * ROWB;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
                *reinterpret_cast<u32x2 *>(turn + r * ROWB + (((2 * j + (g >> 1)) ^ (r & (PPR - 1))) << 4) + (g & 1) * 8) = pack4(BIAS ? acc[i][j] + bias[j] : acc[i][j]);
#pragma unroll
            for (int q = 0; q < READS; ++q) {
                const int row = 64 / PPR * q + sub;
                const u32x4 v = *reinterpret_cast<const u32x4 *>(turn + row * ROWB + ((at ^ (row & (PPR - 1))) << 4));
                if (WHOLE || (there && 16 * i + row < left)) __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(out));
                out += static_cast<size_t>(64 / PPR) * width;
            }
        }
    };
    if (left < 128 || first + 16 * NJ > c.count) leave(std::true_type{}, std::false_type{});
    else if (a.bias) leave(std::true_type{}, std::true_type{});
    else leave(std::false_type{}, std::true_type{});
}

// ---------------------------------------------------------------------------------------------------------------
// Which kernel, which tiles
// ---------------------------------------------------------------------------------------------------------------
struct Pair {
    int8_t mt, nt;
};
constexpr Pair kPairs[] = {{1, 1}, {1, 2}, {1, 3}, {1, 4}, {1, 5}, {2, 1}, {2, 2}, {2, 3}, {2, 4}, {2, 5}, {3, 2}, {3, 3}, {3, 4}, {3, 5}, {4, 2}, {4, 3},
                           {4, 4}, {4, 5}, {4, 6}, {4, 8}, {5, 4}, {5, 5}, {6, 4}, {6, 5}, {6, 6}, {8, 4}, {8, 5}, {8, 6}, {5, 8}, {6, 8}, {8, 8}};
constexpr int kExactPairs = 27;   // of them for results in fp32

struct Choice {
    int mt, nt;   // 0: the 256 x 256 tiles
    double us;
};
// The fewest microseconds by an estimate, fitted to 9600 timings of random products of up to 8192 rows and pairs.  Of 13579 others, of the kernels as they are,
// it is 9 to 13 % off (rms) for the pairs and 30 % too long for the 256 x 256 tiles; what it chooses takes 1.01 of the best's time (geometric mean of 1569
// products, the worst 1.35).  A round of workgroups over the compute units costs its start, its sums (mt nt), and for every 1024 of K its loads (mt + nt) and
// products (mt nt); beside that the memory.
struct Cost {
    double call, round, sums, loads, products, next;
};
constexpr Cost kRowsCost[3] = {{2.6, 0.48, 0.13, 0.117, 0.029, 1.6},     // E8M0
                               {2.2, 0.83, 0.147, 0.083, 0.074, 1.0},    // fp32 scales: sums by vector instructions
                               {2.0, 1.2, 0.155, 0.10, 0.11, 0.9}};      // results in fp32: operands in bf16
constexpr double kTileRound[2][2] = {{7.0, 10.4}, {4.0, 13.0}};           // 256 x 256 tiles, E8M0 and fp32: of a round, and for every 1024 of K
Choice choose(long long M, int K, int N, int blocks, bool e8m0, bool exact)
{
    const double k = 128.0 * ((K + 127) / 128) / 1024;
    const double memory = 2.5 + ((static_cast<double>(M) + N) * K + static_cast<double>(M) * N * (exact ? 4 : 2)) / 6.2e6;
    const auto both = [&](double work) { return work > memory ? work + 0.2 * memory : memory + 0.2 * work; };
    const Cost &c = kRowsCost[exact ? 2 : (e8m0 ? 0 : 1)];
    Choice best{0, 0, 1e30};
    for (int n = 0; n < (exact ? kExactPairs : static_cast<int>(sizeof(kPairs) / sizeof(Pair))); ++n) {
        const int mt = kPairs[n].mt, nt = kPairs[n].nt;
        if (mt > 1 && 16LL * (mt - 1) >= M) continue;   // rows of tiles that nobody needs
        const long long tiles_m = (M + 16 * mt - 1) / (16 * mt), tiles_n = (N + 16 * nt - 1) / (16 * nt);
        if (tiles_m * tiles_n > 0x70000000LL) continue;
        const double rounds = static_cast<double>((fp8_rows_per_xcd(tiles_m, tiles_n) + 31) / 32), p = mt + nt, q = mt * nt;
        const double us = both(c.call + rounds * (c.round + c.sums * q + (c.loads * p + c.products * q) * k) + c.next * (rounds - 1));
        if (us < best.us) best = Choice{mt, nt, us};
    }
    if (!exact) {
        const double tiles = static_cast<double>((M + 255) / 256) * ((blocks + 1) / 2), rounds = __builtin_ceil(tiles / 256);
        const double us = both(3 + rounds * (kTileRound[!e8m0][0] + kTileRound[!e8m0][1] * k));
        if (us < best.us) best = Choice{0, 0, us};
    }
    return best;
}
}  // namespace

hipError_t launch_project_fp8(int64_t M, int K, int n_out, const int32_t *widths, int scale_type, const void *x, const void *x_scale, const void *w,
                              const void *w_scale, const float *bias, int out_dtype, void *const *outs, hipStream_t stream)
{
    Fp8Args a{};
    a.x = static_cast<const uint8_t *>(x);
    a.w = static_cast<const uint8_t *>(w);
    a.xs = x_scale;
    a.ws = w_scale;
    a.bias = bias;
    a.M = M;
    a.K = K;
    a.pitch = scale_pitch(K);
    a.out_f32 = out_dtype == DSLA_F32;
    int blocks = 0, N = 0;
    for (int j = 0; j < DSLA_MAX_PROJECTIONS; ++j) {
        a.out[j] = j < n_out ? outs[j] : nullptr;
        a.width[j] = j < n_out ? widths[j] : 0;
        blocks += (a.width[j] + 127) / 128;
        N += a.width[j];
    }
    ProfileScope ps(DSLA_KERNEL_PROJECT_FP8, stream);
    const bool e8m0 = scale_type == DSLA_SCALE_E8M0, exact = out_dtype == DSLA_F32;
    const Choice c = choose(M, K, N, blocks, e8m0, exact);
    if (c.mt) {
        if (!(exact ? launch_fp8_rows_exact : launch_fp8_rows)(ps, a, N, c.mt, c.nt, e8m0, stream)) return hipErrorInvalidValue;
        return hipGetLastError();
    }
    const int tiles_m = static_cast<int>((M + 255) / 256), tiles_n = (blocks + 1) / 2;
    const long long per_xcd = (static_cast<long long>(tiles_m) * tiles_n + 7) / 8;
    const dim3 block(e8m0 ? 256 : 512), grid = grid_of(8 * per_xcd, block.x);
    const int group = tiles_m <= 5 ? tiles_m : 4;
    if (e8m0) DSLA_LAUNCH(ps, project_fp8_tile_kernel<true>, grid, block, 0, stream, a, tiles_m, tiles_n, blocks, group, per_xcd);
    else DSLA_LAUNCH(ps, project_fp8_tile_kernel<false>, grid, block, 0, stream, a, tiles_m, tiles_n, blocks, group, per_xcd);
    return hipGetLastError();
}

}  // namespace dsla
