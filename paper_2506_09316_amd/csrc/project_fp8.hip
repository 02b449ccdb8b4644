// The projections with e4m3 operands and a scale for each block of 128 (include/dsla.h: dsla_project_fp8):
//     out_j[m][c] = sum_b sx[m][b] sw[c / 128][b] sum_{k in block b} x[m][k] W_j[c][k] (+ bias_j[c])
// One MFMA of 16 x 16 x 128 covers a block of K.  E8M0 scales ride in the instruction; with fp32 scales it starts from zero and the
// block's sum is added times sx sw.  Columns are counted in blocks of 128 that never cross an output, as the scales of W are.
#include "fp8_common.h"
#include "project_common.h"

#include <type_traits>

namespace dsla {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct Fp8Args {
    const uint8_t *x, *w;
    const void *xs, *ws;
    const float *bias;
    void *out[DSLA_MAX_PROJECTIONS];
    int width[DSLA_MAX_PROJECTIONS];
    long long M;
    int K, pitch, out_f32;
};

// A block of 128 columns: its output, where it starts there and in W, and how many columns exist.
struct Columns {
    int j, c0, row, count;
};
__device__ __forceinline__ Columns columns_of(const Fp8Args &a, int block)
{
    Columns c{0, 0, 0, 0};
    int n = (a.width[0] + 127) / 128;
    while (block >= n) {
        block -= n;
        c.row += a.width[c.j++];
        n = (a.width[c.j] + 127) / 128;
    }
    c.c0 = 128 * block;
    c.row += c.c0;
    c.count = a.width[c.j] - c.c0 < 128 ? a.width[c.j] - c.c0 : 128;
    return c;
}

__device__ __forceinline__ u32x2 pack4(f32x4 v)
{
    return u32x2{f32_to_bf16_bits(v[0]) | static_cast<uint32_t>(f32_to_bf16_bits(v[1])) << 16, f32_to_bf16_bits(v[2]) | static_cast<uint32_t>(f32_to_bf16_bits(v[3])) << 16};
}
__device__ __forceinline__ void store4(const Fp8Args &a, const Columns &c, long long m, int col, f32x4 v)   // columns col .. col + 3 of the block
{
    if (a.bias) v += *reinterpret_cast<const f32x4 *>(a.bias + c.row + col);
    const size_t at = static_cast<size_t>(m) * a.width[c.j] + c.c0 + col;
    if (a.out_f32) {
        *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out[c.j]) + at) = v;
    } else {
        *reinterpret_cast<u32x2 *>(static_cast<bf16_t *>(a.out[c.j]) + at) = pack4(v);
    }
}

constexpr int kOne = 127;   // E8M0

__device__ __forceinline__ i32x8 join(u32x4 a, u32x4 b)
{
    return i32x8{static_cast<int>(a[0]), static_cast<int>(a[1]), static_cast<int>(a[2]), static_cast<int>(a[3]),
                 static_cast<int>(b[0]), static_cast<int>(b[1]), static_cast<int>(b[2]), static_cast<int>(b[3])};
}

// The product of two fragments from zero.  EXACT: e4m3 is bf16 with fewer bits, and the bf16 instructions add in fp32; the e4m3 ones add in
// groups of eight products and drop what is below 2^-14 of a group's largest (random operands: 1.4e-5 of the result's 2-norm against
// 1e-8), which results in bf16 do not show and results in fp32 are asked for.
__device__ __forceinline__ bf16x8 wide(uint32_t a, uint32_t b)
{
    const bf16x2 w[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true)};
    return bf16x8{w[0][0], w[0][1], w[1][0], w[1][1], w[2][0], w[2][1], w[3][0], w[3][1]};
}
template <bool EXACT>
struct Operand {
    i32x8 f;
    __device__ __forceinline__ void set(i32x8 x) { f = x; }
};
template <>
struct Operand<true> {
    bf16x8 f[4];
    __device__ __forceinline__ void set(i32x8 x)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = wide(x[2 * i], x[2 * i + 1]);
    }
};
__device__ __forceinline__ f32x4 product(const Operand<false> &w, const Operand<false> &x)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.f, x.f, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, kOne, 0, kOne);
}
__device__ __forceinline__ f32x4 product(const Operand<true> &w, const Operand<true> &x)
{
    f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.f[i], x.f[i], t, 0, 0, 0);
    return t;
}
// What a block's products are multiplied by: two numbers, or 2^exponent (two bytes reach beyond fp32; 255 is NaN).
template <bool E8M0>
struct Factor {
    float f;
    int exponent = 0;
    __device__ __forceinline__ Factor(uint32_t x, uint32_t w)
    {
        if (E8M0) {
            f = x == 255u || w == 255u ? __builtin_nanf("") : 1.f;
            exponent = static_cast<int>(x + w) - 2 * kOne;
        } else {
            f = __uint_as_float(x) * __uint_as_float(w);
        }
    }
    __device__ __forceinline__ void add(f32x4 &acc, f32x4 t) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += (E8M0 ? ldexpf(t[e], exponent) : t[e]) * f;
    }
};

template <bool E8M0, bool EXACT>
__global__ __launch_bounds__(256) void project_fp8_kernel(Fp8Args a, unsigned tiles_m)
{
    __shared__ __attribute__((aligned(16))) u32x4 sx[128 * 8], sw[128 * 8];
    const int block = blockIdx.x / tiles_m;
    const long long m0 = 128LL * (blockIdx.x - static_cast<unsigned>(block) * tiles_m);
    const Columns cb = columns_of(a, block);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, g = lane >> 4;
    const int wm = wave >> 1, wn = wave & 1;
    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int nk = (a.K + 127) / 128;
    for (int ks = 0; ks < nk; ++ks) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = tid + 256 * i, row = n >> 3, c = n & 7, k = 128 * ks + 16 * c, at = row * 8 + (c ^ ((row >> 1) & 7));
            sx[at] = m0 + row < a.M && k < a.K ? *reinterpret_cast<const u32x4 *>(a.x + static_cast<size_t>(m0 + row) * a.K + k) : u32x4{0, 0, 0, 0};
            sw[at] = row < cb.count && k < a.K ? *reinterpret_cast<const u32x4 *>(a.w + static_cast<size_t>(cb.row + row) * a.K + k) : u32x4{0, 0, 0, 0};
        }
        __syncthreads();
        Operand<EXACT> fx[4], fw[4];
        uint32_t scale_x[4];
        auto scale_at = [&](const void *p, size_t row) -> uint32_t {
            return E8M0 ? static_cast<const uint8_t *>(p)[row * a.pitch + ks] : static_cast<const uint32_t *>(p)[row * a.pitch + ks];
        };
        const uint32_t scale_w = scale_at(a.ws, block);   // (a row of scales for every block of columns)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int rx = 64 * wm + 16 * i + r, rw = 64 * wn + 16 * i + r;
            fx[i].set(join(sx[rx * 8 + (g ^ ((rx >> 1) & 7))], sx[rx * 8 + ((4 + g) ^ ((rx >> 1) & 7))]));
            fw[i].set(join(sw[rw * 8 + (g ^ ((rw >> 1) & 7))], sw[rw * 8 + ((4 + g) ^ ((rw >> 1) & 7))]));
            scale_x[i] = m0 + rx < a.M ? scale_at(a.xs, m0 + rx) : 0u;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Factor<E8M0> factor(scale_x[i], scale_w);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (E8M0 && !EXACT) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[j].f, fx[i].f, acc[i][j], 0, 0, 0, scale_w, 0, scale_x[i]);
                else factor.add(acc[i][j], product(fw[j], fx[i]));
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const long long m = m0 + 64 * wm + 16 * i + r;
        if (m >= a.M) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int col = 64 * wn + 16 * j + 4 * g;
            if (col < cb.count) store4(a, cb, m, col, acc[i][j]);
        }
    }
}
// 16 bytes per lane from a buffer (lane offset `voff`, uniform offset `soff`) into LDS at `lds` (uniform) + 16 * lane
__device__ __forceinline__ void buffer_load_lds16(__amdgpu_buffer_rsrc_t res, char *lds, uint32_t voff, int soff)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(res, (__attribute__((address_space(3))) void *)(lds), 16, voff, soff, 0, 0);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const uint8_t *p, size_t offset, long long bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p + offset), 0, static_cast<int>(bytes), 0x00020000);
}
// An offset past the end of every buffer here: zeros.  (The range of a buffer is checked dword by dword, with both offsets.)
constexpr uint32_t kNowhere = 0x80000000u;

// ---------------------------------------------------------------------------------------------------------------
// 256 x 256 tiles
// ---------------------------------------------------------------------------------------------------------------
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
    if (!tile_of(tiles_m, tiles_n, group, per_xcd, tm, tn)) return;
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
// Few rows: the weights are the traffic
// ---------------------------------------------------------------------------------------------------------------
// A workgroup has 16 MT rows and 16 NT columns; its wavefronts take a stretch of K each and share nothing until their sums are added at the
// end: no barrier stands between a wavefront's loads.  Its steps of 128 go through a ring of its own in LDS, filled by buffer loads that write
// LDS directly, an instruction 8 rows of 128 bytes.  What counts is the lines that are asked for, and a scale alone would be one: they come
// as 16 bytes of every row, 12 steps of E8M0 (from a multiple of four down) or four of fp32 at a time.
template <int MT, int NT, int NW>
struct Few {
    static constexpr int LOADS = 2 * (NT + MT);                            // instructions of a step, scales apart
    static constexpr uint32_t STAGE = (NT + MT) * 2048, SLOT = (MT + 1) * 256;   // a step's values; 16 bytes of scales of every row
    static constexpr int ROOM = (160 * 1024 - 256) / NW;                   // bytes of a wavefront
    static constexpr int SLOTS = ROOM / static_cast<int>(STAGE) == (ROOM - 2 * static_cast<int>(SLOT)) / static_cast<int>(STAGE) ? 2 : 1;
    static constexpr int FIT = (ROOM - SLOTS * static_cast<int>(SLOT)) / static_cast<int>(STAGE), MOST = 1 + 60 / LOADS;   // (the counter of loads in flight ends at 63)
    static constexpr int DEPTH = FIT < MOST ? FIT : MOST, MINE = DEPTH * STAGE + SLOTS * SLOT;
};
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// Loads that the compiler does not know: whoever reads what they bring waits with wait_loads() first.
__device__ __forceinline__ void load_to_lds16(uint32_t lds, uint32_t voff, u32x4 res, uint32_t soff)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(voff), "s"(res), "s"(soff) : "m0", "memory");
}
__device__ __forceinline__ void load_to_lds4(uint32_t lds, uint32_t voff, u32x4 res, uint32_t soff)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(lds), "v"(voff), "s"(res), "s"(soff) : "m0", "memory");
}
#pragma clang diagnostic pop
__device__ __forceinline__ u32x4 resource_of(const void *p, size_t offset, uint32_t bytes)
{
    const uint64_t at = reinterpret_cast<uint64_t>(p) + offset;
    return u32x4{static_cast<uint32_t>(at), static_cast<uint32_t>(at >> 32) & 0xffffu, bytes, 0x00020000u};
}

// 16 columns from column `col` of all outputs on: their output, first column there, and their row of scales.
struct Tile {
    int j, c0, scale_row;
};
__device__ __forceinline__ Tile tile_at(const Fp8Args &a, int col)
{
    Tile t{0, col, 0};
    while (t.c0 >= a.width[t.j]) {
        t.scale_row += (a.width[t.j] + 127) / 128;
        t.c0 -= a.width[t.j++];
    }
    t.scale_row += t.c0 / 128;
    return t;
}

template <int MT, int NT, int NW, bool E8M0, bool EXACT>
__global__ __launch_bounds__(64 * NW) void project_fp8_rows_kernel(Fp8Args a, int N, int tiles_m, int tiles_n, long long per_xcd)
{
    using F = Few<MT, NT, NW>;
    constexpr int DEPTH = F::DEPTH, SB = E8M0 ? 1 : 4;
    __shared__ __attribute__((aligned(1024))) char ring[NW * F::MINE];
    int tm, tn;
    if (!tile_of(tiles_m, tiles_n, tiles_m, per_xcd, tm, tn)) return;
    const int n0 = tn * 16 * NT, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const long long m0 = 16LL * MT * tm;
    const int M = a.M - m0 < 16 * MT ? static_cast<int>(a.M - m0) : 16 * MT;   // rows here
    char *mine = ring + wave * F::MINE;
    const uint32_t mine_lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char *)mine));

    // ---- loading: piece c of a row R sits at position c ^ (R / 2 % 8).  What does not exist - rows, pieces behind K - arrives as zeros. ----
    const int cols = N - n0 < 16 * NT ? N - n0 : 16 * NT;
    const u32x4 res_w = resource_of(a.w, static_cast<size_t>(n0) * a.K, static_cast<uint32_t>(cols) * static_cast<uint32_t>(a.K));
    const u32x4 res_x = resource_of(a.x, static_cast<size_t>(m0) * a.K, static_cast<uint32_t>(M) * static_cast<uint32_t>(a.K));
    const uint32_t scale_bytes = static_cast<uint32_t>(a.pitch) * SB;
    // The 16-column tiles one after the other: where their scales are and where their results go.
    __shared__ u32x4 table[NT];   // (address of the first column in the first row, width)
    Tile t = tile_at(a, n0);
    const int first_scale = t.scale_row;
    uint32_t ws_off = kNowhere;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        if (16 * j >= cols) break;
        if (lane == j) ws_off = static_cast<uint32_t>(t.scale_row - first_scale) * scale_bytes;
        const uint64_t to = reinterpret_cast<uint64_t>(a.out[t.j]) + (static_cast<size_t>(m0) * a.width[t.j] + t.c0) * (EXACT ? 4 : 2);
        if (threadIdx.x == 0) table[j] = u32x4{static_cast<uint32_t>(to), static_cast<uint32_t>(to >> 32), static_cast<uint32_t>(a.width[t.j]), 0u};
        if (16 * (j + 1) >= cols) break;
        t.c0 += 16;
        if (t.c0 >= a.width[t.j]) {
            t.c0 = 0;
            ++t.scale_row;
            ++t.j;
        } else if (t.c0 % 128 == 0) {
            ++t.scale_row;
        }
    }
    const u32x4 res_ws = resource_of(a.ws, static_cast<size_t>(first_scale) * scale_bytes, static_cast<uint32_t>(t.scale_row - first_scale + 1) * scale_bytes);
    const u32x4 res_xs = resource_of(a.xs, static_cast<size_t>(m0) * scale_bytes, static_cast<uint32_t>(M) * scale_bytes);
    constexpr uint32_t SCALES = DEPTH * F::STAGE;
    const uint32_t xs_off = lane * scale_bytes;
    const int piece[2] = {(lane & 7) ^ (lane >> 4), (lane & 7) ^ (4 + (lane >> 4))};   // of instructions with an even and an odd number
    const uint32_t row_off = static_cast<uint32_t>(lane >> 3) * static_cast<uint32_t>(a.K), row_step = 8u * static_cast<uint32_t>(a.K);
    // This wavefront's stretch of K; neighbours in N begin with another one, so that what is asked for at one time spreads over the memory channels.
    const int nk = (a.K + 127) / 128, part = (wave + tn) % NW, first = static_cast<int>(static_cast<long long>(nk) * part / NW);
    const int steps = static_cast<int>(static_cast<long long>(nk) * (part + 1) / NW) - first;
    constexpr int CHUNK = E8M0 ? 12 : 4;   // steps that 16 bytes of scales reach for
    auto issue_scales = [&](int i) {   // of the steps from i on (the waits below count without them, and so wait for a little more)
        const int ks = first + i;
        const uint32_t at = mine_lds + SCALES + i / CHUNK % F::SLOTS * F::SLOT, s0 = E8M0 ? ks & ~3 : 4 * ks;
#pragma unroll
        for (int n = 0; n < (MT + 3) / 4; ++n)
            if (lane < 16 * MT - 64 * n) load_to_lds16(at + n * 1024, xs_off + 64 * n * scale_bytes, res_xs, s0);
        if (lane < NT) load_to_lds16(at + MT * 256, ws_off, res_ws, s0);
    };
    auto issue = [&](int i, int slot) {
        const int ks = first + i, left = a.K - 128 * ks;
        const uint32_t at = mine_lds + slot * F::STAGE, k0 = 128 * ks;
        const bool there[2] = {16 * piece[0] < left, 16 * piece[1] < left};
        if (i % CHUNK == 0 && (F::SLOTS == 2 || i == 0)) issue_scales(i);
#pragma unroll
        for (int n = 0; n < 2 * NT; ++n) load_to_lds16(at + n * 1024, there[n & 1] ? row_off + n * row_step + 16 * piece[n & 1] : kNowhere, res_w, k0);
#pragma unroll
        for (int n = 0; n < 2 * MT; ++n) load_to_lds16(at + (2 * NT + n) * 1024, there[n & 1] ? row_off + n * row_step + 16 * piece[n & 1] : kNowhere, res_x, k0);
    };

    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < DEPTH; ++i)
        if (i < steps) issue(i, i);
    const uint32_t pos = static_cast<uint32_t>(g ^ (r >> 1)) << 4;
    int slot = 0;
    for (int i = 0; i < steps; ++i) {
        if (F::SLOTS == 1 && i > 0 && i % CHUNK == 0) {   // (the scales before have been read)
            issue_scales(i);
            wait_loads<0>();
        } else if (i + DEPTH <= steps) {
            wait_loads<F::LOADS * (DEPTH - 1)>();
        } else {
            wait_loads<0>();
        }
        const char *st = mine + slot * F::STAGE;
        i32x8 w[NT], x[MT];
        uint32_t sw[NT], sx[MT];
        auto fragment = [&](int tile) {
            const char *row = st + tile * 2048 + r * 128;
            return join(*reinterpret_cast<const u32x4 *>(row + pos), *reinterpret_cast<const u32x4 *>(row + (pos ^ 64)));
        };
        const int chunk = i - i % CHUNK, ahead = E8M0 ? first + i - ((first + chunk) & ~3) : i - chunk;
        const char *scales = mine + SCALES + i / CHUNK % F::SLOTS * F::SLOT;
        auto scale_of = [&](int row) -> uint32_t {
            if (E8M0) return reinterpret_cast<const uint8_t *>(scales)[16 * row + ahead];
            return *reinterpret_cast<const uint32_t *>(scales + 16 * row + 4 * ahead);
        };
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            w[j] = fragment(j);
            sw[j] = scale_of(16 * MT + j);
        }
#pragma unroll
        for (int j = 0; j < MT; ++j) {
            x[j] = fragment(NT + j);
            sx[j] = scale_of(16 * j + r);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (i + DEPTH < steps) issue(i + DEPTH, slot);
        slot = slot + 1 == DEPTH ? 0 : slot + 1;
        Operand<EXACT> ow[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) ow[j].set(w[j]);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            Operand<EXACT> ox;
            ox.set(x[m]);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if constexpr (E8M0 && !EXACT) acc[m][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(ow[j].f, ox.f, acc[m][j], 0, 0, 0, sw[j], 0, sx[m]);
                else Factor<E8M0>(sx[m], sw[j]).add(acc[m][j], product(ow[j], ox));
            }
        }
    }

    // ---- the wavefronts' sums, added in the order of K, as many rows of tiles at a time as fit; then whole rows leave.  Lane (r, g) of a tile in
    // column j sits at (r + j) % 16, g: 16 lanes that read a row find their own banks ----
    constexpr int ROWS = static_cast<int>(sizeof(ring)) / (NW * NT * 1024) < MT ? static_cast<int>(sizeof(ring)) / (NW * NT * 1024) : MT;
    static_assert(ROWS >= 1, "the sums of a row of tiles have to fit");
    f32x4 *sums = reinterpret_cast<f32x4 *>(ring);
#pragma unroll
    for (int p = 0; p < MT; p += ROWS) {
        __syncthreads();
#pragma unroll
        for (int i = p; i < p + ROWS && i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) sums[((wave * ROWS + i - p) * NT + j) * 64 + ((r + j) & 15) * 4 + g] = acc[i][j];
        __syncthreads();
        constexpr int G = 4 * NT, AT_ONCE = 64 * NW / G;   // groups of four columns of a row; rows at a time
        const int c = threadIdx.x % G, col = n0 + 4 * c, last = M - 16 * p < 16 * ROWS ? M - 16 * p : 16 * ROWS;
        if (threadIdx.x >= AT_ONCE * G || col >= N) continue;
        const u32x4 to = table[c >> 2];
        char *out = reinterpret_cast<char *>(static_cast<uint64_t>(to[1]) << 32 | to[0]) + 4 * (c & 3) * (EXACT ? 4 : 2);
        const f32x4 bias = a.bias ? *reinterpret_cast<const f32x4 *>(a.bias + col) : f32x4{0.f, 0.f, 0.f, 0.f};
        for (int row = threadIdx.x / G; row < last; row += AT_ONCE) {
            const int at = ((row >> 4) * NT + (c >> 2)) * 64 + ((row + (c >> 2)) & 15) * 4 + (c & 3);
            f32x4 v = sums[(-tn & (NW - 1)) * ROWS * NT * 64 + at];
#pragma unroll
            for (int k = 1; k < NW; ++k) v += sums[((k - tn) & (NW - 1)) * ROWS * NT * 64 + at];
            v += bias;
            char *here = out + static_cast<size_t>(16 * p + row) * to[2] * (EXACT ? 4 : 2);
            if (EXACT) *reinterpret_cast<f32x4 *>(here) = v;
            else *reinterpret_cast<u32x2 *>(here) = pack4(v);
        }
    }
}

template <int MT, int NT>
void launch_few(ProfileScope &ps, const Fp8Args &a, int N, bool e8m0, hipStream_t stream)
{
    constexpr int NW = Few<MT, NT, 8>::DEPTH >= 1 ? 8 : 4;
    const int tiles_m = static_cast<int>((a.M + 16 * MT - 1) / (16 * MT)), tiles_n = (N + 16 * NT - 1) / (16 * NT);
    const long long per_xcd = ((static_cast<long long>(tiles_m) * tiles_n + 7) / 8 + tiles_m - 1) / tiles_m * tiles_m;   // whole columns to an XCD
    const dim3 grid(static_cast<unsigned>(8 * per_xcd));
    if (e8m0 && a.out_f32) DSLA_LAUNCH(ps, (project_fp8_rows_kernel<MT, NT, NW, true, true>), grid, dim3(64 * NW), 0, stream, a, N, tiles_m, tiles_n, per_xcd);
    else if (e8m0) DSLA_LAUNCH(ps, (project_fp8_rows_kernel<MT, NT, NW, true, false>), grid, dim3(64 * NW), 0, stream, a, N, tiles_m, tiles_n, per_xcd);
    else if (a.out_f32) DSLA_LAUNCH(ps, (project_fp8_rows_kernel<MT, NT, NW, false, true>), grid, dim3(64 * NW), 0, stream, a, N, tiles_m, tiles_n, per_xcd);
    else DSLA_LAUNCH(ps, (project_fp8_rows_kernel<MT, NT, NW, false, false>), grid, dim3(64 * NW), 0, stream, a, N, tiles_m, tiles_n, per_xcd);
}
template <int MT>
void launch_few_n(ProfileScope &ps, const Fp8Args &a, int N, int nt, bool e8m0, hipStream_t stream)
{
    if (nt <= 1) launch_few<MT, 1>(ps, a, N, e8m0, stream);
    else if (nt == 2) launch_few<MT, 2>(ps, a, N, e8m0, stream);
    else if (nt == 3) launch_few<MT, 3>(ps, a, N, e8m0, stream);
    else if (nt == 4) launch_few<MT, 4>(ps, a, N, e8m0, stream);
    else launch_few<MT, 5>(ps, a, N, e8m0, stream);
}
void launch_few_m(ProfileScope &ps, const Fp8Args &a, int N, int mt, int nt, bool e8m0, hipStream_t stream)
{
    if (mt <= 1) launch_few_n<1>(ps, a, N, nt, e8m0, stream);
    else if (mt == 2) launch_few_n<2>(ps, a, N, nt, e8m0, stream);
    else if (mt == 3) launch_few_n<3>(ps, a, N, nt, e8m0, stream);
    else if (mt == 4) launch_few_n<4>(ps, a, N, nt, e8m0, stream);
    else launch_few_n<5>(ps, a, N, nt, e8m0, stream);
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
    if (M <= 64) {
        const int nt = (N + 16 * 256 - 1) / (16 * 256);
        launch_few_m(ps, a, N, static_cast<int>((M + 15) / 16), nt, e8m0, stream);
        return hipGetLastError();
    }
    if (!exact && M > 512) {
        const int tiles_m = static_cast<int>((M + 255) / 256), tiles_n = (blocks + 1) / 2;
        const long long per_xcd = (static_cast<long long>(tiles_m) * tiles_n + 7) / 8;
        const dim3 grid(static_cast<unsigned>(8 * per_xcd));
        const int group = tiles_m <= 5 ? tiles_m : 4;
        if (e8m0) DSLA_LAUNCH(ps, project_fp8_tile_kernel<true>, grid, dim3(256), 0, stream, a, tiles_m, tiles_n, blocks, group, per_xcd);
        else DSLA_LAUNCH(ps, project_fp8_tile_kernel<false>, grid, dim3(512), 0, stream, a, tiles_m, tiles_n, blocks, group, per_xcd);
        return hipGetLastError();
    }
    const unsigned tiles_m = static_cast<unsigned>((M + 127) / 128);
    const dim3 grid(tiles_m * static_cast<unsigned>(blocks));
    if (e8m0 && exact) DSLA_LAUNCH(ps, (project_fp8_kernel<true, true>), grid, dim3(256), 0, stream, a, tiles_m);
    else if (e8m0) DSLA_LAUNCH(ps, (project_fp8_kernel<true, false>), grid, dim3(256), 0, stream, a, tiles_m);
    else if (exact) DSLA_LAUNCH(ps, (project_fp8_kernel<false, true>), grid, dim3(256), 0, stream, a, tiles_m);
    else DSLA_LAUNCH(ps, (project_fp8_kernel<false, false>), grid, dim3(256), 0, stream, a, tiles_m);
    return hipGetLastError();
}

}  // namespace dsla
