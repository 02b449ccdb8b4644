// What stands around the layer (include/dsla.h): the norms, gate and residual scale of a block's border, the norm and gate of the
// read-out's heads, and values to e4m3 with block scales.  All of them are bound by memory: every value is read once, kept in
// registers and written once, 8 values of a lane at a time; sums and largest magnitudes go through the lanes.  A block of 128
// columns is 16 lanes of 8, one row of the cross-lane operations.  A copy with the same non-temporal hints reaches 6.1 to 6.3 TB/s:
//   border, 16384 rows of 4096, bf16, both norms, gate, e4m3 out   112 to 114 us  5.3 to 5.4 TB/s (vector instructions issued 86 % of the time; two sums
//                                                                   across the workgroup one after the other); without norm of y, gate and 8 bits 6.0
//   heads, 16384 rows of 32 of 128, bf16, gate, e4m3 out            58.6 to 60.8 us  5.6 to 5.8 TB/s
//   quantize, 20480 x 4096 bf16, blocks of 128 x 128                48.8 us  5.2 TB/s (256 bytes of a row at a time)
#include "fp8_common.h"

namespace dsla {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void load8(const bf16_t *p, float (&f)[8])
{
    const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const float *p, float (&f)[8])
{
    const f32x4 a = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(p)), b = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(p + 4));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[i] = a[i];
        f[4 + i] = b[i];
    }
}
__device__ __forceinline__ void load8_kept(const float *p, float (&f)[8])   // weights: every row reads them again
{
    const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[i] = a[i];
        f[4 + i] = b[i];
    }
}
__device__ __forceinline__ void store8(bf16_t *p, const float (&f)[8])
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = f32_to_bf16_bits(f[2 * i]) | static_cast<uint32_t>(f32_to_bf16_bits(f[2 * i + 1])) << 16;
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4 *>(p));
}
__device__ __forceinline__ void store8(float *p, const float (&f)[8])
{
    __builtin_nontemporal_store(f32x4{f[0], f[1], f[2], f[3]}, reinterpret_cast<f32x4 *>(p));
    __builtin_nontemporal_store(f32x4{f[4], f[5], f[6], f[7]}, reinterpret_cast<f32x4 *>(p + 4));
}

// The value of another lane of the 16: N places round.
template <int N>
__device__ __forceinline__ float row_rotate(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + N, 0xf, 0xf, true));
}
__device__ __forceinline__ float max16(float x)
{
    x = fmaxf(x, row_rotate<8>(x));
    x = fmaxf(x, row_rotate<4>(x));
    x = fmaxf(x, row_rotate<2>(x));
    return fmaxf(x, row_rotate<1>(x));
}
__device__ __forceinline__ float sum16(float x)
{
    x += row_rotate<8>(x);
    x += row_rotate<4>(x);
    x += row_rotate<2>(x);
    return x + row_rotate<1>(x);
}

// Sum over the T threads of a workgroup, over a wavefront (T = 64) or over 16 lanes.
template <int T>
__device__ __forceinline__ float sum_all(float x, float *s)
{
    x = sum16(x);
    if (T == 16) return x;
    x += __shfl_xor(x, 16);
    x += __shfl_xor(x, 32);
    if (T == 64) return x;
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < T / 64; ++i) t += s[i];
    return t;
}

// act(z) as a power of two.  exact (results in fp32), by e^-|z|, so that a large gate does not overflow: to 6 ulps, the exponent carries the rounding of
// |z| log2 e along, its whole part goes around the instruction, which has no results below 2^-126, and the inverse takes a step of Newton's.
// Else by 2^-32 e^-z, which overflows where the gate is below all numbers (the instructions take and give none below 2^-126): to 2^-18, by 15 issue slots
// instead of 26; the kernels issue vector instructions all the time.  The exponent is rounded once, below 128 by 2^-18, 44 U of the power; what the fp32 log2 e
// lacks, up to 20 U at z = -87, a factor puts back (for z > 0 it would be of no weight, and is 1).
__device__ __forceinline__ float activated(float z, int act, bool exact)
{
    if (act == DSLA_ACT_NONE) return z;
    constexpr float kLog2e = 1.44269502f, kLog2eRest = 1.92596303e-8f, kLn2 = 0.693147182f;
    if (exact) {
        const float a = fabsf(z) > 200.f ? -200.f : -fabsf(z);   // (e^-200 is 0; NaN stays)
        const float p = a * kLog2e, n = rintf(p), rest = fmaf(a, kLog2eRest, fmaf(a, kLog2e, -p));
        const float t = ldexpf(__builtin_amdgcn_exp2f((p - n) + rest), static_cast<int>(n));
        const float d = 1.f + t, y = __builtin_amdgcn_rcpf(d), inverse = fmaf(y, fmaf(-d, y, 1.f), y);
        const float top = z < 0.f ? t : 1.f;
        return (act == DSLA_ACT_SIGMOID ? top : z * top) * inverse;
    }
    const float t = __builtin_amdgcn_exp2f(fmaf(-z, kLog2e, -32.f)), back = __builtin_amdgcn_fmed3f(fmaf(z, kLog2eRest * kLn2, 1.f), 0.f, 1.f);
    const float sigmoid = 0x1p-32f * __builtin_amdgcn_rcpf(t + 0x1p-32f) * back;
    return act == DSLA_ACT_SIGMOID ? sigmoid : z * sigmoid;
}

// 1 / sqrt(v) to an ulp: the instruction and a step of Newton's; far from 1 (no square of a number, or an infinite one) the library's.
__device__ __forceinline__ float inverse_root(float v)
{
    if (!(v > 0x1p-100f && v < 0x1p127f)) return 1.f / sqrtf(v);
    const float y = __builtin_amdgcn_rsqf(v);
    return fmaf(0.5f * y, fmaf(-v * y, y, 1.f), y);
}

// 8 values of a lane to where they go: as they are, or as e4m3 with the scale of the block that the lane's row of 16 holds (lanes without
// values take part with zeros).
struct Result {
    void *p, *scale;
    int dtype, scale_type, pitch;
};
template <bool E8M0>
__device__ __forceinline__ void store_block(const Result &o, const float (&f)[8], bool valid, size_t at, long long row, int block)
{
    const BlockScale<E8M0> s(max16(largest(f)));
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = f[i] * s.inverse;
    if (valid) __builtin_nontemporal_store(u32x2{e4m3x4(v[0], v[1], v[2], v[3]), e4m3x4(v[4], v[5], v[6], v[7])},
                                           reinterpret_cast<u32x2 *>(static_cast<uint8_t *>(o.p) + at));
    if (valid && threadIdx.x % 16 == 0) s.store(o.scale, static_cast<size_t>(row) * o.pitch + block);
}
__device__ __forceinline__ void store_result(const Result &o, const float (&f)[8], bool valid, size_t at, long long row, int block)
{
    if (o.dtype == DSLA_E4M3) {
        if (o.scale_type == DSLA_SCALE_E8M0) store_block<true>(o, f, valid, at, row, block);
        else store_block<false>(o, f, valid, at, row, block);
    } else if (valid) {
        if (o.dtype == DSLA_BF16) store8(static_cast<bf16_t *>(o.p) + at, f);
        else store8(static_cast<float *>(o.p) + at, f);
    }
}

// ---------------------------------------------------------------------------------------------------------------
// A block's border
// ---------------------------------------------------------------------------------------------------------------
struct BorderArgs {
    const void *x, *y, *gate;
    void *x_out;
    const float *post_weight, *pre_weight;
    Result h;
    long long rows;
    int D, act;
    float eps, residual_scale;
    bool exact;   // a result in fp32
};

// T threads to a row, NV times 8 values to a thread: value 8 (T c + t) .. + 7 of the row for c < NV.  T = 64 and 16: a wavefront, or 16 lanes, to a
// row, and 256 threads to a workgroup.
template <int T, int NV, class TX, class TY>
__global__ __launch_bounds__(T < 256 ? 256 : T) void residual_norm_kernel(BorderArgs a)
{
    constexpr int ROWS = T < 256 ? 256 / T : 1;
    __shared__ float s_post[(T + 63) / 64], s_pre[(T + 63) / 64];
    const int t = threadIdx.x % T;
    const long long row = static_cast<long long>(workgroup_index()) * ROWS + threadIdx.x / T;
    if (row >= a.rows) return;   // (rows of one workgroup share nothing)
    const size_t base = static_cast<size_t>(row) * a.D;
    float r[NV][8], u[NV][8], g[NV][8];
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int col = 8 * (T * c + t);
#pragma unroll
        for (int i = 0; i < 8; ++i) r[c][i] = u[c][i] = g[c][i] = 0.f;
        if (col >= a.D) continue;
        load8(static_cast<const TX *>(a.x) + base + col, r[c]);
        if (a.y) load8(static_cast<const TY *>(a.y) + base + col, u[c]);
        if (a.gate) load8(static_cast<const TY *>(a.gate) + base + col, g[c]);
    }
    float factor = a.residual_scale;
    if (a.post_weight) {
        float q = 0.f;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) q += u[c][i] * u[c][i];
        q = sum_all<T>(q, s_post);
        const float inv = inverse_root(q / a.D + a.eps);
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = 8 * (T * c + t);
            if (col >= a.D) continue;
            float w[8];
            load8_kept(a.post_weight + col, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) u[c][i] *= inv * w[i];
        }
    }
    float q = 0.f;
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int col = 8 * (T * c + t);
        if (col >= a.D) continue;
        if (a.y) {
#pragma unroll
            for (int i = 0; i < 8; ++i) r[c][i] += factor * (a.gate ? u[c][i] * activated(g[c][i], a.act, a.exact) : u[c][i]);
        }
        if (a.x_out) store8(static_cast<TX *>(a.x_out) + base + col, r[c]);
#pragma unroll
        for (int i = 0; i < 8; ++i) q += r[c][i] * r[c][i];
    }
    if (!a.h.p) return;
    float inv = 1.f;
    if (a.pre_weight) {
        q = sum_all<T>(q, s_pre);
        inv = inverse_root(q / a.D + a.eps);
    }
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int col = 8 * (T * c + t);
        const bool valid = col < a.D;
        if (valid && a.pre_weight) {
            float w[8];
            load8_kept(a.pre_weight + col, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) r[c][i] *= inv * w[i];
        }
        store_result(a.h, r[c], valid, base + col, row, col >> 7);
    }
}

template <int T, int NV>
void launch_border(ProfileScope &ps, const BorderArgs &a, bool x32, bool y32, hipStream_t stream)
{
    constexpr int ROWS = T < 256 ? 256 / T : 1;
    const dim3 block(T < 256 ? 256 : T), grid = grid_of((a.rows + ROWS - 1) / ROWS, block.x);
    if (x32 && y32) DSLA_LAUNCH(ps, (residual_norm_kernel<T, NV, float, float>), grid, block, 0, stream, a);
    else if (x32) DSLA_LAUNCH(ps, (residual_norm_kernel<T, NV, float, bf16_t>), grid, block, 0, stream, a);
    else if (y32) DSLA_LAUNCH(ps, (residual_norm_kernel<T, NV, bf16_t, float>), grid, block, 0, stream, a);
    else DSLA_LAUNCH(ps, (residual_norm_kernel<T, NV, bf16_t, bf16_t>), grid, block, 0, stream, a);
}

// ---------------------------------------------------------------------------------------------------------------
// Heads, and plain rows
// ---------------------------------------------------------------------------------------------------------------
struct RowsArgs {
    const void *x, *gate;
    const float *weight;   // [d], null: no norm
    Result o;
    uint32_t blocks;       // rows * blocks of a row
    int cols, per_row, act;
    float eps;
    Divisor by_row;
};

// 16 lanes to a block of 128 columns of a row - one head of 128, two of 64, or 128 plain values - and NB blocks to 16 lanes, all of them
// asked for before the first is used.
template <int D, int NB, class TIO>
__global__ __launch_bounds__(256) void rows_kernel(RowsArgs a)
{
    const int l = threadIdx.x & 15;
    float f[NB][8], g[NB][8], w[8];
    uint32_t row[NB];
    int block[NB];
    bool valid[NB];
#pragma unroll
    for (int u = 0; u < NB; ++u) {
        const uint32_t n = (workgroup_index() * NB + u) * 16u + (threadIdx.x >> 4);
        const bool there = n < a.blocks;
        row[u] = a.by_row.quotient(there ? n : 0u);
        block[u] = there ? static_cast<int>(n - row[u] * a.per_row) : 0;
        valid[u] = there && 128 * block[u] + 8 * l < a.cols;
        const size_t at = static_cast<size_t>(row[u]) * a.cols + 128 * block[u] + 8 * l;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[u][i] = g[u][i] = 0.f;
        if (valid[u]) {
            load8(static_cast<const TIO *>(a.x) + at, f[u]);
            if (D && a.gate) load8(static_cast<const TIO *>(a.gate) + at, g[u]);
        }
    }
    if (D && a.weight) load8_kept(a.weight + (8 * l) % (D ? D : 8), w);
#pragma unroll
    for (int u = 0; u < NB; ++u) {
        if (D && a.weight) {
            float q = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) q += f[u][i] * f[u][i];
            if (D == 128) {
                q = sum16(q);
            } else {   // 8 lanes: l ^ 4, l ^ 2, l ^ 1
                q += __shfl_xor(q, 4);
                q += __shfl_xor(q, 2);
                q += __shfl_xor(q, 1);
            }
            const float inv = inverse_root(q * (1.f / (D ? D : 1)) + a.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[u][i] *= inv * w[i];
        }
        if (D && a.gate) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[u][i] *= activated(g[u][i], a.act, a.o.dtype == DSLA_F32);
        }
        store_result(a.o, f[u], valid[u], static_cast<size_t>(row[u]) * a.cols + 128 * block[u] + 8 * l, row[u], block[u]);
    }
}

template <int D, int NB>
void launch_rows(ProfileScope &ps, const RowsArgs &a, bool f32, hipStream_t stream)
{
    const dim3 grid = grid_of((a.blocks + 16u * NB - 1) / (16u * NB), 256);
    if (f32) DSLA_LAUNCH(ps, (rows_kernel<D, NB, float>), grid, dim3(256), 0, stream, a);
    else DSLA_LAUNCH(ps, (rows_kernel<D, NB, bf16_t>), grid, dim3(256), 0, stream, a);
}
// Several blocks to 16 lanes where every compute unit has eight workgroups of them (heads, 16384 rows of 32: one 69 us, two 67.8, four 77.9).
template <int D>
void launch_rows_of(ProfileScope &ps, const RowsArgs &a, bool f32, hipStream_t stream)
{
    constexpr int NB = D ? 2 : 4;
    if (a.blocks >= 8u * 256u * 16u * NB) launch_rows<D, NB>(ps, a, f32, stream);
    else launch_rows<D, 1>(ps, a, f32, stream);
}

// ---------------------------------------------------------------------------------------------------------------
// Blocks of 128 x 128
// ---------------------------------------------------------------------------------------------------------------
struct SquareArgs {
    const void *x;
    uint8_t *q;
    void *scale;
    long long rows;
    int cols, pitch, per_row;
};

template <class TIO, bool E8M0>
__global__ __launch_bounds__(256) void square_kernel(SquareArgs a)
{
    __shared__ float s_max[16];
    const int l = threadIdx.x & 15, r0 = threadIdx.x >> 4;
    const uint32_t n = workgroup_index(), brow = n / a.per_row;
    if (128LL * brow >= a.rows) return;
    const int bcol = static_cast<int>(n - brow * a.per_row), col = 128 * bcol + 8 * l;
    float f[8][8], m = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const long long row = 128LL * brow + 16 * c + r0;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[c][i] = 0.f;
        if (row < a.rows && col < a.cols) load8(static_cast<const TIO *>(a.x) + static_cast<size_t>(row) * a.cols + col, f[c]);
    }
#pragma unroll
    for (int c = 0; c < 8; ++c) m = fmaxf(m, largest(f[c]));
    m = max16(m);
    if (l == 0) s_max[r0] = m;
    __syncthreads();
    const BlockScale<E8M0> s(max16(s_max[l]));
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const long long row = 128LL * brow + 16 * c + r0;
        if (row >= a.rows || col >= a.cols) continue;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = f[c][i] * s.inverse;
        __builtin_nontemporal_store(u32x2{e4m3x4(v[0], v[1], v[2], v[3]), e4m3x4(v[4], v[5], v[6], v[7])},
                                    reinterpret_cast<u32x2 *>(a.q + static_cast<size_t>(row) * a.cols + col));
    }
    if (threadIdx.x == 0) s.store(a.scale, static_cast<size_t>(brow) * a.pitch + bcol);
}

Result result_of(void *p, void *scale, int dtype, int scale_type, int cols) { return Result{p, scale, dtype, scale_type, scale_pitch(cols)}; }
}  // namespace

hipError_t launch_residual_norm(const dsla_norm &n, int64_t rows, const void *x, const void *y, const void *gate, void *x_out, void *h, void *h_scale,
                                hipStream_t stream)
{
    BorderArgs a{x, y, gate, x_out, n.post_weight, n.pre_weight, result_of(h, h_scale, n.h_dtype, n.scale_type, n.D), rows, n.D, n.gate_act, n.eps, n.residual_scale,
                 (x_out && n.x_dtype == DSLA_F32) || (h && n.h_dtype == DSLA_F32)};
    const bool x32 = n.x_dtype == DSLA_F32, y32 = n.y_dtype == DSLA_F32;
    ProfileScope ps(DSLA_KERNEL_RESIDUAL_NORM, stream);
    // 8 values a lane above 1024 and up to 8192 columns: more rows' loads are in flight at once than with more of them.  Up to 4096 columns 256 lanes of 16
    // values / 512 of 8, above 256 of 32 / 1024 of 8 (us), without norm of y, gate and 8 bits: 8192 rows of 4096 46.0 / 44.6 (128 of 32 slower than both),
    // 256 of 4096 4.08 / 3.85, 16384 of 2560 57.4 / 55.8, 16384 of 2064 51.0 / 51.5, 8192 of 5120 62.0 / 60.4, 4096 of 7168 43.8 / 41.5, 4096 of 8192
    // 48.9 / 46.2.  With all of it the lanes that have no values and the larger barrier weigh more: 16384 of 4096 110.2 / 112.4, of 2560 81.8 / 85.8, of
    // 2064 77.5 / 83.8, but 8192 of 5120 96.6 / 83.1, of 8192 134.8 / 114.5.
    if (n.D <= 128) launch_border<16, 1>(ps, a, x32, y32, stream);
    else if (n.D <= 512) launch_border<64, 1>(ps, a, x32, y32, stream);
    else if (n.D <= 1024) launch_border<64, 2>(ps, a, x32, y32, stream);
    else if (n.D <= 2048) launch_border<256, 1>(ps, a, x32, y32, stream);
    else if (n.D <= 4096) launch_border<512, 1>(ps, a, x32, y32, stream);
    else if (n.D <= 8192) launch_border<1024, 1>(ps, a, x32, y32, stream);
    else if (n.D <= 16384) launch_border<1024, 2>(ps, a, x32, y32, stream);
    else launch_border<1024, 4>(ps, a, x32, y32, stream);
    return hipGetLastError();
}

hipError_t launch_head_norm(const dsla_heads &n, int64_t rows, const void *o, const void *gate, void *out, void *out_scale, hipStream_t stream)
{
    const int cols = n.H * n.d, per_row = (cols + 127) / 128;
    RowsArgs a{o, gate, n.weight, result_of(out, out_scale, n.out_dtype, n.scale_type, cols), static_cast<uint32_t>(rows * per_row), cols, per_row, n.gate_act, n.eps, Divisor(per_row)};
    ProfileScope ps(DSLA_KERNEL_HEAD_NORM, stream);
    if (n.d == 128) launch_rows_of<128>(ps, a, n.io_dtype == DSLA_F32, stream);
    else launch_rows_of<64>(ps, a, n.io_dtype == DSLA_F32, stream);
    return hipGetLastError();
}

hipError_t launch_quantize(int64_t rows, int cols, int in_dtype, int block_rows, int scale_type, const void *x, void *q, void *scale, hipStream_t stream)
{
    const int per_row = (cols + 127) / 128;
    ProfileScope ps(DSLA_KERNEL_QUANTIZE, stream);
    if (block_rows == 1) {
        RowsArgs a{x, nullptr, nullptr, result_of(q, scale, DSLA_E4M3, scale_type, cols), static_cast<uint32_t>(rows * per_row), cols, per_row, DSLA_ACT_NONE, 0.f, Divisor(per_row)};
        launch_rows_of<0>(ps, a, in_dtype == DSLA_F32, stream);
    } else {
        const SquareArgs a{x, static_cast<uint8_t *>(q), scale, rows, cols, scale_pitch(cols), per_row};
        const dim3 grid = grid_of((rows + 127) / 128 * per_row, 256);
        if (in_dtype == DSLA_F32 && scale_type == DSLA_SCALE_E8M0) DSLA_LAUNCH(ps, (square_kernel<float, true>), grid, dim3(256), 0, stream, a);
        else if (in_dtype == DSLA_F32) DSLA_LAUNCH(ps, (square_kernel<float, false>), grid, dim3(256), 0, stream, a);
        else if (scale_type == DSLA_SCALE_E8M0) DSLA_LAUNCH(ps, (square_kernel<bf16_t, true>), grid, dim3(256), 0, stream, a);
        else DSLA_LAUNCH(ps, (square_kernel<bf16_t, false>), grid, dim3(256), 0, stream, a);
    }
    return hipGetLastError();
}

}  // namespace dsla
