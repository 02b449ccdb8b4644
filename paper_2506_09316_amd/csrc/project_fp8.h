// What the products of e4m3 operands share (project_fp8.hip: large tiles; project_fp8_rows.h: few rows, or results in fp32).
#pragma once
#include "fp8_common.h"
#include "project_common.h"

namespace dsla {

struct Fp8Args {
    const uint8_t *x, *w;
    const void *xs, *ws;
    const float *bias;
    void *out[DSLA_MAX_PROJECTIONS];
    int width[DSLA_MAX_PROJECTIONS];
    long long M;
    int K, pitch, out_f32;
};

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

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
constexpr int kOne = 127;   // E8M0
// An offset past the end of every buffer here: zeros.  (The range of a buffer is checked dword by dword, with both offsets.)
constexpr uint32_t kNowhere = 0x80000000u;

__device__ __forceinline__ i32x8 join(u32x4 a, u32x4 b)
{
    return i32x8{static_cast<int>(a[0]), static_cast<int>(a[1]), static_cast<int>(a[2]), static_cast<int>(a[3]),
                 static_cast<int>(b[0]), static_cast<int>(b[1]), static_cast<int>(b[2]), static_cast<int>(b[3])};
}

// tile_of() of a launch that may be filled up (grid_of()).
__device__ __forceinline__ bool tile_here(int tiles_m, int tiles_n, int GM, long long per_xcd, int &tm, int &tn)
{
    const uint32_t workgroup = workgroup_index();
    return workgroup / 8 < per_xcd && tile_of(workgroup, tiles_m, tiles_n, GM, per_xcd, tm, tn);
}

}  // namespace

// Tiles of an XCD: whole columns, whose rows of W then come from memory once, where that takes no further round over its 32 compute units (a
// column alone, such as 2000 rows of 128 columns, would be on one XCD: 19 us instead of 6).
inline long long fp8_rows_per_xcd(long long tiles_m, long long tiles_n)
{
    const long long even = (tiles_m * tiles_n + 7) / 8, whole = (even + tiles_m - 1) / tiles_m * tiles_m;
    return (whole + 31) / 32 == (even + 31) / 32 ? whole : even;
}

// Launches the kernel for few rows in tiles of 16 mt x 16 nt; false: not built for such tiles.
bool launch_fp8_rows(ProfileScope &ps, const Fp8Args &a, int N, int mt, int nt, bool e8m0, hipStream_t stream);
bool launch_fp8_rows_exact(ProfileScope &ps, const Fp8Args &a, int N, int mt, int nt, bool e8m0, hipStream_t stream);

}  // namespace dsla
