// What the attention kernels share that stream keys and values through LDS: the image of a block there, the transposing read of
// values, and the barrier behind the loads that go from memory straight to LDS.
#pragma once
#include "dsla_internal.h"

namespace dsla {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kKeys = 64;            // keys per block: two score tiles of 32

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    f32x2 x = {a, b};
    bf16x2 y = __builtin_convertvector(x, bf16x2);
    return __builtin_bit_cast(uint32_t, y);
}
// LDS image of a block of 64 keys (and of its values): rows of d elements WITHOUT padding, because the block is
// written by loads that go from memory straight to LDS (a wavefront's 64 lanes fill 1 KB of consecutive LDS).  Bank
// conflicts are avoided by WHERE in its row a 16-byte piece is put:
// - keys: piece c of row r sits at piece position c ^ swz_k(r); the 16 rows that 16 lanes read at one time at the
//   same logical piece then fall into 16 different groups of four banks;
// - values: the 64-byte quarter q of row r sits at quarter position q ^ swz_v(r); a pass of the transposing read
//   takes one quarter from each of 4 consecutive rows, which then fall into the four quarters of the banks.
// The lane that fills LDS slot (row, position) simply fetches the piece that belongs there.
template <int D>
struct AttnTiles {
    static constexpr int RB = D * 2;                    // bytes per row
    static constexpr int NC = D / 8;                    // 16-byte pieces per row (16 or 8)
    static constexpr int NQ = RB / 64;                  // 64-byte quarters per row (4 or 2)
    static constexpr uint32_t K_BYTES = kKeys * RB;
    static constexpr uint32_t V_BYTES = kKeys * RB;
    static constexpr uint32_t BUF_BYTES = K_BYTES + V_BYTES;
    static __device__ __forceinline__ uint32_t swz_k(uint32_t row) { return NC == 16 ? (row & 15u) : ((row >> 1) & 7u); }
    static __device__ __forceinline__ uint32_t swz_v(uint32_t row) { return NQ == 4 ? (row & 3u) : ((row >> 1) & 1u); }
};

// Fragment of V^T for a block of 16 keys from V rows in LDS, by two transposing 8-byte reads: the 16 lanes of a group
// address 4 keys x 4 pieces of 4 columns and each receives 4 keys of ONE column.  With `a` as computed in the kernel
// lane l ends up with column (tile) + l % 32 and keys 4 g + 0..3 (from a) and 8 + 4 g + 0..3 (from a + 8 rows): the
// order in which the result registers of a score tile hold the keys.
__device__ __forceinline__ bf16x8 load_vt_frag(const char *a, uint32_t step)
{
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef s16x4 __attribute__((address_space(3))) *lds_ptr;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(a));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(a + step));
    const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
    return __builtin_bit_cast(bf16x8, u32x4{l2[0], l2[1], h2[0], h2[1]});
}

__device__ __forceinline__ void loads_landed_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

}  // namespace
}  // namespace dsla
