// Tiles of K and V rows (bf16) in LDS, as the attention kernels read them.
#pragma once

#include "civic_internal.h"

namespace civic {

typedef short s16x4 __attribute__((ext_vector_type(4)));

// LDS transpose read (gfx950): the 16 lanes of a group each name 4 consecutive bf16 of a 4 x 16 block
// (lane i -> row i/4, columns 4(i%4)..+3); lane i receives column i of the block, rows 0..3.
__device__ __forceinline__ s16x4 lds_read_tr16(const __bf16* p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (s16x4 __attribute__((address_space(3)))*)(const_cast<__bf16*>(p)));
}

// K/V tiles live in LDS with a fixed row pitch of PITCH 16-byte chunks and an XOR swizzle of the chunk
// index by a function of the row, so that no padding is needed (global -> LDS loads write 64
// consecutive 16-byte slots per wavefront instruction) and both the 128-bit K reads (16 lanes = 16
// consecutive rows, same logical chunk) and the transposing 64-bit V reads (32 lanes = 4 consecutive
// rows x 4 chunks) fall on distinct banks.
template <int PITCH>
__device__ __forceinline__ int swz(int row)
{
    if constexpr (PITCH == 16 || PITCH == 32) return ((row & 3) << 2) | ((row >> 2) & 3);
    else if constexpr (PITCH == 12) return (row >> 2) & 3;   // (rows 12 chunks apart start in 4 different quarters of the 16 by themselves)
    else return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}

typedef short s16x8 __attribute__((ext_vector_type(8)));

}  // namespace civic
