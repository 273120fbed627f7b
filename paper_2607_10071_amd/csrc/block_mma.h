// Matrix products of 32 x 32 blocks over a granule of 16 bytes from each operand's row.
#pragma once

#include "block_common.h"

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int DT>
__device__ __forceinline__ void mma(f32x16 &c, const u32x4 &a, const u32x4 &b)
{
    if constexpr (DT == FLASHBEV_BF16) {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                    __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else if constexpr (DT == FLASHBEV_F16) {
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                   __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    } else {
        const f32x4 fa = __builtin_bit_cast(f32x4, a), fb = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[q], fb[q], c, 0, 0, 0);
    }
}

// The MFMA leaves a lane with four groups of four columns of a row in each block
// (group k: columns 8 k + 4 (lane / 32) ..); swapping halves of the wavefront
// between groups 2 q and 2 q + 1 makes them columns 16 q + 8 (lane / 32) .. + 7.
__device__ __forceinline__ void columns_of(const f32x16 &acc, int q, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float x = acc[8 * q + i], y = acc[8 * q + 4 + i];
        const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x),
                                                        __builtin_bit_cast(unsigned, y), false, false);
        const unsigned a = r[0], b = r[1];
        v[i] = __builtin_bit_cast(float, a);
        v[4 + i] = __builtin_bit_cast(float, b);
    }
}

}  // namespace
