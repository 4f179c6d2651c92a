// Tiles of 32 x 32 scores whose keys and values lie in LDS for all waves: where pieces lie, products, transposing reads.
#pragma once
#include "attention_common.h"

namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;

// A row's weights are held relative to a reference: kWeightsAt powers of two below the largest score so far when it is set, and moved
// when a score passes that one by kWeightsUpTo.  fp16 has no normal values below 2^-14 and none below 2^-24: with weights of up to 2^15
// those that are 2^21 times smaller than the row's largest keep their bits, and down to 2^-32 of it they count (relative to the
// largest itself 60000 weights of 2^-25.5 were lost beside it: off by 0.13 %, five half steps).  The factor cancels in the division.
template <int DT>
constexpr float kWeightsAt = DT == kF16 ? 7.f : 0.f;
constexpr float kWeightsUpTo = 8.f;

// Place of 16-byte piece c of row r in LDS (bytes), rows of `pieces` pieces.
template <int PIECES>
__device__ __forceinline__ int tile_place(int r, int c) {
    const int f = PIECES == 8 ? (r >> 1 & 1) << 2 | (r >> 2 & 3) : (r & 3) << 2 | (r >> 2 & 3);
    return (r * PIECES + (c ^ f)) * 16;
}

template <int DT>
__device__ __forceinline__ f32x16_t mfma_32(uint4 a, uint4 b, f32x16_t acc) {
    if (DT == kF16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), acc, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
}
// Four rows of LDS, 16 columns: lane l of sixteen gets column l of the rows whose pieces the lanes point at (lane l: row
// l / 4, columns 4 (l % 4) on).
__device__ __forceinline__ uint2 lds_transposed(const char* at) {
    const s16x4_t r = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)const_cast<char*>(at));
    return __builtin_bit_cast(uint2, r);
}

// acc plus two values.
template <int DT>
__device__ __forceinline__ float add_pair(unsigned w, float acc) {
    if (DT == kF16) return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2_t, w), __builtin_bit_cast(f16x2_t, 0x3c003c00u), acc, false);
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w), __builtin_bit_cast(bf16x2_t, 0x3f803f80u), acc, false);
}
}  // namespace
