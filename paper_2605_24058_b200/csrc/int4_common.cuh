// The 4-bit carrier's words as pairs of 16-bit numbers (int4.cu, int4_few.cu).
#pragma once

#include "block_common.cuh"

namespace lordba {

// A number u = 0 ... 15 put into the low bits of this pattern is the float 128 + u (bfloat16) or 1024 + u (float16), exactly;
// less the same pattern with the zero point z in it, it is u - z, exactly.  So a pair costs a shift, one three-input logic
// operation and one subtraction of two halves.
template <typename E> struct Int4Pair;
template <> struct Int4Pair<__nv_bfloat16> {
    using Two = __nv_bfloat162;
    static constexpr uint32_t kOnes = 0x43004300u;
};
template <> struct Int4Pair<__half> {
    using Two = __half2;
    static constexpr uint32_t kOnes = 0x64006400u;
};

// The pattern of a zero point, in both halves.
template <typename E>
__device__ __forceinline__ uint32_t int4_zero(uint32_t z) { return Int4Pair<E>::kOnes | z | z << 16; }

// Columns 2 i and 2 i + 1 of a word, less the zero point.
template <typename E>
__device__ __forceinline__ uint32_t int4_pair(uint32_t word, int i, uint32_t zero)
{
    using Two = typename Int4Pair<E>::Two;
    const uint32_t u = ((word >> 4 * i) & 0x000f000fu) | Int4Pair<E>::kOnes;
    const Two v = __hsub2(*reinterpret_cast<const Two *>(&u), *reinterpret_cast<const Two *>(&zero));
    return *reinterpret_cast<const uint32_t *>(&v);
}

// A pair times a scale (in both halves), rounded once.
template <typename E>
__device__ __forceinline__ uint32_t int4_scaled(uint32_t pair, uint32_t scale)
{
    using Two = typename Int4Pair<E>::Two;
    const Two v = __hmul2(*reinterpret_cast<const Two *>(&pair), *reinterpret_cast<const Two *>(&scale));
    return *reinterpret_cast<const uint32_t *>(&v);
}

// The columns of a piece (16 bytes) of a row: its word j holds columns 128 (piece / 4) + 32 j + 8 (piece % 4) ... + 7.
__device__ __forceinline__ int64_t int4_column(int64_t piece, int j) { return piece / 4 * 128 + 32 * j + 8 * (piece % 4); }

}  // namespace lordba
