// The 4-bit carrier's words as pairs of 16-bit numbers (int4.cu, int4_few.cu).
#pragma once

#include <type_traits>

#include "block_common.cuh"

namespace lordba {

// A number u = 0 ... 15 put into the low bits of this pattern is the float 128 + u (bfloat16) or 1024 + u (float16), exactly;
// the same pattern with a sign and the zero point z in it is -(128 + z), and their sum is u - z, exactly.  So a pair costs a
// shift, one three-input logic operation and one multiply-add of two halves.
template <typename E> constexpr uint32_t kInt4Ones = 0x64006400u;
template <> constexpr uint32_t kInt4Ones<__nv_bfloat16> = 0x43004300u;
template <typename E> constexpr uint32_t kOnePair = 0x3c003c00u;
template <> constexpr uint32_t kOnePair<__nv_bfloat16> = 0x3f803f80u;

// a b + c of two halves, each rounded once.
template <typename E>
__device__ __forceinline__ uint32_t fma_pair(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    if constexpr (std::is_same_v<E, __nv_bfloat16>) asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    else asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}

// The pattern of a zero point, in both halves.
template <typename E>
__host__ __device__ __forceinline__ uint32_t int4_zero(uint32_t z) { return kInt4Ones<E> | 0x80008000u | z | z << 16; }

// Columns 2 i and 2 i + 1 of a word, less the zero point.  An instruction has room for one constant: `ones` (kInt4Ones) and
// `zero` want to come from memory, or each is moved into a register again for every pair.
template <typename E>
__device__ __forceinline__ uint32_t int4_pair(uint32_t word, int i, uint32_t zero, uint32_t ones = kInt4Ones<E>)
{
    uint32_t u;          // (word >> 4 i) & mask | ones
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(u) : "r"(word >> 4 * i), "r"(0x000f000fu), "r"(ones));
    return fma_pair<E>(u, kOnePair<E>, zero);
}

// A pair times a scale (in both halves), rounded once.
template <typename E>
__device__ __forceinline__ uint32_t int4_scaled(uint32_t pair, uint32_t scale) { return fma_pair<E>(pair, scale, 0x80008000u); }

// The columns of a piece (16 bytes) of a row: its word j holds columns 128 (piece / 4) + 32 j + 8 (piece % 4) ... + 7.
__device__ __forceinline__ int64_t int4_column(int64_t piece, int j) { return piece / 4 * 128 + 32 * j + 8 * (piece % 4); }

}  // namespace lordba
