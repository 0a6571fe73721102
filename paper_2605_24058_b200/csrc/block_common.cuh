// Element access shared by the kernels next to the adapters.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "lordba_internal.h"

namespace lordba {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename E> __device__ __forceinline__ E from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// Two neighbouring 16-bit elements in one word, lower address in the low half.
template <typename E> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w)
{
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w)
{
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}
template <typename E> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// Eight consecutive elements as they lie in memory: 16 bytes, or 32 of float.
template <typename E> struct Group8 { uint4 w; };
template <> struct Group8<float> { uint4 w, w2; };

template <typename E>
__device__ __forceinline__ Group8<E> load_group(const E *p)
{
    Group8<E> g;
    g.w = *reinterpret_cast<const uint4 *>(p);
    if constexpr (sizeof(E) == 4) g.w2 = *reinterpret_cast<const uint4 *>(p + 4);
    return g;
}
template <typename E>
__device__ __forceinline__ void unpack_group(const Group8<E> &g, float v[8])
{
    const uint32_t w[4] = {g.w.x, g.w.y, g.w.z, g.w.w};
    if constexpr (sizeof(E) == 4) {
        const uint32_t w2[4] = {g.w2.x, g.w2.y, g.w2.z, g.w2.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = __uint_as_float(w[i]); v[4 + i] = __uint_as_float(w2[i]); }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack2<E>(w[i]);
            v[2 * i] = f.x; v[2 * i + 1] = f.y;
        }
    }
}
template <typename E>
__device__ __forceinline__ void store_group(E *p, const float v[8])
{
    if constexpr (sizeof(E) == 4) {
        *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack2<E>(v[0], v[1]), pack2<E>(v[2], v[3]), pack2<E>(v[4], v[5]),
                                                  pack2<E>(v[6], v[7]));
    }
}

// Two floats in one register pair, worked on by one instruction.
struct Two {
    uint64_t v;
};
__device__ __forceinline__ Two two(float a, float b)
{
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 halves(Two t)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(t.v));
    return r;
}
__device__ __forceinline__ Two fma_two(Two a, Two b, Two c)
{
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ Two mul_two(Two a, Two b)
{
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Two add_two(Two a, Two b)
{
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}

// Sixteen bytes at an address that is `by` (0 ... 15) past an aligned one, from the two aligned pieces there.
__device__ __forceinline__ uint4 join_pieces(uint4 a, uint4 b, uint32_t by)
{
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    const bool eight = by & 8u, four = by & 4u;
    const uint32_t shift = 8 * (by & 3u);
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = eight ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = four ? w[i + 1] : w[i];
    return make_uint4(__funnelshift_r(w[0], w[1], shift), __funnelshift_r(w[1], w[2], shift),
                      __funnelshift_r(w[2], w[3], shift), __funnelshift_r(w[3], w[4], shift));
}

// The sixteen bytes at any address at < end; bytes from `end` on read as zero, and an aligned piece is read
// only when it holds a byte before `end`.  CONST: nothing writes there while the kernel runs.
template <bool CONST = true>
__device__ __forceinline__ uint4 load_bytes16(uintptr_t at, uintptr_t end)
{
    const uintptr_t first = at & ~(uintptr_t)15;
    const uintptr_t second = (at & 15) && first + 16 < end ? first + 16 : first;
    const uint4 *pa = reinterpret_cast<const uint4 *>(first), *pb = reinterpret_cast<const uint4 *>(second);
    const uint4 v = CONST ? join_pieces(__ldg(pa), __ldg(pb), (uint32_t)at & 15u) : join_pieces(*pa, *pb, (uint32_t)at & 15u);
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
    const int left = end - at < 16 ? (int)(end - at) : 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int bytes = left - 4 * i;
        w[i] &= bytes >= 4 ? 0xffffffffu : bytes <= 0 ? 0u : (1u << 8 * bytes) - 1u;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Columns 8 g ... 8 g + 7 of a row of d elements; what lies past d reads as zero.  (Dropout may run in place:
// these are ordinary loads.)
template <typename E>
__device__ __noinline__ Group8<E> load8_last(const E *row, int64_t g, int64_t d)
{
    Group8<E> v;
    const uintptr_t at = reinterpret_cast<uintptr_t>(row + 8 * g), end = reinterpret_cast<uintptr_t>(row + d);
    v.w = load_bytes16<false>(at, end);
    if constexpr (sizeof(E) == 4) v.w2 = at + 16 < end ? load_bytes16<false>(at + 16, end) : make_uint4(0, 0, 0, 0);
    return v;
}

template <typename E>
__device__ __forceinline__ Group8<E> load8(const E *row, int64_t g, int64_t d, bool vec)
{
    if (8 * g + 8 > d) return load8_last(row, g, d);
    if (vec) return load_group(row + 8 * g);
    // a whole group, off the 16-byte grid: the aligned pieces that hold it all hold bytes of it
    const uintptr_t at = reinterpret_cast<uintptr_t>(row + 8 * g);
    const uint4 *p = reinterpret_cast<const uint4 *>(at & ~(uintptr_t)15);
    const uint32_t by = (uint32_t)at & 15u;
    constexpr int kWhole = sizeof(Group8<E>) / 16;
    uint4 x[kWhole + 1];
#pragma unroll
    for (int i = 0; i < kWhole; ++i) x[i] = p[i];
    x[kWhole] = p[by ? kWhole : 0];
    Group8<E> v;
    v.w = join_pieces(x[0], x[1], by);
    if constexpr (sizeof(E) == 4) v.w2 = join_pieces(x[1], x[2], by);
    return v;
}

template <typename E>
__device__ __noinline__ void store8_parts(E *row, int64_t g, int64_t d, float v0, float v1, float v2, float v3, float v4, float v5,
                                          float v6, float v7)
{
    const float v[8] = {v0, v1, v2, v3, v4, v5, v6, v7};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (8 * g + i < d) row[8 * g + i] = from_float<E>(v[i]);
}

template <typename E>
__device__ __forceinline__ void store8(E *row, int64_t g, int64_t d, bool vec, const float v[8])
{
    if (vec && 8 * g + 8 <= d) store_group<E>(row + 8 * g, v);
    else store8_parts(row, g, d, v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]);
}

// FULL: every matrix allows 16-byte accesses and d is a multiple of 8, so nothing is looked at per access
template <bool FULL, typename E>
__device__ __forceinline__ Group8<E> load_either(const E *row, int64_t g, int64_t d, bool vec)
{
    return FULL ? load_group(row + 8 * g) : load8(row, g, d, vec);
}
template <bool FULL, typename E>
__device__ __forceinline__ void store_either(E *row, int64_t g, int64_t d, bool vec, const float v[8])
{
    if (FULL) store_group<E>(row + 8 * g, v);
    else store8(row, g, d, vec, v);
}

// Programmatic dependent launch: a kernel's first global access comes after grid_wait(), so that the
// kernels before it are complete; its successor may become resident as soon as every CTA has passed
// grid_release().
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// act(g) = g f(k(g)), f the logistic function: k(g) = g for silu, 2 sqrt(2/pi) (g + 0.044715 g^3) for the
// tanh form of gelu, since (1 + tanh(z)) / 2 = f(2 z).
constexpr float kGelu = 1.5957691216057308f;      // 2 sqrt(2 / pi)
constexpr float kGeluCubic = 0.044715f;

// 1 / (1 + e^-z) with the hardware's exponential and reciprocal (2^-22 each), subnormals flushed: the
// forms that keep them cost eight instructions more, and the epilogues are bound by their instructions.
__device__ __forceinline__ float logistic(float z)
{
    constexpr float kLog2E = 1.4426950408889634f;
    float e, f;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-kLog2E * z));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(f) : "f"(1.0f + e));
    return f;
}

// Beyond |g| = 128 f is 0 or 1 in 32 bits, so a factor beside it may be clamped there without changing a result: an
// infinity then does not meet that zero (act(-inf) is 0, as for any g below -128), and a NaN still comes through f.
constexpr float kFlat = 128.0f;

template <int ACT>
__device__ __forceinline__ float act_gate(float g)
{
    return fmaxf(g, -kFlat) * logistic(ACT == LORDBA_ACT_SILU ? g : kGelu * g * fmaf(kGeluCubic * g, g, 1.0f));
}

// act(g) and act'(g) = f + g f (1 - f) k'(g)
template <int ACT>
__device__ __forceinline__ void act_and_slope(float g, float &value, float &slope)
{
    const float f = logistic(ACT == LORDBA_ACT_SILU ? g : kGelu * g * fmaf(kGeluCubic * g, g, 1.0f));
    const float low = fmaxf(g, -kFlat), c = fminf(low, kFlat);
    const float inner = ACT == LORDBA_ACT_SILU ? 1.0f : kGelu * fmaf(3.0f * kGeluCubic * c, c, 1.0f);
    value = low * f;
    slope = fmaf(c * f * (1.0f - f), inner, f);
}

// One launch with programmatic stream serialization: the kernel must call grid_wait().
template <typename... Args>
int launch_kernel(void (*kernel)(Args...), dim3 grid, unsigned block, unsigned smem, cudaStream_t stream, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) {
        cudaGetLastError();
        return LORDBA_ECUDA;
    }
    count_launch();
    return LORDBA_OK;
}

}  // namespace lordba
