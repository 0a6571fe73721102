// What the two product kernels share: their operands as the copy engine sees them, and the epilogue.
#pragma once

#include "block_common.cuh"
#include "sm100.cuh"

namespace lordba {

// The epilogue of a product, in global memory.  vec flags: rows start on 16-byte boundaries.
struct Finish {
    void *out[2];
    int64_t ldo;
    const float *s_row, *s_col[2];
    const void *add[2];
    void *pre[2];
    int64_t ld_add, ld_pre, M, N;
    int dtype, act;
    int vec_out, vec_add, vec_pre;
};

// Whether the copy engine can take an operand of e-byte elements: base and pitch on 16-byte boundaries.  The
// tile kernel wants them all so; the stream kernel reads others itself.
inline bool taken_as_is(const Operand &o, int e) { return !o.p || (aligned(o.p, 16) && (o.ld * e) % 16 == 0); }

// The kernels' times in microseconds, as far as choosing between them needs; < 0: cannot be had.
double stream_estimate(const Product &p);
double tile_estimate(const Product &p);
int launch_product_tile(const Product &p, const Finish &f, cudaStream_t stream);     // product_tile.cu
int launch_product_stream(const Product &p, const Finish &f, cudaStream_t stream);   // product_stream.cu

// Encode a map of the row-major rows x cols matrix (pitch ld elements of e bytes) read in boxes of box_rows
// rows of 128 bytes, 128-byte swizzled; what lies outside the matrix reads as zero.
bool encode_map(CUtensorMap *map, const void *p, int64_t rows, int64_t cols, int64_t ld, int e, int box_rows);

int sm_count();      // of the current device

// ---- epilogue pieces ----------------------------------------------------------------------------------------
// COUNT consecutive elements of a row, of which the first n exist.
template <int COUNT>
__device__ __forceinline__ void load_row(const void *p, int64_t at, int n, int vec, int dtype, float v[COUNT])
{
    const uint16_t *q = static_cast<const uint16_t *>(p) + at;
    if (vec && n >= COUNT) {
        uint32_t w[COUNT / 2];
        if constexpr (COUNT % 8 == 0) {
#pragma unroll
            for (int i = 0; i < COUNT / 2; i += 4) {
                const uint4 x = *reinterpret_cast<const uint4 *>(q + 2 * i);
                w[i] = x.x; w[i + 1] = x.y; w[i + 2] = x.z; w[i + 3] = x.w;
            }
        } else {
            const uint2 x = *reinterpret_cast<const uint2 *>(q);
            w[0] = x.x; w[1] = x.y;
        }
#pragma unroll
        for (int i = 0; i < COUNT / 2; ++i) {
            const float2 f = dtype == LORDBA_BF16 ? unpack2<__nv_bfloat16>(w[i]) : unpack2<__half>(w[i]);
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
            v[i] = i >= n ? 0.0f
                   : dtype == LORDBA_BF16 ? to_float(reinterpret_cast<const __nv_bfloat16 *>(q)[i])
                                          : to_float(reinterpret_cast<const __half *>(q)[i]);
    }
}

template <int COUNT>
__device__ __forceinline__ void store_row(void *p, int64_t at, int n, int vec, int dtype, const float v[COUNT])
{
    if (dtype == LORDBA_F32) {
        float *q = static_cast<float *>(p) + at;
        if (vec && n >= COUNT) {
#pragma unroll
            for (int i = 0; i < COUNT; i += 4) *reinterpret_cast<float4 *>(q + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < COUNT; ++i)
                if (i < n) q[i] = v[i];
        }
        return;
    }
    uint16_t *q = static_cast<uint16_t *>(p) + at;
    uint32_t w[COUNT / 2];
#pragma unroll
    for (int i = 0; i < COUNT / 2; ++i)
        w[i] = dtype == LORDBA_BF16 ? pack2<__nv_bfloat16>(v[2 * i], v[2 * i + 1]) : pack2<__half>(v[2 * i], v[2 * i + 1]);
    if (vec && n >= COUNT) {
        if constexpr (COUNT % 8 == 0) {
#pragma unroll
            for (int i = 0; i < COUNT / 2; i += 4) *reinterpret_cast<uint4 *>(q + 2 * i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
        } else {
            *reinterpret_cast<uint2 *>(q) = make_uint2(w[0], w[1]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
            if (i < n) q[i] = (uint16_t)((i & 1) ? w[i / 2] >> 16 : w[i / 2] & 0xffffu);
    }
}

// The epilogue of COUNT columns of one row: acc0 the sums (of the gate), acc1 those of up.
template <bool INT8, bool GATED, int COUNT>
__device__ __forceinline__ void finish_row(const Finish &F, int problem, int64_t m, int64_t n, const uint32_t acc0[COUNT],
                                           const uint32_t acc1[COUNT])
{
    const int left = (int)(F.N - n < COUNT ? F.N - n : COUNT);
    float v[COUNT], w[COUNT];
    const float s = INT8 ? __ldg(F.s_row + m) : 0.0f;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        if (INT8) {
            const int64_t c = n + (i < left ? i : 0);
            v[i] = (float)(int)acc0[i] * s * __ldg(F.s_col[0] + c);
            if (GATED) w[i] = (float)(int)acc1[i] * s * __ldg(F.s_col[1] + c);
        } else {
            v[i] = __uint_as_float(acc0[i]);
            if (GATED) w[i] = __uint_as_float(acc1[i]);
        }
    }
    if (GATED) {
        if (F.add[0]) {
            float a[COUNT];
            load_row<COUNT>(F.add[0], m * F.ld_add + n, left, F.vec_add, F.dtype, a);
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[i] += a[i];
            load_row<COUNT>(F.add[1], m * F.ld_add + n, left, F.vec_add, F.dtype, a);
#pragma unroll
            for (int i = 0; i < COUNT; ++i) w[i] += a[i];
        }
        if (F.pre[0]) {
            store_row<COUNT>(F.pre[0], m * F.ld_pre + n, left, F.vec_pre, F.dtype, v);
            store_row<COUNT>(F.pre[1], m * F.ld_pre + n, left, F.vec_pre, F.dtype, w);
        }
        if (F.act == LORDBA_ACT_SILU) {
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[i] = act_gate<LORDBA_ACT_SILU>(v[i]) * w[i];
        } else {
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[i] = act_gate<LORDBA_ACT_GELU_TANH>(v[i]) * w[i];
        }
    }
    store_row<COUNT>(F.out[problem], m * F.ldo + n, left, F.vec_out, F.dtype, v);
}

}  // namespace lordba
