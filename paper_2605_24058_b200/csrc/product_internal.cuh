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
    int vec_out, vec_add, vec_pre, vec_scale;
};

// Whether the copy engine can take an operand of e-byte elements: base and pitch on 16-byte boundaries.  The
// tile kernel wants them all so; the stream kernel reads others itself.
inline bool taken_as_is(const Operand &o, int e) { return !o.p || (aligned(o.p, 16) && (o.ld * e) % 16 == 0); }

// The kernels' times in microseconds, as far as choosing between them needs; < 0: cannot be had.
double stream_estimate(const Product &p);
double tile_estimate(const Product &p);
int launch_product_tile(const Product &p, const Finish &f, cudaStream_t stream);     // product_tile.cu
size_t stream_workspace_bytes(const Product &p);                                     // product_stream.cu
int launch_product_stream(const Product &p, const Finish &f, void *workspace, cudaStream_t stream);

// Encode a map of the row-major rows x cols matrix (pitch ld elements of e bytes) read in boxes of box_rows
// rows of 128 bytes, 128-byte swizzled; what lies outside the matrix reads as zero.
bool encode_map(CUtensorMap *map, const void *p, int64_t rows, int64_t cols, int64_t ld, int e, int box_rows);
// The same for writing boxes of 32 rows of 64 bytes, 64-byte swizzled (e = 2 or 4).
bool encode_store_map(CUtensorMap *map, void *p, int64_t rows, int64_t cols, int64_t ld, int e);

int sm_count();      // of the current device

// ---- epilogue pieces ----------------------------------------------------------------------------------------
// COUNT scales, of which the first n exist.
template <int COUNT>
__device__ __forceinline__ void load_scales(const float *p, int n, int vec, float v[COUNT])
{
    if (vec && n >= COUNT) {
#pragma unroll
        for (int i = 0; i < COUNT; i += 4) {
            const float4 x = __ldg(reinterpret_cast<const float4 *>(p + i));
            v[i] = x.x; v[i + 1] = x.y; v[i + 2] = x.z; v[i + 3] = x.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = __ldg(p + (i < n ? i : 0));
    }
}

// The sums of COUNT columns from n on, `left` of which exist, as the products they stand for.
template <bool INT8, bool GATED, int COUNT>
__device__ __forceinline__ void products_of(const Finish &F, int64_t m, int64_t n, int left, const uint32_t acc0[COUNT],
                                            const uint32_t acc1[COUNT], float v[COUNT], float w[COUNT])
{
    if (INT8) {
        const float s = __ldg(F.s_row + m);
        load_scales<COUNT>(F.s_col[0] + n, left, F.vec_scale, v);
        if (GATED) load_scales<COUNT>(F.s_col[1] + n, left, F.vec_scale, w);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            v[i] *= (float)(int)acc0[i] * s;
            if (GATED) w[i] *= (float)(int)acc1[i] * s;
        }
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            v[i] = __uint_as_float(acc0[i]);
            if (GATED) w[i] = __uint_as_float(acc1[i]);
        }
    }
}

// v = act(v) w
template <int COUNT>
__device__ __forceinline__ void gate(int act, float v[COUNT], const float w[COUNT])
{
    if (act == LORDBA_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = act_gate<LORDBA_ACT_SILU>(v[i]) * w[i];
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = act_gate<LORDBA_ACT_GELU_TANH>(v[i]) * w[i];
    }
}

__device__ __forceinline__ float2 unpack2_any(uint32_t w, int dtype)
{
    return dtype == LORDBA_BF16 ? unpack2<__nv_bfloat16>(w) : unpack2<__half>(w);
}
__device__ __forceinline__ uint32_t pack2_any(float lo, float hi, int dtype)
{
    return dtype == LORDBA_BF16 ? pack2<__nv_bfloat16>(lo, hi) : pack2<__half>(lo, hi);
}

}  // namespace lordba
