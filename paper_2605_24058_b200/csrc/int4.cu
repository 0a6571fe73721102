// The 4-bit carrier: packing, quantisation and its way back to 16-bit weights.
//
// Packing and quantising happen once a weight and are no part of a step; the way back stands before products of many tokens, which take the
// weights as a 16-bit matrix (int4_linear).  11008 x 4096, floors by bytes in brackets: way back 21.7 us (17.3), pack 25.5 (10.3: a byte an
// access), quantise from bf16 116 us (17.3), from f32 113 (31): the exact quotients take it, a division and its check a weight.
#include "int4_common.cuh"

namespace lordba {
namespace {

constexpr int kThreads = 256;

// ---- lordba_int4_pack: a thread makes a word ---------------------------------------------------------------------
__global__ void __launch_bounds__(kThreads)
int4_pack_kernel(const uint8_t *__restrict__ values, int64_t ldv, uint8_t *__restrict__ q, int64_t ldq, int64_t rows, int64_t d_in, int64_t words)
{
    const int64_t w = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    grid_wait();
    grid_release();
    if (w >= words) return;
    const int64_t c0 = int4_column(w / 4, (int)(w % 4));
    for (int64_t n = blockIdx.y; n < rows; n += gridDim.y) {
        const uint8_t *v = values + n * ldv + c0;
        uint32_t word = 0;
#pragma unroll
        for (int c = 0; c < 8; ++c)
            if (c0 + c < d_in) word |= (uint32_t)(v[c] & 15u) << (4 * (c / 2) + 16 * (c % 2));
        *reinterpret_cast<uint32_t *>(q + n * ldq + 4 * w) = word;
    }
}

// ---- lordba_int4_quantize -----------------------------------------------------------------------------------------
// w / scale to the nearest whole number, ties to even, of the exact quotient: rint of the rounded one may be off where
// that lies next to a half, and what is left of w then says so (it is exact: few bits times a small number).
__device__ __forceinline__ float nearest(float w, float scale)
{
    float r = rintf(__fdiv_rn(w, scale));
    const float left = fmaf(-r, scale, w), half = 0.5f * scale;
    if (fabsf(left) > half || (fabsf(left) == half && fmodf(r, 2.0f) != 0.0f)) r += copysignf(1.0f, left);
    return r;
}

// `lanes` lanes of a warp hold a group: they look for its largest and smallest value, then write its words.  A row's units are
// its groups and, where its last block reaches further, the words behind them.
template <typename W, typename S, bool ZERO>
__global__ void __launch_bounds__(kThreads)
int4_quantize_kernel(const W *__restrict__ w, int64_t ldw, uint8_t *__restrict__ q, int64_t ldq, S *__restrict__ scale, int64_t ld_scale,
                     uint8_t *__restrict__ zero, int64_t ld_zero, int64_t rows, int64_t d_in, int64_t groups, int64_t units, int64_t runs, int group_runs, int lanes)
{
    const int lane = threadIdx.x % 32, sub = lane % lanes, per_warp = 32 / lanes;
    const int64_t warp = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 32;
    grid_wait();
    grid_release();
    const int64_t unit = warp * per_warp + lane / lanes;
    if (warp * per_warp >= units) return;
    for (int64_t n = blockIdx.y; n < rows; n += gridDim.y) {
        const W *row = w + n * ldw;
        float lo = 0.0f, hi = 0.0f;
        bool nan = false;
        if (unit < groups)
            for (int i = sub; i < group_runs; i += lanes) {
                const int64_t c0 = 8 * (unit * group_runs + i);
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    if (c0 + c >= d_in) break;
                    const float v = to_float(row[c0 + c]);
                    lo = fminf(lo, v);
                    hi = fmaxf(hi, v);
                    nan |= v != v;
                }
            }
        for (int o = lanes / 2; o; o /= 2) {
            lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
            hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
            nan |= __shfl_xor_sync(0xffffffffu, (int)nan, o) != 0;
        }
        const float wide = ZERO ? __fdiv_rn(hi - lo, 15.0f) : __fdiv_rn(fmaxf(hi, -lo), 7.0f);
        const S s = from_float<S>(wide);
        const float sf = to_float(s);
        const bool finite = sf < INFINITY && !nan, live = finite && sf > 0.0f;
        const float z = ZERO && live ? fminf(nearest(-lo, sf), 15.0f) : 8.0f;
        if (unit < groups && sub == 0) {
            scale[n * ld_scale + unit] = finite ? s : from_float<S>(__uint_as_float(0x7fc00000u));
            if (ZERO) zero[n * ld_zero + unit] = (uint8_t)z;
        }
        if (unit < units)
            for (int i = sub; i < group_runs; i += lanes) {
                const int64_t run = unit * group_runs + i;
                if (run >= runs) break;
                uint32_t word = 0;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    float u = z;
                    if (live && 8 * run + c < d_in) u = fminf(fmaxf(nearest(to_float(row[8 * run + c]), sf) + z, 0.0f), 15.0f);
                    word |= (uint32_t)u << (4 * (c / 2) + 16 * (c % 2));
                }
                // run 16 b + 4 j + t is word 4 t + j of block b
                *reinterpret_cast<uint32_t *>(q + n * ldq + 4 * (run / 16 * 16 + run % 4 * 4 + run / 4 % 4)) = word;
            }
    }
}

// ---- the way back --------------------------------------------------------------------------------------------------
// A thread takes a piece (16 bytes) of a row: four runs of eight columns, 32 columns apart; four neighbouring threads
// write 64 bytes side by side.
template <typename E, bool VEC>
__global__ void __launch_bounds__(kThreads)
int4_dequantize_kernel(const uint8_t *__restrict__ q, int64_t ldq, const E *__restrict__ scale, int64_t ld_scale, const uint8_t *__restrict__ zero,
                       int64_t ld_zero, E *__restrict__ out, int64_t ldo, int64_t rows, int64_t d_in, int64_t pieces, int group_log2)
{
    const int64_t piece = (int64_t)blockIdx.x * 32 + threadIdx.x % 32;
    grid_wait();
    grid_release();
    if (piece >= pieces) return;
    for (int64_t n = (int64_t)blockIdx.y * (kThreads / 32) + threadIdx.x / 32; n < rows; n += (int64_t)gridDim.y * (kThreads / 32)) {
        const uint4 x = __ldg(reinterpret_cast<const uint4 *>(q + n * ldq) + piece);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t c0 = int4_column(piece, j);
            if (c0 >= d_in) break;
            const int64_t g = c0 >> group_log2;
            const uint16_t s = __ldg(reinterpret_cast<const uint16_t *>(scale + n * ld_scale + g));
            const uint32_t z = int4_zero<E>(zero ? __ldg(zero + n * ld_zero + g) & 15u : 8u), ss = s | (uint32_t)s << 16;
            uint32_t v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = int4_scaled<E>(int4_pair<E>(w[j], i, z), ss);
            E *to = out + n * ldo + c0;
            if (VEC && c0 + 8 <= d_in) {
                *reinterpret_cast<uint4 *>(to) = make_uint4(v[0], v[1], v[2], v[3]);
            } else {
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (c0 + c < d_in) reinterpret_cast<uint16_t *>(to)[c] = (uint16_t)(v[c / 2] >> 16 * (c % 2));
            }
        }
    }
}

int log2_of(int group)
{
    int n = 0;
    while ((1 << n) < group) ++n;
    return n;
}

unsigned rows_grid(int64_t rows) { return (unsigned)(rows < 65535 ? rows : 65535); }

template <typename W, typename S>
int quantize_typed(const void *w, int64_t ldw, uint8_t *q, int64_t ldq, void *scale, int64_t ld_scale, uint8_t *zero, int64_t ld_zero,
                   int64_t d_out, int64_t d_in, int group, cudaStream_t stream)
{
    const int64_t groups = (d_in + group - 1) / group, runs = (d_in + 127) / 128 * 16;
    const int64_t group_runs = group / 8 < runs ? group / 8 : runs, units = (runs + group_runs - 1) / group_runs;
    const int lanes = group_runs < 32 ? (int)group_runs : 32;
    const int64_t warps = (units + 32 / lanes - 1) / (32 / lanes);
    const dim3 grid((unsigned)((warps + kThreads / 32 - 1) / (kThreads / 32)), rows_grid(d_out), 1);
    const auto kernel = zero ? int4_quantize_kernel<W, S, true> : int4_quantize_kernel<W, S, false>;
    return launch_kernel(kernel, grid, kThreads, 0, stream, static_cast<const W *>(w), ldw, q, ldq, static_cast<S *>(scale), ld_scale, zero,
                         ld_zero, d_out, d_in, groups, units, runs, (int)group_runs, lanes);
}

template <typename W>
int quantize_scaled(const void *w, int64_t ldw, uint8_t *q, int64_t ldq, void *scale, int64_t ld_scale, uint8_t *zero, int64_t ld_zero,
                    int64_t d_out, int64_t d_in, int group, int dtype, cudaStream_t stream)
{
    return dtype == LORDBA_BF16 ? quantize_typed<W, __nv_bfloat16>(w, ldw, q, ldq, scale, ld_scale, zero, ld_zero, d_out, d_in, group, stream)
                                : quantize_typed<W, __half>(w, ldw, q, ldq, scale, ld_scale, zero, ld_zero, d_out, d_in, group, stream);
}

template <typename E>
int dequantize_typed(const lordba_int4_proj &p, cudaStream_t stream)
{
    const int64_t pieces = (p.d_in + 127) / 128 * 4, rows = (p.d_out + kThreads / 32 - 1) / (kThreads / 32);
    const bool vec = aligned(p.out, 16) && p.ld_out % 8 == 0;
    const dim3 grid((unsigned)((pieces + 31) / 32), rows_grid(rows), 1);
    const auto kernel = vec ? int4_dequantize_kernel<E, true> : int4_dequantize_kernel<E, false>;
    return launch_kernel(kernel, grid, kThreads, 0, stream, p.q, p.ldq, static_cast<const E *>(p.scale), p.ld_scale, p.zero, p.ld_zero,
                         static_cast<E *>(p.out), p.ld_out, p.d_out, p.d_in, pieces, log2_of(p.group));
}

}  // namespace

int launch_int4_pack(const uint8_t *values, int64_t ldv, uint8_t *q, int64_t ldq, int64_t d_out, int64_t d_in, cudaStream_t stream)
{
    const int64_t words = (d_in + 127) / 128 * 16;
    const dim3 grid((unsigned)((words + kThreads - 1) / kThreads), rows_grid(d_out), 1);
    return launch_kernel(int4_pack_kernel, grid, kThreads, 0, stream, values, ldv, q, ldq, d_out, d_in, words);
}

int launch_int4_quantize(const void *w, int64_t ldw, int wdtype, uint8_t *q, int64_t ldq, void *scale, int64_t ld_scale, uint8_t *zero,
                         int64_t ld_zero, int64_t d_out, int64_t d_in, int group, int dtype, cudaStream_t stream)
{
    const auto f = wdtype == LORDBA_F32 ? quantize_scaled<float> : wdtype == LORDBA_BF16 ? quantize_scaled<__nv_bfloat16> : quantize_scaled<__half>;
    return f(w, ldw, q, ldq, scale, ld_scale, zero, ld_zero, d_out, d_in, group, dtype, stream);
}

int launch_int4_dequantize(const lordba_int4_proj &p, int dtype, cudaStream_t stream)
{
    return dtype == LORDBA_BF16 ? dequantize_typed<__nv_bfloat16>(p, stream) : dequantize_typed<__half>(p, stream);
}

}  // namespace lordba
