// The streaming kernels next to the adapters: per-token quantisation to 8 bits, dropout from a
// counter-based generator, the elementwise part of the gated block's backward pass, and the copy that
// gives an operand a pitch the copy engine can take.
//
// All of them are bound by HBM: each element is read once and written once, eight elements (16 bytes of a
// 16-bit type) an access.  Rows whose base or pitch does not allow such accesses go element by element
// (the VEC = false instantiations).
#include "block_common.cuh"

namespace lordba {
namespace {

constexpr int kEltThreads = 256;

// Eight elements of a row starting at column 8 g; columns past d read as zero.
template <typename E, bool VEC>
__device__ __forceinline__ void load8(const E *row, int64_t g, int64_t d, float v[8])
{
    if (VEC && 8 * g + 8 <= d) {
        unpack_group<E>(load_group(row + 8 * g), v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 8 * g + i < d ? to_float(row[8 * g + i]) : 0.0f;
    }
}

template <typename E, bool VEC>
__device__ __forceinline__ void store8(E *row, int64_t g, int64_t d, const float v[8])
{
    if (VEC && 8 * g + 8 <= d) {
        store_group<E>(row + 8 * g, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (8 * g + i < d) row[8 * g + i] = from_float<E>(v[i]);
    }
}

// ---- lordba_int8_quantize_rows ----------------------------------------------------------------------
// TPR threads hold a row: its groups of eight stay in registers between the search for the maximum and
// the rounding (NV groups a thread; what a longer row has beyond them is read again, from L2).  The
// maximum is taken over the bit patterns of |x|, which order like the numbers with NaN above infinity.
template <typename E, int TPR, int NV, bool VEC>
__global__ void __launch_bounds__(kEltThreads)
quantize_rows_kernel(const E *__restrict__ x, int64_t ldx, int8_t *__restrict__ q, int64_t ldq, int qvec,
                     float *__restrict__ scale, int64_t T, int64_t d)
{
    constexpr int kRows = kEltThreads / TPR;
    __shared__ uint32_t part[kEltThreads / 32];
    const int tid = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
    const int64_t groups = (d + 7) / 8;
    grid_wait();
    grid_release();
    if (TPR == 32 && row >= T) return;          // whole warps; with TPR = 256 every block has its row
    const E *xr = x + row * ldx;
    float v[NV][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t g = tid + (int64_t)i * TPR;
        if (g < groups) {
            load8<E, VEC>(xr, g, d, v[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[i][j]) & 0x7fffffffu);
    for (int64_t g = tid + (int64_t)NV * TPR; g < groups; g += TPR) {
        float w[8];
        load8<E, VEC>(xr, g, d, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(w[j]) & 0x7fffffffu);
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (TPR > 32) {
        if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = top;
        __syncthreads();
        top = part[threadIdx.x % (kEltThreads / 32)];
        top = __reduce_max_sync(0xffffffffu, top);
    }
    const bool finite = top < 0x7f800000u;
    const float amax = __uint_as_float(top);
    const bool live = finite && amax >= 0x1p-120f;      // below it 127 / amax could overflow
    const float inverse = live ? 127.0f / amax : 0.0f;
    if (tid == 0) scale[row] = finite ? (live ? amax / 127.0f : 0.0f) : __uint_as_float(0x7fc00000u);
    int8_t *qr = q + row * ldq;
    auto put = [&](int64_t g, const float w[8]) {
        int b[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = live ? __float2int_rn(w[j] * inverse) : 0;
        if (qvec && 8 * g + 8 <= d) {
            const uint32_t lo = (b[0] & 255) | (b[1] & 255) << 8 | (b[2] & 255) << 16 | (uint32_t)b[3] << 24;
            const uint32_t hi = (b[4] & 255) | (b[5] & 255) << 8 | (b[6] & 255) << 16 | (uint32_t)b[7] << 24;
            *reinterpret_cast<uint2 *>(qr + 8 * g) = make_uint2(lo, hi);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (8 * g + j < d) qr[8 * g + j] = (int8_t)b[j];
        }
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t g = tid + (int64_t)i * TPR;
        if (g < groups) put(g, v[i]);
    }
    for (int64_t g = tid + (int64_t)NV * TPR; g < groups; g += TPR) {
        float w[8];
        load8<E, VEC>(xr, g, d, w);
        put(g, w);
    }
}

// ---- the shape of the elementwise grids ---------------------------------------------------------------
// Thread (bx, by) of a block owns column group blockIdx.x * width + bx of rows blockIdx.y * height + by +
// k * gridDim.y * height: no division by the row length anywhere.
struct EltGrid {
    int width_log2;       // a block is 2^width_log2 groups wide and kEltThreads >> width_log2 rows high
    dim3 grid;
};

EltGrid elementwise_grid(int64_t T, int64_t d)
{
    const int64_t groups = (d + 7) / 8;
    // the width that leaves the fewest threads without a column; the wider one of two equals
    int best = 3;
    int64_t best_cover = -1;
    for (int w = 8; w >= 3; --w) {
        const int64_t cover = ((groups + (1 << w) - 1) >> w) << w;
        if (best_cover < 0 || cover < best_cover) { best = w; best_cover = cover; }
    }
    const int64_t height = kEltThreads >> best;
    int64_t gx = (groups + (1 << best) - 1) >> best, gy = (T + height - 1) / height;
    // eight resident blocks per SM and a few rounds of them are enough; the rows beyond are a loop
    const int64_t most = gx >= 148 * 32 ? 1 : 148 * 32 / gx;
    if (gy > most) gy = most;
    if (gy > 65535) gy = 65535;
    if (gy < 1) gy = 1;
    EltGrid e;
    e.width_log2 = best;
    e.grid = dim3((unsigned)gx, (unsigned)gy, 1);
    return e;
}

// ---- lordba_dropout -----------------------------------------------------------------------------------
// Philox4x32-10: ten rounds of two 32 x 32 -> 64 bit products; the multipliers and the key increments are
// the published ones.
__device__ __forceinline__ uint4 philox(uint4 c, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)c.x * 0xD2511F53u, b = (uint64_t)c.z * 0xCD9E8D57u;
        c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k1, (uint32_t)a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return c;
}

// out may be x or residual: a thread writes only the elements that it alone has read before.
template <typename E, bool VEC>
__global__ void __launch_bounds__(kEltThreads)
dropout_kernel(const E *x, int64_t ldx, const E *residual, int64_t ldr, E *out, int64_t ldo, int64_t T, int64_t d,
               uint32_t cut, float scale, uint64_t seed, uint64_t offset, int width_log2)
{
    const int64_t g = ((int64_t)blockIdx.x << width_log2) + (threadIdx.x & ((1 << width_log2) - 1));
    const int64_t height = kEltThreads >> width_log2;
    grid_wait();
    grid_release();
    if (8 * g >= d) return;
    for (int64_t t = blockIdx.y * height + (threadIdx.x >> width_log2); t < T; t += gridDim.y * height) {
        float v[8], r[8];
        load8<E, VEC>(x + t * ldx, g, d, v);
        if (residual) load8<E, VEC>(residual + t * ldr, g, d, r);
        const uint4 bits = philox(make_uint4((uint32_t)g, (uint32_t)t, (uint32_t)offset, (uint32_t)(offset >> 32)),
                                  (uint32_t)seed, (uint32_t)(seed >> 32));
        const uint32_t w[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t number = (i & 1) ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
            const float kept = number >= cut ? v[i] * scale : 0.0f;      // a choice, not a product with 0: x may be inf
            v[i] = residual ? kept + r[i] : kept;
        }
        store8<E, VEC>(out + t * ldo, g, d, v);
    }
}

// ---- dgate = dh up act'(gate), dup = dh act(gate) ---------------------------------------------------------
template <typename E, int ACT, bool VEC>
__global__ void __launch_bounds__(kEltThreads)
gated_grad_kernel(const E *__restrict__ dh, int64_t ld_dh, const E *__restrict__ gate, const E *__restrict__ up,
                  int64_t ld_pre, E *__restrict__ dgate, E *__restrict__ dup, int64_t ld_dpre, int64_t T, int64_t d,
                  int width_log2)
{
    const int64_t g = ((int64_t)blockIdx.x << width_log2) + (threadIdx.x & ((1 << width_log2) - 1));
    const int64_t height = kEltThreads >> width_log2;
    grid_wait();
    grid_release();
    if (8 * g >= d) return;
    for (int64_t t = blockIdx.y * height + (threadIdx.x >> width_log2); t < T; t += gridDim.y * height) {
        float vh[8], vg[8], vu[8];
        load8<E, VEC>(dh + t * ld_dh, g, d, vh);
        load8<E, VEC>(gate + t * ld_pre, g, d, vg);
        load8<E, VEC>(up + t * ld_pre, g, d, vu);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float value, slope;
            act_and_slope<ACT>(vg[i], value, slope);
            vu[i] *= vh[i] * slope;
            vh[i] *= value;
        }
        store8<E, VEC>(dgate + t * ld_dpre, g, d, vu);
        store8<E, VEC>(dup + t * ld_dpre, g, d, vh);
    }
}

// ---- repack ---------------------------------------------------------------------------------------------
// A thread writes 16 aligned bytes from the 4 or 5 aligned words that hold them; a word is read only when it
// holds a byte of the row.
__global__ void __launch_bounds__(kEltThreads)
repack_kernel(const uint8_t *__restrict__ src, int64_t ld_src, uint8_t *__restrict__ dst, int64_t ld_dst, int64_t rows,
              int64_t cols, int width_log2)
{
    const int64_t g = ((int64_t)blockIdx.x << width_log2) + (threadIdx.x & ((1 << width_log2) - 1));
    const int64_t height = kEltThreads >> width_log2;
    grid_wait();
    grid_release();
    if (16 * g >= cols) return;
    for (int64_t t = blockIdx.y * height + (threadIdx.x >> width_log2); t < rows; t += gridDim.y * height) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(src + t * ld_src + 16 * g);
        const uintptr_t end = reinterpret_cast<uintptr_t>(src + t * ld_src + cols);
        const uint32_t *p = reinterpret_cast<const uint32_t *>(at & ~(uintptr_t)3);
        const uint32_t shift = 8 * (uint32_t)(at & 3);
        uint32_t w[5];
#pragma unroll
        for (int i = 0; i < 5; ++i)
            w[i] = (reinterpret_cast<uintptr_t>(p + i) < end && (i < 4 || shift)) ? __ldg(p + i) : 0u;
        // bytes past the end of the row land in the destination's padding, which nothing reads
        *reinterpret_cast<uint4 *>(dst + t * ld_dst + 16 * g) =
            make_uint4(__funnelshift_r(w[0], w[1], shift), __funnelshift_r(w[1], w[2], shift),
                       __funnelshift_r(w[2], w[3], shift), __funnelshift_r(w[3], w[4], shift));
    }
}

// whether rows can be accessed eight elements at a time
bool vec_ok(const void *p, int64_t ld, size_t e) { return !p || (aligned(p, 16) && ((size_t)ld * e) % 16 == 0); }

template <typename E, bool VEC>
int quantize_typed(const E *x, int64_t ldx, int8_t *q, int64_t ldq, float *scale, int64_t T, int64_t d, cudaStream_t s)
{
    const int qvec = aligned(q, 8) && ldq % 8 == 0;
    // up to 1024 columns a warp holds a row (32 lanes x 4 groups of 8), beyond that a block (256 x 6 x 8 = 12288)
    if (d <= 1024)
        return launch_kernel(quantize_rows_kernel<E, 32, 4, VEC>, dim3((unsigned)((T + 7) / 8)), kEltThreads, 0, s, x, ldx, q,
                             ldq, qvec, scale, T, d);
    return launch_kernel(quantize_rows_kernel<E, 256, 6, VEC>, dim3((unsigned)T), kEltThreads, 0, s, x, ldx, q, ldq, qvec,
                         scale, T, d);
}

template <typename E>
int quantize_any(const void *x, int64_t ldx, int8_t *q, int64_t ldq, float *scale, int64_t T, int64_t d, cudaStream_t s)
{
    const E *xe = static_cast<const E *>(x);
    return vec_ok(x, ldx, sizeof(E)) ? quantize_typed<E, true>(xe, ldx, q, ldq, scale, T, d, s)
                                     : quantize_typed<E, false>(xe, ldx, q, ldq, scale, T, d, s);
}

template <typename E>
int dropout_any(const void *x, int64_t ldx, const void *r, int64_t ldr, void *out, int64_t ldo, int64_t T, int64_t d, int cut,
                uint64_t seed, uint64_t offset, cudaStream_t s)
{
    const EltGrid e = elementwise_grid(T, d);
    const float scale = cut < 65536 ? 65536.0f / (float)(65536 - cut) : 0.0f;
    const bool vec = vec_ok(x, ldx, sizeof(E)) && vec_ok(r, ldr, sizeof(E)) && vec_ok(out, ldo, sizeof(E));
    return launch_kernel(vec ? dropout_kernel<E, true> : dropout_kernel<E, false>, e.grid, kEltThreads, 0, s,
                         static_cast<const E *>(x), ldx, static_cast<const E *>(r), ldr, static_cast<E *>(out), ldo, T, d,
                         (uint32_t)cut, scale, seed, offset, e.width_log2);
}

template <typename E, int ACT>
int gated_grad_any(const lordba_gated_grad &g, int64_t T, cudaStream_t s)
{
    const EltGrid e = elementwise_grid(T, g.d_hidden);
    const bool vec = vec_ok(g.dh, g.ld_dh, 2) && vec_ok(g.gate, g.ld_pre, 2) && vec_ok(g.up, g.ld_pre, 2) &&
                     vec_ok(g.dgate, g.ld_dpre, 2) && vec_ok(g.dup, g.ld_dpre, 2);
    return launch_kernel(vec ? gated_grad_kernel<E, ACT, true> : gated_grad_kernel<E, ACT, false>, e.grid, kEltThreads, 0, s,
                         static_cast<const E *>(g.dh), g.ld_dh, static_cast<const E *>(g.gate),
                         static_cast<const E *>(g.up), g.ld_pre, static_cast<E *>(g.dgate), static_cast<E *>(g.dup),
                         g.ld_dpre, T, g.d_hidden, e.width_log2);
}

}  // namespace

int launch_quantize_rows(const void *x, int64_t ldx, int8_t *q, int64_t ldq, float *scale, int64_t T, int64_t d, int dtype,
                         cudaStream_t s)
{
    switch (dtype) {
        case LORDBA_BF16: return quantize_any<__nv_bfloat16>(x, ldx, q, ldq, scale, T, d, s);
        case LORDBA_F16: return quantize_any<__half>(x, ldx, q, ldq, scale, T, d, s);
        default: return quantize_any<float>(x, ldx, q, ldq, scale, T, d, s);
    }
}

int launch_dropout(const void *x, int64_t ldx, const void *residual, int64_t ldr, void *out, int64_t ldo, int64_t T,
                   int64_t d, int cut, uint64_t seed, uint64_t offset, int dtype, cudaStream_t s)
{
    switch (dtype) {
        case LORDBA_BF16: return dropout_any<__nv_bfloat16>(x, ldx, residual, ldr, out, ldo, T, d, cut, seed, offset, s);
        case LORDBA_F16: return dropout_any<__half>(x, ldx, residual, ldr, out, ldo, T, d, cut, seed, offset, s);
        default: return dropout_any<float>(x, ldx, residual, ldr, out, ldo, T, d, cut, seed, offset, s);
    }
}

int launch_gated_grad(const lordba_gated_grad &g, int64_t T, int dtype, cudaStream_t s)
{
    if (dtype == LORDBA_BF16)
        return g.act == LORDBA_ACT_SILU ? gated_grad_any<__nv_bfloat16, LORDBA_ACT_SILU>(g, T, s)
                                        : gated_grad_any<__nv_bfloat16, LORDBA_ACT_GELU_TANH>(g, T, s);
    return g.act == LORDBA_ACT_SILU ? gated_grad_any<__half, LORDBA_ACT_SILU>(g, T, s)
                                    : gated_grad_any<__half, LORDBA_ACT_GELU_TANH>(g, T, s);
}

int launch_repack(const void *src, int64_t ld_src, void *dst, int64_t ld_dst, int64_t rows, int64_t cols, cudaStream_t s)
{
    const EltGrid e = elementwise_grid(rows, (cols + 1) / 2);      // groups of 16 bytes
    return launch_kernel(repack_kernel, e.grid, kEltThreads, 0, s, static_cast<const uint8_t *>(src), ld_src,
                         static_cast<uint8_t *>(dst), ld_dst, rows, cols, e.width_log2);
}

}  // namespace lordba
