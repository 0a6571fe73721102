// The streaming kernels next to the adapters: per-token quantisation to 8 bits, dropout from a
// counter-based generator, the elementwise part of the gated block's backward pass, and the copy that
// gives an operand a pitch the copy engine can take.
//
// All of them are bound by HBM: each element is read once and written once, eight elements (16 bytes of a
// 16-bit type) an access.  Rows whose base or pitch is not a multiple of 16 bytes are read as the aligned
// pieces that hold them.
#include "block_common.cuh"

namespace lordba {
namespace {

constexpr int kEltThreads = 256;

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

// ---- lordba_int8_quantize_rows ----------------------------------------------------------------------
// The largest |x| is looked for among bit patterns, which order like the numbers with NaN above infinity;
// 16-bit types two at a time.
template <typename E>
__device__ __forceinline__ uint32_t top_of(const Group8<E> &h, uint32_t top)
{
    if constexpr (sizeof(E) == 2) {
        top = __vmaxu2(__vmaxu2(top, h.w.x & 0x7fff7fffu), h.w.y & 0x7fff7fffu);
        return __vmaxu2(__vmaxu2(top, h.w.z & 0x7fff7fffu), h.w.w & 0x7fff7fffu);
    } else {
        const uint32_t w[8] = {h.w.x, h.w.y, h.w.z, h.w.w, h.w2.x, h.w2.y, h.w2.z, h.w2.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, w[j] & 0x7fffffffu);
        return top;
    }
}

// four values, rounded to whole numbers (ties to even) and packed: of v + 1.5 * 2^23 the low byte is v's whole
// number, and the sum and three permutes take fewer cycles than four conversions.  |v| stays below 128.
__device__ __forceinline__ uint32_t pack_whole(float v0, float v1, float v2, float v3)
{
    const float m = 12582912.0f;
    const uint32_t lo = __byte_perm(__float_as_uint(__fadd_rn(v0, m)), __float_as_uint(__fadd_rn(v1, m)), 0x0040);
    const uint32_t hi = __byte_perm(__float_as_uint(__fadd_rn(v2, m)), __float_as_uint(__fadd_rn(v3, m)), 0x0040);
    return __byte_perm(lo, hi, 0x5410);
}

// TPR threads hold a row: its groups of eight stay in registers between the search for the maximum and
// the rounding (NV groups a thread; what a longer row has beyond them is read again, from L2).
//
// Measured (bf16): 8192 x 11008 41 us, 6.6 TB/s, the copy rate; 8192 x 4096 18 us, 2048 x 4096 5.5 us, 5.6 and
// 4.6 TB/s.  A row's block waits twice, for its loads and for the maximum, so what counts is how many blocks an
// SM holds (with eight, registers held to 32, 8192 x 4096 takes 18 us instead of 19.5; with masked accesses and
// conversions one by one it took 23).  Blocks that walk rows and load the next one early took 23 us.
template <typename E, int TPR, int NV, bool FULL>
__global__ void __launch_bounds__(kEltThreads, sizeof(E) == 4 ? 4 : FULL && NV == 2 ? 8 : 5)
quantize_rows_kernel(const E *__restrict__ x, int64_t ldx, int vec, int8_t *__restrict__ q, int64_t ldq, int qvec,
                     float *__restrict__ scale, int64_t T, int64_t d)
{
    constexpr int kRows = kEltThreads / TPR, kWarps = kEltThreads / 32;
    __shared__ uint32_t part[kWarps];
    const int tid = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR, groups = (d + 7) / 8;
    grid_wait();
    grid_release();
    if (TPR == 32 && row >= T) return;          // whole warps; with TPR = 256 every block has its row
    const E *xr = x + row * ldx;
    Group8<E> held[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t g = tid + (int64_t)i * TPR;
        if (g < groups) held[i] = load_either<FULL>(xr, g, d, vec);
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (tid + (int64_t)i * TPR < groups) top = top_of(held[i], top);
    for (int64_t g = tid + (int64_t)NV * TPR; g < groups; g += TPR) top = top_of(load_either<FULL>(xr, g, d, vec), top);
    if constexpr (sizeof(E) == 2) top = max(top & 0xffffu, top >> 16);
    top = __reduce_max_sync(0xffffffffu, top);
    if (TPR > 32) {
        if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = top;
        __syncthreads();
        top = __reduce_max_sync(0xffffffffu, part[threadIdx.x % kWarps]);
    }
    float amax;
    if constexpr (sizeof(E) == 2) amax = unpack2<E>(top).x;
    else amax = __uint_as_float(top);
    const bool finite = amax < INFINITY;                // not for NaN either
    const bool live = finite && amax >= 0x1p-120f;      // below it 127 / amax could overflow
    const float inverse = live ? 127.0f / amax : 0.0f;
    if (tid == 0) scale[row] = finite ? (live ? amax / 127.0f : 0.0f) : __uint_as_float(0x7fc00000u);
    int8_t *qr = q + row * ldq;
    auto put = [&](int64_t g, const Group8<E> &h) {
        float v[8];
        unpack_group<E>(h, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __fmul_rn(v[j], inverse);
        uint2 b = make_uint2(pack_whole(v[0], v[1], v[2], v[3]), pack_whole(v[4], v[5], v[6], v[7]));
        if (!live) b = make_uint2(0, 0);
        if (FULL || (qvec && 8 * g + 8 <= d)) {
            *reinterpret_cast<uint2 *>(qr + 8 * g) = b;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (8 * g + j < d) qr[8 * g + j] = (int8_t)((j < 4 ? b.x : b.y) >> 8 * (j % 4));
        }
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t g = tid + (int64_t)i * TPR;
        if (g < groups) put(g, held[i]);
    }
    for (int64_t g = tid + (int64_t)NV * TPR; g < groups; g += TPR) put(g, load_either<FULL>(xr, g, d, vec));
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
    // a few rounds of resident blocks are enough; the rows beyond are a loop
    const int64_t most = gx >= 148 * 32 ? 1 : 148 * 32 / gx;
    if (gy > most) gy = most;
    if (gy > 65535) gy = 65535;
    EltGrid e;
    e.width_log2 = best;
    e.grid = dim3((unsigned)gx, (unsigned)gy, 1);
    return e;
}

// ---- lordba_dropout -----------------------------------------------------------------------------------
// Philox4x32-10: ten rounds of two 32 x 32 -> 64 bit products; the multipliers and the key increments are
// the published ones.  The rounds' keys are the same for every element: the host lays them out, the kernel
// reads them as constants.
struct PhiloxKeys {
    uint32_t k[10][2];
};

PhiloxKeys philox_keys(uint64_t seed)
{
    PhiloxKeys p;
    for (uint32_t i = 0; i < 10; ++i) {
        p.k[i][0] = (uint32_t)seed + i * 0x9E3779B9u;
        p.k[i][1] = (uint32_t)(seed >> 32) + i * 0xBB67AE85u;
    }
    return p;
}

__device__ __forceinline__ uint4 philox(uint4 c, const PhiloxKeys &keys)
{
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)c.x * 0xD2511F53u, b = (uint64_t)c.z * 0xCD9E8D57u;
        c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ keys.k[i][0], (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ keys.k[i][1], (uint32_t)a);
    }
    return c;
}

struct Vec3 { int a, b, c; };      // which matrices allow 16-byte accesses

// out may be x or residual: a thread writes only elements that it alone has read before.
// Measured (8192 x 11008 bf16 with residual, 541 MB): 82 us, 6.58 TB/s, the copy rate.  The generator's 60
// instructions per eight elements fit beside the loads only with its keys out of the registers: kept there (20
// words a thread) the same call took 127 us, and two or four rows a thread at a time 91 and 97 us.
template <typename E, bool RESIDUAL, bool FULL>
__global__ void __launch_bounds__(kEltThreads, FULL ? 5 : 4)
dropout_kernel(const E *x, int64_t ldx, const E *residual, int64_t ldr, E *out, int64_t ldo, int64_t T, int64_t d,
               uint32_t cut, float scale, const __grid_constant__ PhiloxKeys keys, uint64_t offset, int width_log2, Vec3 vec)
{
    const int64_t g = ((int64_t)blockIdx.x << width_log2) + (threadIdx.x & ((1 << width_log2) - 1));
    const int64_t height = kEltThreads >> width_log2;
    grid_wait();
    grid_release();
    if (8 * g >= d) return;
    for (int64_t t = blockIdx.y * height + (threadIdx.x >> width_log2); t < T; t += gridDim.y * height) {
        float v[8], r[8];
        unpack_group<E>(load_either<FULL>(x + t * ldx, g, d, vec.a), v);
        if (RESIDUAL) unpack_group<E>(load_either<FULL>(residual + t * ldr, g, d, vec.b), r);
        const uint4 bits = philox(make_uint4((uint32_t)g, (uint32_t)t, (uint32_t)offset, (uint32_t)(offset >> 32)), keys);
        const uint32_t w[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t number = (i & 1) ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
            const float kept = number >= cut ? v[i] * scale : 0.0f;      // a choice, not a product with 0: x may be inf
            v[i] = RESIDUAL ? kept + r[i] : kept;
        }
        store_either<FULL>(out + t * ldo, g, d, vec.c, v);
    }
}

// v, made what rounding to E took from it; nothing where the rounded value is not finite
template <typename E>
__device__ __forceinline__ float *rest_of(float v[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float r = v[i] - to_float(from_float<E>(v[i]));
        v[i] = fabsf(r) < INFINITY ? r : 0.0f;
    }
    return v;
}

// ---- dgate = dh up act'(gate), dup = dh act(gate) ---------------------------------------------------------
// Measured (2048 x 11008 bf16, 225 MB): 35 us, 6.4 TB/s.
template <typename E, int ACT, bool FULL>
__global__ void __launch_bounds__(kEltThreads, FULL ? 4 : 3)
gated_grad_kernel(const E *__restrict__ dh, int64_t ld_dh, const E *__restrict__ gate, const E *__restrict__ up,
                  int64_t ld_pre, E *__restrict__ dgate, E *__restrict__ dup, int64_t ld_dpre, E *__restrict__ lo_gate,
                  E *__restrict__ lo_up, int64_t ld_lo, int64_t T, int64_t d, int width_log2, Vec3 vec)
{
    const int64_t g = ((int64_t)blockIdx.x << width_log2) + (threadIdx.x & ((1 << width_log2) - 1));
    const int64_t height = kEltThreads >> width_log2;
    grid_wait();
    grid_release();
    if (8 * g >= d) return;
    for (int64_t t = blockIdx.y * height + (threadIdx.x >> width_log2); t < T; t += gridDim.y * height) {
        float vh[8], vg[8], vu[8];
        unpack_group<E>(load_either<FULL>(dh + t * ld_dh, g, d, vec.a), vh);
        unpack_group<E>(load_either<FULL>(gate + t * ld_pre, g, d, vec.b), vg);
        unpack_group<E>(load_either<FULL>(up + t * ld_pre, g, d, vec.b), vu);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float value, slope;
            act_and_slope<ACT>(vg[i], value, slope);
            vu[i] *= vh[i] * slope;
            vh[i] *= value;
        }
        store_either<FULL>(dgate + t * ld_dpre, g, d, vec.c, vu);
        store_either<FULL>(dup + t * ld_dpre, g, d, vec.c, vh);
        if (lo_gate) {
            store_either<FULL>(lo_gate + t * ld_lo, g, d, true, rest_of<E>(vu));
            store_either<FULL>(lo_up + t * ld_lo, g, d, true, rest_of<E>(vh));
        }
    }
}

// ---- repack ---------------------------------------------------------------------------------------------
// Up to four matrices a launch, one a grid layer; a thread writes 16 aligned bytes.
__global__ void __launch_bounds__(kEltThreads)
repack_kernel(const __grid_constant__ RepackList list, int width_log2)
{
    const RepackList::Item &m = list.item[blockIdx.z];
    const int64_t g = ((int64_t)blockIdx.x << width_log2) + (threadIdx.x & ((1 << width_log2) - 1));
    const int64_t height = kEltThreads >> width_log2;
    grid_wait();
    grid_release();
    if (16 * g >= m.cols) return;
    const uint8_t *src = static_cast<const uint8_t *>(m.src);
    uint8_t *dst = static_cast<uint8_t *>(m.dst);
    for (int64_t t = blockIdx.y * height + (threadIdx.x >> width_log2); t < m.rows; t += gridDim.y * height) {
        const uintptr_t row = reinterpret_cast<uintptr_t>(src + t * m.ld_src);
        *reinterpret_cast<uint4 *>(dst + t * m.ld_dst + 16 * g) = load_bytes16(row + 16 * g, row + m.cols);
    }
}

// whether rows can be accessed eight elements at a time
bool vec_ok(const void *p, int64_t ld, size_t e) { return aligned(p, 16) && ((size_t)ld * e) % 16 == 0; }

template <typename E, bool FULL>
int quantize_full(const E *x, int64_t ldx, int vec, int8_t *q, int64_t ldq, int qvec, float *scale, int64_t T, int64_t d, cudaStream_t s)
{
    // up to 1024 columns a warp holds a row (32 lanes x 4 groups of 8), beyond that a block (256 x NV x 8)
    const bool warps = d <= 1024;
    const auto kernel = warps ? quantize_rows_kernel<E, 32, 4, FULL>
                              : d <= 4096 ? quantize_rows_kernel<E, 256, 2, FULL> : quantize_rows_kernel<E, 256, 6, FULL>;
    return launch_kernel(kernel, dim3((unsigned)(warps ? (T + 7) / 8 : T)), kEltThreads, 0, s, x, ldx, vec, q, ldq, qvec, scale, T, d);
}

template <typename E>
int quantize_any(const void *x, int64_t ldx, int8_t *q, int64_t ldq, float *scale, int64_t T, int64_t d, cudaStream_t s)
{
    const int vec = vec_ok(x, ldx, sizeof(E)), qvec = aligned(q, 8) && ldq % 8 == 0;
    const E *xe = static_cast<const E *>(x);
    if (vec && qvec && d % 8 == 0) return quantize_full<E, true>(xe, ldx, vec, q, ldq, qvec, scale, T, d, s);
    return quantize_full<E, false>(xe, ldx, vec, q, ldq, qvec, scale, T, d, s);
}

template <typename E>
int dropout_any(const void *x, int64_t ldx, const void *r, int64_t ldr, void *out, int64_t ldo, int64_t T, int64_t d, int cut,
                uint64_t seed, uint64_t offset, cudaStream_t s)
{
    const EltGrid e = elementwise_grid(T, d);
    const float scale = cut < 65536 ? 65536.0f / (float)(65536 - cut) : 0.0f;
    const Vec3 vec{vec_ok(x, ldx, sizeof(E)), vec_ok(r, ldr, sizeof(E)), vec_ok(out, ldo, sizeof(E))};
    const bool full = vec.a && (!r || vec.b) && vec.c && d % 8 == 0;
    const auto kernel = full ? (r ? dropout_kernel<E, true, true> : dropout_kernel<E, false, true>)
                             : (r ? dropout_kernel<E, true, false> : dropout_kernel<E, false, false>);
    return launch_kernel(kernel, e.grid, kEltThreads, 0, s, static_cast<const E *>(x),
                         ldx, static_cast<const E *>(r), ldr, static_cast<E *>(out), ldo, T, d, (uint32_t)cut, scale, philox_keys(seed),
                         offset, e.width_log2, vec);
}

template <typename E, int ACT>
int gated_grad_any(const lordba_gated_grad &g, int64_t T, void *lo_gate, void *lo_up, int64_t ld_lo, cudaStream_t s)
{
    const EltGrid e = elementwise_grid(T, g.d_hidden);
    const Vec3 vec{vec_ok(g.dh, g.ld_dh, 2), vec_ok(g.gate, g.ld_pre, 2) && aligned(g.up, 16),
                   vec_ok(g.dgate, g.ld_dpre, 2) && aligned(g.dup, 16)};
    const bool full = vec.a && vec.b && vec.c && g.d_hidden % 8 == 0;
    return launch_kernel(full ? gated_grad_kernel<E, ACT, true> : gated_grad_kernel<E, ACT, false>, e.grid, kEltThreads, 0, s, static_cast<const E *>(g.dh), g.ld_dh,
                         static_cast<const E *>(g.gate), static_cast<const E *>(g.up), g.ld_pre, static_cast<E *>(g.dgate),
                         static_cast<E *>(g.dup), g.ld_dpre, static_cast<E *>(lo_gate), static_cast<E *>(lo_up), ld_lo, T,
                         g.d_hidden, e.width_log2, vec);
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

int launch_gated_grad(const lordba_gated_grad &g, int64_t T, int dtype, void *lo_gate, void *lo_up, int64_t ld_lo, cudaStream_t s)
{
    if (dtype == LORDBA_BF16)
        return g.act == LORDBA_ACT_SILU ? gated_grad_any<__nv_bfloat16, LORDBA_ACT_SILU>(g, T, lo_gate, lo_up, ld_lo, s)
                                        : gated_grad_any<__nv_bfloat16, LORDBA_ACT_GELU_TANH>(g, T, lo_gate, lo_up, ld_lo, s);
    return g.act == LORDBA_ACT_SILU ? gated_grad_any<__half, LORDBA_ACT_SILU>(g, T, lo_gate, lo_up, ld_lo, s)
                                    : gated_grad_any<__half, LORDBA_ACT_GELU_TANH>(g, T, lo_gate, lo_up, ld_lo, s);
}

int launch_repack(const RepackList &list, cudaStream_t s)
{
    if (list.n == 0) return LORDBA_OK;
    int64_t rows = 0, cols = 0;
    for (int i = 0; i < list.n; ++i) {
        rows = rows > list.item[i].rows ? rows : list.item[i].rows;
        cols = cols > list.item[i].cols ? cols : list.item[i].cols;
    }
    EltGrid e = elementwise_grid(rows, (cols + 1) / 2);      // groups of 16 bytes
    e.grid.z = (unsigned)list.n;
    return launch_kernel(repack_kernel, e.grid, kEltThreads, 0, s, list, e.width_log2);
}

}  // namespace lordba
