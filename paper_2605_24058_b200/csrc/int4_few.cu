// Products of a few tokens with 4-bit weights: the weights stream past the tokens once.
//
//   y[t,n] = sum over groups of  scale[n,g] * sum_{k in g} x[t,k] (u[n,k] - zero[n,g])
//
// Floor: HBM, half a byte a weight; what holds it off is below, at the kernel.  A CTA holds 16 or 32 weight rows, each of its four or eight warps every fourth or eighth block
// of 128 columns.  A lane's 16 bytes of a block are four runs of eight columns, 32 apart, so that the four lanes of a row and one word
// of each make 32 neighbouring columns: two matrix instructions (weights are the 16 rows, tokens the 8 columns), whose
// order of columns is the carrier's and needs no exchange, and never more than one group's.  The integers go in as they are
// (exact in 16 bits); a group's sum is scaled in float32.  The warps' sums meet in shared memory, in a fixed order.
//
// Measured, weights from HBM: one token 4096 x 4096 4.6 us, 4096 x 11008 9.4 us (23 MB: 2.5 TB/s), 16 tokens 6.5 and 13.8 us.
//
// Weights and activations come through a warp's own ring of asynchronous copies in shared memory: no barrier between warps,
// and many blocks on the way without a register.  Scales and zeros are few; the CTA's are laid into shared memory at the
// start (again every kChunk groups of a long row).
#include <atomic>
#include <cstring>
#include <type_traits>

#include "int4_common.cuh"
#include "product_internal.cuh"

namespace lordba {
namespace {

using namespace sm100;

struct FewArgs {
    const void *x;
    void *y;
    const uint8_t *q;
    const void *scale;
    const uint8_t *zero;
    int64_t d_in, d_out, ldx, ldy, ldq, ld_scale, ld_zero;
    int T, blocks, group_log2;
    uint32_t ones, middle;    // patterns of int4_pair: kInt4Ones, and the zero point 8
    int chunk;                // blocks whose scales are in shared memory at a time: a multiple of the warps
    int stride;               // of a row of scales there: odd, so that eight rows lie in eight banks
};

constexpr int kTokenBytes = 256 + 64;       // of a block's activations in a slot: two tokens, eight lanes, lie in different banks
__host__ __device__ constexpr int slot_of(int rows, int tokens) { return rows * 1024 + (tokens * kTokenBytes + 127) / 128 * 128; }

// Sixteen bytes from an aligned global address, of which the first `bytes` are read and the rest is zeros.
__device__ __forceinline__ void fetch_part(uint32_t to, const void *from, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}

// c += a b, or c = a b where FIRST
template <typename E, bool FIRST>
__device__ __forceinline__ void mma_16x8x16(float c[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (FIRST && std::is_same_v<E, __nv_bfloat16>)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
    else if constexpr (FIRST)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
    else if constexpr (std::is_same_v<E, __nv_bfloat16>)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t load_shared(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

// ROWS: tiles of 16 weight rows a CTA has.  TOK: tokens there is room for.  WARPS share the blocks, DEPTH slots each.  SPB:
// scales of a block and row, 1, 2 or 4.
//
// A block costs a warp 88 instructions for the integers of 16 rows (a pair a shift, a choice of bits, a subtraction), and should cost little
// more: whatever is the same for all blocks is worked out before, and slots are known when it is compiled.  No unit is full: one token
// through 4096 x 11008 issues in 58 % of the SMs' cycles, with the integer pipe at 47 % and DRAM at 23 %; warps wait for their copies, for one
// another's turn and for that pipe, in this order.  16 tokens and few rows (11008 -> 4096) leave eight warps an SM, which issue in 38 %
// of the cycles and wait for their copies.
template <typename E, int ROWS, int TOK, int WARPS, int DEPTH, int SPB, bool ZERO>
__global__ void __launch_bounds__(32 * WARPS)
int4_few_kernel(const __grid_constant__ FewArgs A)
{
    extern __shared__ __align__(128) uint8_t smem[];
    constexpr int kTileRows = 16 * ROWS, kThreads = 32 * WARPS, TILES = (TOK + 7) / 8, kSlot = slot_of(ROWS, TOK);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, r = lane / 4, t = lane % 4;
    const uint32_t ring = smem_addr(smem) + warp * DEPTH * kSlot;
    float *scales = reinterpret_cast<float *>(smem + WARPS * DEPTH * kSlot);
    uint32_t *zeros = reinterpret_cast<uint32_t *>(scales + kTileRows * A.stride);           // as patterns
    __shared__ __align__(16) uint8_t none[208];
    if (threadIdx.x < 52) reinterpret_cast<uint32_t *>(none)[threadIdx.x] = 0;       // in time for the first barrier
    const int64_t n0 = (int64_t)blockIdx.x * kTileRows;
    const int groups = (int)((A.d_in + (int64_t(1) << A.group_log2) - 1) >> A.group_log2);

    // what a lane fetches of each block: its pieces of 2 ROWS rows, and of the activations pieces lane + 32 i, sixteen a token
    constexpr int kShare = (TOK + 1) / 2;
    const uint8_t *q[2 * ROWS];
#pragma unroll
    for (int h = 0; h < 2 * ROWS; ++h) {
        const int64_t n = n0 + r + 8 * h < A.d_out ? n0 + r + 8 * h : A.d_out - 1;       // rows behind the last repeat it and are not written
        q[h] = A.q + n * A.ldq + 64 * warp + 16 * t;
    }
    const uint8_t *x[kShare];
    bool mine[kShare];
#pragma unroll
    for (int i = 0; i < kShare; ++i) {
        mine[i] = 2 * i + lane / 16 < A.T;
        x[i] = static_cast<const uint8_t *>(A.x) + (2 * i + lane / 16) * A.ldx * 2 + 256 * warp + 16 * (lane % 16);
    }
    const int left = (int)(2 * (A.d_in - 128 * (int64_t)(A.blocks - 1))) - 16 * (lane % 16);           // bytes of a token's row from its piece of
    const int tail = left < 0 ? 0 : left < 16 ? left : 16;                                             // the last block on, and of the piece
    const uint32_t weights_to = ring + 16 * lane, tokens_to = ring + 1024 * ROWS + kTokenBytes * (lane / 16) + 16 * (lane % 16);
    // block b, which lies `on` blocks of the warp's behind the pointers, into a slot
    auto fetch = [&](int b, int on, int slot) {
        if (b < A.blocks) {
#pragma unroll
            for (int h = 0; h < 2 * ROWS; ++h) fetch_part(weights_to + slot * kSlot + 512 * h, q[h] + 64 * WARPS * on, 16);
            const int bytes = b + 1 < A.blocks ? 16 : tail;
#pragma unroll
            for (int i = 0; i < kShare; ++i)
                if (mine[i]) fetch_part(tokens_to + slot * kSlot + 2 * kTokenBytes * i, x[i] + 256 * WARPS * on, bytes);
        }
        fetch_commit();                  // also where there is nothing left: the groups are counted
    };
    float acc[ROWS][TILES][4] = {};
    // of its token; a lane without one reads zeros
    const uint32_t weights_from = ring + 16 * lane;
    uint32_t tokens_from[TILES];
    int step[TILES];
#pragma unroll
    for (int k = 0; k < TILES; ++k) {
        const bool has = r + 8 * k < A.T;
        step[k] = has ? kSlot : 0;
        tokens_from[k] = has ? ring + 1024 * ROWS + kTokenBytes * (r + 8 * k) + 16 * t : smem_addr(none);
    }
    const uint32_t ones = A.ones, middle = A.middle;
    const int row_step = 32 * A.stride;                      // bytes from a row's scales to those of the row 8 on
    auto add = [&](int slot, uint32_t scale_at, uint32_t zero_at) {
        uint4 w[2 * ROWS];
#pragma unroll
        for (int h = 0; h < 2 * ROWS; ++h) w[h] = load_shared_v4(weights_from + slot * kSlot + 512 * h);
        float c[ROWS][TILES][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint4 v[TILES];
#pragma unroll
            for (int k = 0; k < TILES; ++k) v[k] = load_shared_v4(tokens_from[k] + 64 * j + slot * step[k]);
            constexpr int kWords = 4 / SPB;                    // of a block's share of a group
            const int i = j / kWords;
#pragma unroll
            for (int m = 0; m < ROWS; ++m) {
                uint32_t z[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) z[h] = ZERO ? load_shared(zero_at + (2 * m + h) * row_step + 4 * i) : middle;
                const uint4 &w0 = w[2 * m], &w1 = w[2 * m + 1];
                const uint32_t u0 = j == 0 ? w0.x : j == 1 ? w0.y : j == 2 ? w0.z : w0.w, u1 = j == 0 ? w1.x : j == 1 ? w1.y : j == 2 ? w1.z : w1.w;
#pragma unroll
                for (int p = 0; p < 4; p += 2) {
                    const uint32_t a0 = int4_pair<E>(u0, p, z[0], ones), a1 = int4_pair<E>(u1, p, z[1], ones), a2 = int4_pair<E>(u0, p + 1, z[0], ones),
                                   a3 = int4_pair<E>(u1, p + 1, z[1], ones);
#pragma unroll
                    for (int k = 0; k < TILES; ++k) {
                        if (p == 0 && j % kWords == 0) mma_16x8x16<E, true>(c[m][k], a0, a1, a2, a3, v[k].x, v[k].y);
                        else mma_16x8x16<E, false>(c[m][k], a0, a1, a2, a3, p ? v[k].z : v[k].x, p ? v[k].w : v[k].y);
                    }
                }
                if ((j + 1) % kWords == 0) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float s = __uint_as_float(load_shared(scale_at + (2 * m + h) * row_step + 4 * i));
#pragma unroll
                        for (int k = 0; k < TILES; ++k)
#pragma unroll
                            for (int e = 2 * h; e < 2 * h + 2; ++e) acc[m][k][e] = fmaf(s, c[m][k][e], acc[m][k][e]);
                    }
                }
            }
        }
    };
    grid_wait();
    grid_release();
#pragma unroll
    for (int d = 0; d < DEPTH - 1; ++d) fetch(warp + WARPS * d, d, d);
    for (int c0 = 0; c0 < A.blocks; c0 += A.chunk) {
        const int c1 = c0 + A.chunk < A.blocks ? c0 + A.chunk : A.blocks;
        const int g0 = (int)((128 * (int64_t)c0) >> A.group_log2);
        const int count = SPB == 1 ? (int)((128 * (int64_t)c1 - 1) >> A.group_log2) + 1 - g0 : SPB * (c1 - c0);
        if (c0 > 0) __syncthreads();                     // the scales' last readers
        // a warp lays out every WARPS-th row; of groups behind the last, in the last block, scale and product are zero
#pragma unroll 1
        for (int g = lane; g < count; g += 32)
#pragma unroll
            for (int i = 0; i < kTileRows / WARPS; ++i) {
                const int row = warp + WARPS * i;
                const int64_t n = n0 + row < A.d_out ? n0 + row : A.d_out - 1;
                const bool in = g0 + g < groups;
                const uint16_t s = in ? __ldg(static_cast<const uint16_t *>(A.scale) + n * A.ld_scale + g0 + g) : 0;
                scales[row * A.stride + g] = unpack2<E>(s).x;
                if (ZERO) zeros[row * A.stride + g] = int4_zero<E>(in ? __ldg(A.zero + n * A.ld_zero + g0 + g) & 15u : 8u);
            }
        __syncthreads();
        const uint32_t scale_row = smem_addr(scales + r * A.stride), zero_row = smem_addr(zeros + r * A.stride);
        for (int b0 = c0 + warp; b0 < c1; b0 += WARPS * DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                const int b = b0 + WARPS * d;
                if (b >= c1) break;
                fetch_wait(DEPTH - 2);
                __syncwarp();                            // the block is whole, and the slot before it has been read
                fetch(b + WARPS * (DEPTH - 1), d + DEPTH - 1, (d + DEPTH - 1) % DEPTH);
                const uint32_t g = 4 * (SPB == 1 ? (uint32_t)((128 * (int64_t)b) >> A.group_log2) - g0 : SPB * (b - c0));
                add(d, scale_row + g, zero_row + g);
            }
#pragma unroll
            for (int h = 0; h < 2 * ROWS; ++h) q[h] += 64 * WARPS * DEPTH;
#pragma unroll
            for (int i = 0; i < kShare; ++i) x[i] += 256 * WARPS * DEPTH;
        }
    }
    fetch_wait(0);
    __syncthreads();                                     // the ring becomes the place of the sums: [warp][token][row]
    float *sums = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int m = 0; m < ROWS; ++m)
#pragma unroll
        for (int k = 0; k < TILES; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (8 * k + 2 * t + e % 2 < A.T) sums[(warp * TOK + 8 * k + 2 * t + e % 2) * kTileRows + 16 * m + r + 8 * (e / 2)] = acc[m][k][e];
    __syncthreads();
    for (int i = threadIdx.x; i < A.T * kTileRows; i += kThreads) {
        const int token = i / kTileRows, row = i % kTileRows;
        if (n0 + row >= A.d_out) continue;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) v += sums[(w * TOK + token) * kTileRows + row];
        static_cast<E *>(A.y)[token * A.ldy + n0 + row] = from_float<E>(v);
    }
}

template <typename E, int ROWS, int TOK, int WARPS, int DEPTH, int SPB, bool ZERO>
int launch_few(FewArgs A, cudaStream_t stream)
{
    constexpr int kTileRows = 16 * ROWS, kChunk = 256 / ROWS, kMostSmem = 226 * 1024;      // kChunk: groups at a time
    const int64_t groups = (A.d_in + (int64_t(1) << A.group_log2) - 1) >> A.group_log2;
    A.chunk = kChunk / SPB / (WARPS * DEPTH) * (WARPS * DEPTH);
    const int64_t most = SPB == 1 ? groups : SPB * (int64_t)A.blocks;
    A.stride = (int)(most < kChunk ? most : kChunk) | 1;
    const int smem = WARPS * DEPTH * slot_of(ROWS, TOK) + kTileRows * A.stride * (ZERO ? 8 : 4);
    static_assert(WARPS * TOK * kTileRows * 4 <= WARPS * DEPTH * slot_of(ROWS, TOK), "the sums have room in the ring");
    static_assert(WARPS * DEPTH * slot_of(ROWS, TOK) + kTileRows * (kChunk + 1) * 8 <= kMostSmem, "shared memory");
    static_assert(kChunk / SPB >= WARPS * DEPTH, "a chunk goes round the ring");
    const auto kernel = int4_few_kernel<E, ROWS, TOK, WARPS, DEPTH, SPB, ZERO>;
    A.ones = kInt4Ones<E>;
    A.middle = int4_zero<E>(8u);
    // said once a device: the call takes as long as a launch
    static std::atomic<uint64_t> said{0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return LORDBA_ECUDA;
    const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
    if (!(said.load(std::memory_order_relaxed) & bit)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem) != cudaSuccess) {
            cudaGetLastError();
            return LORDBA_ECUDA;
        }
        said.fetch_or(bit, std::memory_order_relaxed);
    }
    return launch_kernel(kernel, dim3((unsigned)((A.d_out + kTileRows - 1) / kTileRows), 1, 1), 32 * WARPS, smem, stream, A);
}

template <typename E, int ROWS, int TOK, int WARPS, int DEPTH>
int launch_grouped(const FewArgs &A, cudaStream_t stream)
{
    if (A.group_log2 >= 7) return A.zero ? launch_few<E, ROWS, TOK, WARPS, DEPTH, 1, true>(A, stream) : launch_few<E, ROWS, TOK, WARPS, DEPTH, 1, false>(A, stream);
    if (A.group_log2 == 6) return A.zero ? launch_few<E, ROWS, TOK, WARPS, DEPTH, 2, true>(A, stream) : launch_few<E, ROWS, TOK, WARPS, DEPTH, 2, false>(A, stream);
    return A.zero ? launch_few<E, ROWS, TOK, WARPS, DEPTH, 4, true>(A, stream) : launch_few<E, ROWS, TOK, WARPS, DEPTH, 4, false>(A, stream);
}

template <typename E>
int launch_typed(const FewArgs &A, cudaStream_t stream)
{
    // More tokens, more weight rows a CTA: its activations come from L2 once for all of them.  Where the CTAs are one to an SM, each
    // wants more warps and more on the way; where there are more, two that share an SM do better (11008 x 4096 and 4096 x 11008, of
    // 128 and 344 CTAs: 16 tokens with eight warps 11.9 and 16.6 us, with four 12.9 and 13.9; 8 tokens with three slots a warp 9.9 and,
    // groups of 64 with zeros, 15.6 us, with two 11.5 and 12.3; 4 tokens with eight warps 9.2 and 17.2 us, groups of 32, with four 10.2 and 10.8; 32
    // tokens with eight warps 17.6 and 23.7 us, with four 20.2 and 19.3, widened for the tensor core's own tiles 22.4 and 19.6).
    if (A.T == 1) return launch_grouped<E, 1, 1, 8, 3>(A, stream);
    const bool alone = (A.d_out + 31) / 32 <= sm_count();
    if (A.T <= 4) return alone ? launch_grouped<E, 2, 4, 8, 4>(A, stream) : launch_grouped<E, 2, 4, 4, 4>(A, stream);
    if (A.T <= 8) return alone ? launch_grouped<E, 2, 8, 8, 3>(A, stream) : launch_grouped<E, 2, 8, 8, 2>(A, stream);
    if (A.T > 16) return alone ? launch_grouped<E, 2, 32, 8, 2>(A, stream) : launch_grouped<E, 2, 32, 4, 2>(A, stream);
    return alone ? launch_grouped<E, 2, 16, 8, 3>(A, stream) : launch_grouped<E, 2, 16, 4, 3>(A, stream);
}

}  // namespace

// x: rows on 16-byte boundaries.
int launch_int4_few(const lordba_int4_proj &p, int64_t T, int dtype, cudaStream_t stream)
{
    FewArgs A;
    std::memset(&A, 0, sizeof(A));
    A.x = p.in; A.y = p.out; A.q = p.q; A.scale = p.scale; A.zero = p.zero;
    A.d_in = p.d_in; A.d_out = p.d_out; A.ldx = p.ld_in; A.ldy = p.ld_out; A.ldq = p.ldq; A.ld_scale = p.ld_scale; A.ld_zero = p.ld_zero;
    A.T = (int)T;
    A.blocks = (int)((p.d_in + 127) / 128);
    while ((int64_t(1) << A.group_log2) < p.group) ++A.group_log2;
    return dtype == LORDBA_BF16 ? launch_typed<__nv_bfloat16>(A, stream) : launch_typed<__half>(A, stream);
}

}  // namespace lordba
