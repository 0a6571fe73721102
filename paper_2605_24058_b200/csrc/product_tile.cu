// The product kernel for many rows: 256 x 256 outputs a CTA pair on tcgen05 (cta_group::2), persistent.
//
//   D[m,n] = sum_k A[m,k] B[n,k]; 16-bit operands with sums in float32, int8 with sums in int32.
//
// Bound: the tensor core.  A pair's two SMs each hold 128 rows of A and 128 of the 256 rows of B (of the
// gated form: one the gate's, the other up's 128 rows, so that g and u of the same outputs land in the
// same thread), 128 bytes of the contraction a stage: 32 KB of loads per 128 x 256 x 64 products (16-bit),
// half of what two lone SMs would load, in a ring of six stages.  An accumulator is 256 of the 512 TMEM
// columns: while the epilogue drains one, the next tile is summed into the other.
//
//   warp 0      copies: both CTAs' producers fill their own halves; every copy completes on the leader's barrier
//   warp 1      the leader's issues all MMAs (one thread) and frees stages and accumulators in both CTAs
//   warps 4-11  epilogue, 32 columns of 32 rows at a time, addends fetched a step ahead.  It is a chain of
//               latencies, so two groups of four warps take turns at the tiles, one computing while the other
//               waits; where every pair has but one tile they share it.
//
// Measured, in short bursts and, second, sustained under the power cap: 8-bit 8192 x 11008 -> 4096 230 and 275 us
// (3.2 and 2.7 Pop/s); gated 2048 x 4096 -> 11008 in bf16 246 and 289 us (1.50 and 1.28 PFLOP/s), with addends and saved
// pre-activations 286 and 333 us.  A library product of the same size, without gate, takes 239 and 282 us, with an addend
// 269 and 313 us.  Gradients of the same block: dx 249 and 294 us, both dW 261 and 307 us (library 239 and 276, 246 and
// 286).  What is left is the loads: 3.1 - 3.7 GB from L2 a product, 13 TB/s, and at 1.4 GHz their power.
// Sixteen epilogue warps, or 16 columns a step, cost such products 2 - 6 % and gain 5 - 20 % only where the
// contraction is so short that the epilogue is all there is.
//
// Operands come contraction-contiguous or (gradients) m- or n-contiguous: then a stage holds 64 contraction
// steps as rows of 64 columns and the MMA reads it transposed.
#include <cstring>
#include <mutex>

#include "product_internal.cuh"

namespace lordba {
namespace {

using namespace sm100;

constexpr int kStages = 6;
constexpr int kHalf = 128 * 128;                   // bytes of one CTA's half of an operand in a stage
constexpr int kStageBytes = 2 * kHalf;
constexpr int kTileM = 256;
constexpr int kEpiWarps = 8;
constexpr int kTileThreads = (4 + kEpiWarps) * 32;
constexpr int kBarBytes = (2 * kStages + 4) * 8 + 16;
constexpr int kCh = 32;                            // columns of an epilogue step
constexpr int kPatchBytes = 32 * 64;               // 32 rows of 64 bytes on their way to memory; two for each warp
constexpr int kTileSmem = kStages * kStageBytes + 2 * kEpiWarps * kPatchBytes + kBarBytes + 1024;

struct TileArgs {
    CUtensorMap a[4], b[2];      // of two problems, the second one's A (and rest of A) are a[1] (and a[3])
    CUtensorMap out[2], pre[2];  // where rows start on 16-byte boundaries
    Finish f;
    int k_blocks;          // stages per operand pair
    int parts;             // operand pairs summed into one accumulator
    int tiles_m, tiles_n, tiles, problems;
    int skip;              // -1; the test-hooks build can name a stage whose copies are left out
    int *status;
    uint32_t idesc;
};

// Tiles in groups of eight rows of tiles (2048 rows), m fastest: the pairs at work share a few columns of
// tiles of B and the group's rows of A, which L2 holds, and B is read from HBM once a group.
struct Tile { int m, n, problem; };
__device__ __forceinline__ Tile tile_at(const TileArgs &P, int i)
{
    const int per = P.tiles_m * P.tiles_n;
    Tile t;
    t.problem = P.problems > 1 ? i / per : 0;
    i -= t.problem * per;
    const int group = i / (8 * P.tiles_n), first = group * 8;
    const int rows = P.tiles_m - first < 8 ? P.tiles_m - first : 8;
    i -= group * 8 * P.tiles_n;
    t.n = i / rows;
    t.m = first + i - t.n * rows;
    return t;
}

// ---- epilogue: a warp's 32 rows x 64 bytes of a matrix -----------------------------------------------------------
// TMEM gives a lane a row.  A lane reads the addends of its row itself; results go through a patch of shared memory,
// from which the copy engine writes them (64-byte swizzled: the lanes' rows do not meet in a bank).  Rows that
// it cannot take are written element by element.  What is rare stays out of line: where a CTA has one tile,
// fetching instructions is a good part of its time.
__device__ __noinline__ uint4 fetch_part(const uint8_t *q, int64_t left)
{
    return left > 0 ? load_bytes16<false>(reinterpret_cast<uintptr_t>(q), reinterpret_cast<uintptr_t>(q) + 2 * left) : make_uint4(0, 0, 0, 0);
}

// 32 columns of 16 bits, `left` of which exist
__device__ __forceinline__ void fetch(uint4 x[4], const uint8_t *q, int vec, int64_t left)
{
    if (vec && left >= 32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const uint4 *>(q + 16 * i);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = fetch_part(q + 16 * i, left - 8 * i);
    }
}

__device__ __forceinline__ void add(const uint4 x[4], float v[32], int dtype)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 f = unpack2_any(w[j], dtype);
            v[8 * i + 2 * j] += f.x;
            v[8 * i + 2 * j + 1] += f.y;
        }
    }
}

__device__ __forceinline__ uint32_t patch_piece(uint32_t patch, int row, int i) { return patch + 64 * row + 16 * (i ^ (row >> 1 & 3)); }

// rows x left elements of e bytes from a patch to q (row pitch ld bytes), whatever the alignment
__device__ __noinline__ void put_elements(uint32_t patch, uint8_t *q, int64_t ld, int rows, int64_t left, int e)
{
    const int lane = threadIdx.x % 32, per = 64 / e;
    const int n = left < per ? (int)left : per;
#pragma unroll 1
    for (int i = lane; i < rows * per; i += 32) {
        const int r = i / per, c = i % per;
        if (c >= n) continue;
        const uint32_t at = patch_piece(patch, r, c * e / 16) + c * e % 16;
        if (e == 4) {
            uint32_t v;
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
            reinterpret_cast<uint32_t *>(q + r * ld)[c] = v;
        } else {
            uint16_t v;
            asm volatile("ld.shared.b16 %0, [%1];" : "=h"(v) : "r"(at) : "memory");
            reinterpret_cast<uint16_t *>(q + r * ld)[c] = v;
        }
    }
}

// the first n elements of a piece to q
__device__ __noinline__ void put_tail(uint4 x, uint8_t *q, int n, int e)
{
    uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll 1
    for (int j = 0; j < n; ++j) {
        if (e == 4) {
            reinterpret_cast<uint32_t *>(q)[j] = w[0];
            w[0] = w[1]; w[1] = w[2];
        } else {
            reinterpret_cast<uint16_t *>(q)[j] = (uint16_t)w[0];
            w[0] = __funnelshift_r(w[0], w[1], 16);
            w[1] = __funnelshift_r(w[1], w[2], 16);
            w[2] = __funnelshift_r(w[2], w[3], 16);
            w[3] >>= 16;
        }
    }
}

// A matrix that results go to.
struct Target {
    const CUtensorMap *map;
    void *p;
    int64_t ld;
    int vec, e;
};

struct Patches {
    uint32_t base;
    int which = 0;

    // sixteen words of the lane's row m0 + lane, from column n on.  Every call makes one group of stores, also an empty
    // one, because the wait that frees a patch counts groups: all but the latest is the patch's own and older ones.
    __device__ __forceinline__ void put(const uint32_t w[16], const Target &t, int64_t m0, int64_t n, int rows, int64_t left, int lane)
    {
        const uint32_t patch = base + which * kPatchBytes;
        which ^= 1;
        if (lane == 0) stores_read_but_one();          // what went out of this patch has left it
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) store_shared_v4(patch_piece(patch, lane, i), make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
        fence_proxy_async();
        __syncwarp();
        if (t.vec) {
            // the copy engine writes whole 16-byte pieces, so its map ends with the last of them; what the row has
            // beyond it goes by hand
            const int piece = 16 / t.e, tail = left < 64 / t.e ? (int)left % piece : 0;
            if (lane == 0 && left >= piece) store_tile(t.map, patch, (int)n, (int)m0);
            if (tail && lane < rows)
                put_tail(load_shared_v4(patch_piece(patch, lane, (int)left / piece)),
                         static_cast<uint8_t *>(t.p) + ((m0 + lane) * t.ld + n + left - tail) * t.e, tail, t.e);
        } else {
            put_elements(patch, static_cast<uint8_t *>(t.p) + (m0 * t.ld + n) * t.e, t.ld * t.e, rows, left, t.e);
            __syncwarp();
        }
        if (lane == 0) stores_commit();
    }
    // 32 values, in the target's type
    __device__ __forceinline__ void put32(const float v[32], const Target &t, int64_t m0, int64_t n, int rows, int64_t left, int lane, int dtype)
    {
        uint32_t w[16];
        if (t.e == 4) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (left <= 16 * h) break;
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(v[16 * h + i]);
                put(w, t, m0, n + 16 * h, rows, left - 16 * h, lane);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = pack2_any(v[2 * i], v[2 * i + 1], dtype);
            put(w, t, m0, n, rows, left, lane);
        }
    }
};

// DT: type of the outputs and addends (known here: with a choice at each element the epilogue takes a third more
// instructions).
template <bool INT8, bool GATED, bool A_MN, bool B_MN, int DT>
__global__ void __launch_bounds__(kTileThreads, 1)
product_tile_kernel(const __grid_constant__ TileArgs P)
{
    extern __shared__ uint8_t smem_raw[];
    constexpr int kTileN = GATED ? 128 : 256;        // columns of the output
    constexpr int kBlockK = INT8 ? 128 : 64;
    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const uint32_t patches = base + kStages * kStageBytes, bars = patches + 2 * kEpiWarps * kPatchBytes;
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (kStages + s); };
    auto sum_full = [&](int b) { return bars + 8u * (2 * kStages + b); };
    auto sum_empty = [&](int b) { return bars + 8u * (2 * kStages + 2 + b); };
    uint8_t *misc = smem_raw + (bars - smem_addr(smem_raw)) + (2 * kStages + 4) * 8;
    volatile uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(misc);
    volatile int *abort_flag = reinterpret_cast<int *>(misc + 4);
    const Bounded bound{abort_flag, P.status};

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = cluster_rank();
    const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;
    const int blocks = P.k_blocks * P.parts;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            bar_init(full(s), 1);
            bar_init(empty(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            bar_init(sum_full(b), 1);
            bar_init(sum_empty(b), kEpiWarps);       // the group's warps in both CTAs
        }
        *abort_flag = 0;
        bar_init_fence();
    }
    if (warp == 1) tmem_alloc<2>(smem_addr(misc), 512);
    if (warp == 2 && lane == 0) {
        prefetch_map(&P.a[0]);
        prefetch_map(&P.b[GATED ? rank : 0]);
    }
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    const uint32_t tmem = *tmem_slot;
    grid_wait();
    grid_release();

    if (warp == 0) {
        if (lane == 0) {
            Ring r;
            bool alive = true;
            int count = 0;
            for (int i = pair; i < P.tiles; i += pairs) {
                const Tile t = tile_at(P, i);
                const int m0 = t.m * kTileM + 128 * rank;
                const int n0 = t.n * kTileN + (GATED ? 0 : 128 * (int)rank);
                for (int kb = 0; kb < blocks; ++kb, ++count) {
                    alive = alive && bound.wait(empty(r.stage), r.phase ^ 1u, kDevTmaWaitTimeout);
                    if (!alive) break;
                    if (rank == 0) bar_expect(full(r.stage), 2 * kStageBytes);
                    if (count != P.skip) {
                        const int part = kb >= P.k_blocks ? 1 : 0;
                        const int k0 = (kb - part * P.k_blocks) * kBlockK;
                        const CUtensorMap *ma = &P.a[P.problems > 1 ? t.problem + 2 * part : part];
                        const CUtensorMap *mb = &P.b[GATED ? (int)rank : P.problems > 1 ? 0 : part];
                        const uint32_t sa = base + r.stage * kStageBytes, sb = sa + kHalf;
                        const uint32_t bar = peer_addr(full(r.stage), 0);
                        if (A_MN) {
                            load_tile_pair(sa, ma, m0, k0, bar);
                            load_tile_pair(sa + kHalf / 2, ma, m0 + 64, k0, bar);
                        } else {
                            load_tile_pair(sa, ma, k0, m0, bar);
                        }
                        if (B_MN) {
                            load_tile_pair(sb, mb, n0, k0, bar);
                            load_tile_pair(sb + kHalf / 2, mb, n0 + 64, k0, bar);
                        } else {
                            load_tile_pair(sb, mb, k0, n0, bar);
                        }
                    }
                    r.next(kStages);
                }
                if (!alive) break;
            }
            // the MMAs' last arrivals on this CTA's barriers come before it leaves
            for (int s = 0; alive && s < kStages; ++s) {
                alive = bound.wait(empty(r.stage), r.phase ^ 1u, kDevTmaWaitTimeout);
                r.next(kStages);
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && lane == 0) {
            Ring r;
            bool alive = true;
            int buf = 0;
            uint32_t buf_phase = 0;
            for (int i = pair; alive && i < P.tiles; i += pairs) {
                alive = bound.wait(sum_empty(buf), buf_phase ^ 1u, kDevEpilogueWaitTimeout);
                if (!alive) break;
                fence_after();
                const uint32_t d = tmem + 256u * buf;
                for (int kb = 0; kb < blocks; ++kb) {
                    alive = bound.wait(full(r.stage), r.phase, kDevMmaWaitTimeout);
                    if (!alive) break;
                    fence_after();
                    const uint32_t sa = base + r.stage * kStageBytes;
                    const uint32_t a = desc_low(sa, A_MN ? kHalf / 2 : 0), b = desc_low(sa + kHalf, B_MN ? kHalf / 2 : 0);
#pragma unroll
                    for (int j = 0; j < 4; ++j)      // 32 bytes of the contraction each (16 rows where m or n is contiguous)
                        mma<2, INT8>(d, a + j * (A_MN ? 128 : 2), b + j * (B_MN ? 128 : 2), P.idesc, kb + j > 0);
                    mma_commit<2>(empty(r.stage));
                    r.next(kStages);
                }
                if (alive) mma_commit<2>(sum_full(buf));
                buf ^= 1;
                buf_phase ^= buf == 0;
            }
        }
    } else if (warp >= 4) {
        const bool share = P.tiles <= pairs;
        const int quadrant = warp % 4, group = share ? 0 : (warp - 4) / (kEpiWarps / 2);
        const int parts = share ? kEpiWarps / 4 : kEpiWarps / 8, part = (warp - 4) / 4 % parts;
        const int cols = kTileN / parts;                       // of one warp
        Patches patch{patches + (warp - 4) * 2 * kPatchBytes};
        const bool adds = GATED && P.f.add[0];
        const int buf = group;
        uint32_t buf_phase = 0;
        bool alive = true;
        for (int i = pair + group * pairs; i < P.tiles; i += share ? pairs : 2 * pairs) {
            const Tile t = tile_at(P, i);
            const int64_t m0 = (int64_t)t.m * kTileM + 128 * rank + 32 * quadrant;
            const int64_t n0 = (int64_t)t.n * kTileN + cols * part;
            const int64_t m = m0 + lane < P.f.M ? m0 + lane : 0;
            const int rows = P.f.M - m0 < 32 ? (int)(P.f.M - m0) : 32;          // of the warp's that exist (<= 0: none)
            const Target out{&P.out[t.problem], P.f.out[t.problem], P.f.ldo, P.f.vec_out, DT == LORDBA_F32 ? 4 : 2};
            const uint8_t *add0 = static_cast<const uint8_t *>(P.f.add[0]) + 2 * (m * P.f.ld_add + n0);
            const uint8_t *add1 = static_cast<const uint8_t *>(P.f.add[1]) + 2 * (m * P.f.ld_add + n0);
            uint4 xg[4], xu[4];                                // the addends, fetched a step ahead
            if (adds) {
                fetch(xg, add0, P.f.vec_add, P.f.N - n0);
                fetch(xu, add1, P.f.vec_add, P.f.N - n0);
            }
            alive = __all_sync(0xffffffffu, bound.wait(sum_full(buf), buf_phase, kDevEpilogueWaitTimeout));
            if (!alive) break;
            fence_after();
            const uint32_t d = tmem + ((uint32_t)(32 * quadrant) << 16) + 256u * buf + cols * part;
#pragma unroll 1
            for (int c = 0; c < cols; c += kCh) {
                const int64_t n = n0 + c, left = P.f.N - n;
                if (rows <= 0 || left <= 0) break;             // the warp's rows or columns lie outside
                uint32_t g[kCh], u[kCh];
#pragma unroll
                for (int k = 0; k < kCh; k += 16) {
                    tmem_load16(d + c + k, g + k);
                    if (GATED) tmem_load16(d + 128 + c + k, u + k);
                }
                float v[kCh], w[kCh];
                tmem_wait_load();
                products_of<INT8, GATED, kCh>(P.f, m, n, (int)(left < kCh ? left : kCh), g, u, v, w);
                if (GATED) {
                    if (adds) {
                        add(xg, v, DT);
                        add(xu, w, DT);
                        if (c + kCh < cols) {
                            fetch(xg, add0 + 2 * (c + kCh), P.f.vec_add, left - kCh);
                            fetch(xu, add1 + 2 * (c + kCh), P.f.vec_add, left - kCh);
                        }
                    }
                    if (P.f.pre[0]) {
                        patch.put32(v, Target{&P.pre[0], P.f.pre[0], P.f.ld_pre, P.f.vec_pre, 2}, m0, n, rows, left, lane, DT);
                        patch.put32(w, Target{&P.pre[1], P.f.pre[1], P.f.ld_pre, P.f.vec_pre, 2}, m0, n, rows, left, lane, DT);
                    }
                    gate<kCh>(P.f.act, v, w);
                }
                patch.put32(v, out, m0, n, rows, left, lane, DT);
            }
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive_cluster(peer_addr(sum_empty(buf), 0));
            buf_phase ^= 1u;
        }
        if (lane == 0) stores_complete();
    }

    if (*abort_flag) {
        // time for copies still in flight to land before the CTA goes away
        const long long start = clock64();
        while (clock64() - start < 2000000LL) __nanosleep(1000);
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    cluster_sync();
    if (warp == 1) {
        fence_after();
        tmem_free<2>(tmem, 512);
    }
}

template <bool INT8, bool GATED, bool A_MN, bool B_MN, int DT>
int launch_tile(const TileArgs &args, cudaStream_t stream)
{
    const void *func = reinterpret_cast<const void *>(&product_tile_kernel<INT8, GATED, A_MN, B_MN, DT>);
    // co-resident pairs, asked for once a device: the query is slow
    static std::mutex mu;
    static int pairs_of[64] = {0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return LORDBA_ECUDA;
    int pairs;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (pairs_of[dev] == 0) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(2, 1, 1);
            cfg.blockDim = dim3(kTileThreads, 1, 1);
            cfg.dynamicSmemBytes = kTileSmem;
            cudaLaunchAttribute attr;
            attr.id = cudaLaunchAttributeClusterDimension;
            attr.val.clusterDim.x = 2; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
            cfg.attrs = &attr;
            cfg.numAttrs = 1;
            int n = 0;
            if (cudaFuncSetAttribute(func, cudaFuncAttributeMaxDynamicSharedMemorySize, kTileSmem) != cudaSuccess ||
                cudaOccupancyMaxActiveClusters(&n, func, &cfg) != cudaSuccess || n < 1) {
                cudaGetLastError();
                return LORDBA_ECUDA;
            }
            pairs_of[dev] = n;
        }
        pairs = pairs_of[dev];
    }
    LaunchRec rec;
    std::memset(&rec, 0, sizeof(rec));
    rec.func = func;
    rec.grid[0] = 2u * (unsigned)(args.tiles < pairs ? args.tiles : pairs);
    rec.grid[1] = rec.grid[2] = 1;
    rec.block = kTileThreads;
    rec.smem = kTileSmem;
    rec.cluster = 2;
    rec.pdl = 1;
    rec.n_args = 1;
    rec.arg_bytes[0] = sizeof(TileArgs);
    return launch_record(rec, &args, nullptr, stream);
}

template <int DT>
int launch_typed(const TileArgs &a, bool int8, bool gated, bool pair, bool b_mn, cudaStream_t stream)
{
    if (int8) return gated ? launch_tile<true, true, false, false, DT>(a, stream) : launch_tile<true, false, false, false, DT>(a, stream);
    if (gated) return launch_tile<false, true, false, false, DT>(a, stream);
    if (pair) return launch_tile<false, false, true, true, DT>(a, stream);
    return b_mn ? launch_tile<false, false, false, true, DT>(a, stream) : launch_tile<false, false, false, false, DT>(a, stream);
}

}  // namespace

// A round of tiles takes 0.285 us a stage (its MMAs at the clock under load), or the epilogue's time, or what its columns
// of B take from HBM at 4.2 TB/s (few rows: 2560 x 6912 gated 20 us), whichever is longest; the last round's
// epilogue shows; 5.4 us around them.
double tile_estimate(const Product &p)
{
    const bool gated = p.form == Product::kGated, int8 = p.kind == kProductInt8;
    const int block_k = int8 ? 128 : 64, parts = p.form == Product::kSum ? 2 : 1, pairs = sm_count() / 2;
    const int64_t tiles_m = (p.M + kTileM - 1) / kTileM;
    const int64_t tiles = tiles_m * ((p.N + (gated ? 127 : 255)) / (gated ? 128 : 256)) * (p.form == Product::kPair ? 2 : 1);
    const double column = 256.0 * (double)p.K * (int8 ? 1 : 2) * parts / 4.2e6;
    const int64_t across = tiles_m < 8 ? tiles_m : 8;
    const double walk = 0.285 * (double)((p.K + block_k - 1) / block_k) * parts;
    const double finish = 2.7 + (int8 ? 0.8 : 0.0) + (int8 && gated ? 0.7 : 0.0) + (p.add[0] ? 2.0 : 0.0) + (p.pre[0] ? 1.5 : 0.0);
    auto round = [&](int64_t n) {              // of n tiles
        const double loads = column * (double)((n + across - 1) / across);
        return walk > loads ? walk : loads;
    };
    const double full = round(pairs), last = round((tiles - 1) % pairs + 1);
    return 5.4 + (double)((tiles - 1) / pairs) * (full > finish ? full : finish) + last + finish - 2.7;
}

int launch_product_tile(const Product &p, const Finish &f, cudaStream_t stream)
{
    const bool int8 = p.kind == kProductInt8, gated = p.form == Product::kGated, pair = p.form == Product::kPair;
    const int e = int8 ? 1 : 2, block_k = int8 ? 128 : 64;
    TileArgs a;
    std::memset(&a, 0, sizeof(a));
    for (int i = 0; i < 2; ++i) {
        const Operand &oa = p.a[i], &ob = p.b[i];
        if (oa.p && !(oa.mn_major ? encode_map(&a.a[i], oa.p, p.K, p.M, oa.ld, e, 64) : encode_map(&a.a[i], oa.p, p.M, p.K, oa.ld, e, 128)))
            return LORDBA_ECUDA;
        if (ob.p && !(ob.mn_major ? encode_map(&a.b[i], ob.p, p.K, p.N, ob.ld, e, 64) : encode_map(&a.b[i], ob.p, p.N, p.K, ob.ld, e, 128)))
            return LORDBA_ECUDA;
    }
    for (int i = 0; i < 2; ++i) {
        const Operand &ol = p.lo[i];
        if (ol.p && !encode_map(&a.a[2 + i], ol.p, p.K, p.M, ol.ld, e, 64)) return LORDBA_ECUDA;
    }
    for (int i = 0; i < 2; ++i) {
        const int eo = f.dtype == LORDBA_F32 ? 4 : 2;
        const int64_t cols = f.N - f.N % (16 / eo);             // whole 16-byte pieces
        if (cols == 0) break;
        if (f.vec_out && f.out[i] && !encode_store_map(&a.out[i], f.out[i], f.M, cols, f.ldo, eo)) return LORDBA_ECUDA;
        if (f.vec_pre && f.pre[i] && !encode_store_map(&a.pre[i], f.pre[i], f.M, cols, f.ld_pre, 2)) return LORDBA_ECUDA;
    }
    const bool a_mn = p.a[0].mn_major, b_mn = p.b[0].mn_major;
    a.f = f;
    a.k_blocks = (int)((p.K + block_k - 1) / block_k);
    a.parts = p.form == Product::kSum || p.lo[0].p ? 2 : 1;
    a.problems = pair ? 2 : 1;
    const int64_t tm = (p.M + kTileM - 1) / kTileM, tn = (p.N + (gated ? 127 : 255)) / (gated ? 128 : 256);
    if (tm * tn * a.problems > (int64_t)1 << 30) return LORDBA_EUNSUPPORTED;
    a.tiles_m = (int)tm; a.tiles_n = (int)tn;
    a.tiles = (int)(tm * tn) * a.problems;
    a.skip = test_skip_item();
    a.status = device_status_word();
    if (!a.status) return LORDBA_ECUDA;
    a.idesc = instr_desc(int8, p.kind == kProductBf16, a_mn, b_mn, 256, 256);
    switch (p.dtype) {
        case LORDBA_BF16: return launch_typed<LORDBA_BF16>(a, int8, gated, pair, b_mn, stream);
        case LORDBA_F16: return launch_typed<LORDBA_F16>(a, int8, gated, pair, b_mn, stream);
        default: return launch_tile<true, false, false, false, LORDBA_F32>(a, stream);      // 8-bit products only
    }
}

}  // namespace lordba
