// Products of some tens of tokens with 4-bit weights, in either direction, on tcgen05: the weights stream past the tokens
// and are widened on the way.
//
//   forward     y[t,n]  = sum_k x[t,k] w[n,k]       a CTA's 128 MMA rows are weight rows, the contraction runs along them
//   backward    dx[t,k] = sum_n dy[t,n] w[n,k]      they are 128 columns (a block of the carrier), the contraction runs over rows
//
// Sixteen warps fetch packed pieces of 16 bytes, several steps ahead in registers, widen them (u - zero, exactly; times the scale,
// rounded once to the type of x) and write them as the swizzled tiles that the tensor core reads; the tokens come through the copy
// engine.  The contraction is split over a cluster of up to eight CTAs, whose sums meet in distributed shared memory and are
// added in rank order.
//
// Bound: latency, and the hand-over of stages.  A step takes a lone CTA 0.85 us (plan_stream), of which the widening's instructions are a
// quarter (a pair: a shift, a choice of bits, a subtraction and a product); 64 tokens through 4096 x 11008 keep the integer pipe 32 % and
// the issue slots 44 % busy, and the warps wait for weights, for one another at the stages' barriers, and for shared memory.  It is done once
// for up to 128 tokens.
// Measured, weights from HBM: 4096 x 4096, 64 / 128 / 256 tokens 12.6 / 14.9 / 22.2 us, 4096 x 11008 21.4 / 26.0 / 48.9 us (int4_way in
// base4_api.cu has the other way beside them).  Rings of 4 ... 12 stages, one CTA an
// SM, and half as many warps with two pieces each gained nothing.
//
//   warps 0-15 widen (0-3 also move the sums), warp 16 issues MMAs and warp 17 the tokens' copies (one thread each)
#include <cstring>
#include <mutex>

#include "int4_common.cuh"
#include "product_internal.cuh"

namespace lordba {
namespace {

using namespace sm100;

constexpr int kRows = 128;                     // MMA rows: weight rows, or columns
constexpr int kTile = kRows * 128;             // bytes of a stage's weights: 64 contraction steps
constexpr int kLoaders = 16, kThreads = 32 * (kLoaders + 2);
constexpr int kMaxStages = 6, kMaxSplit = 8;
constexpr int kBarBytes = (2 * kMaxStages + 1) * 8 + 16;
constexpr int kSmem = 113 * 1024;              // of a CTA: two share an SM

struct StreamArgs {
    CUtensorMap t;
    const uint8_t *q;
    const uint16_t *scale;
    const uint8_t *zero;
    void *out;
    uint32_t ldq, ld_scale, ld_zero;
    int64_t ld_out;
    int64_t T, N;            // of the output
    int rows, groups;        // of the weights
    int group_log2;
    int steps;               // of 128 contraction steps
    int tail;                // PARTIAL: columns of the last block
    int tokens, stages, split, tmem_columns, vec_out;
    int skip;                // -1; the test-hooks build can name a stage whose copy is left out
    int *status;
    uint32_t idesc;
};

// Loads that are issued where they stand: left to itself the compiler puts them off until shortly before their use.
__device__ __forceinline__ uint4 load_piece(const uint8_t *p)
{
    uint4 v;
    asm volatile("ld.global.nc.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t load_now(const uint16_t *p)
{
    uint32_t v;
    asm volatile("ld.global.nc.u16 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t load_now(const uint8_t *p)
{
    uint32_t v;
    asm volatile("ld.global.nc.u8 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}

// SPB: scales of a block and row, 1, 2 or 4.  PARTIAL (forward): the last block is not whole; looked for in every step it would
// cost whole ones up to 9 % (4096 -> 11008, 128 tokens, groups of 64 with zeros, 30.6 and 33.4 us).
template <typename E, bool BACK, int SPB, bool ZERO, bool PARTIAL>
__global__ void __launch_bounds__(kThreads, 2)
int4_stream_kernel(const __grid_constant__ StreamArgs P)
{
    extern __shared__ uint8_t smem_raw[];
    constexpr int DEPTH = SPB == 4 ? 2 : SPB == 2 ? 3 : 4;        // steps fetched ahead
    const uint32_t raw = smem_addr(smem_raw), bars = raw, base = (raw + kBarBytes + 1023u) & ~1023u;
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (kMaxStages + s); };
    const uint32_t sum_full = bars + 8u * (2 * kMaxStages);
    uint8_t *misc = smem_raw + (2 * kMaxStages + 1) * 8;
    volatile uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(misc);
    volatile int *abort_flag = reinterpret_cast<int *>(misc + 4);
    const Bounded bound{abort_flag, P.status};
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, rank = (int)cluster_rank();
    const int stage_bytes = kTile + P.tokens * 128;
    const int t0 = blockIdx.z * P.tokens, n0 = blockIdx.y * kRows;
    // the cluster's share of the steps, in whole ones
    const int first = P.steps * rank / P.split, last = P.steps * (rank + 1) / P.split;

    if (threadIdx.x == 0) {
        for (int s = 0; s < P.stages; ++s) {
            bar_init(full(s), (BACK ? kLoaders / 2 : kLoaders) + 1);
            bar_init(empty(s), 1);
        }
        bar_init(sum_full, 1);
        *abort_flag = 0;
        bar_init_fence();
    }
    if (warp == kLoaders) tmem_alloc<1>(smem_addr(misc), P.tmem_columns);
    if (warp == kLoaders + 1 && lane == 0) prefetch_map(&P.t);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = *tmem_slot;
    grid_wait();
    grid_release();

    if (warp == kLoaders + 1) {
        if (lane == 0) {
            Ring r;
            for (int kb = 2 * first; kb < 2 * last; ++kb) {
                if (!bound.wait(empty(r.stage), r.phase ^ 1u, kDevTmaWaitTimeout)) break;
                bar_expect(full(r.stage), P.tokens * 128);
                if (kb - 2 * first != P.skip) load_tile(base + r.stage * stage_bytes + kTile, &P.t, kb * 64, t0, full(r.stage));
                r.next(P.stages);
            }
        }
    } else if (warp == kLoaders) {
        if (lane == 0) {
            Ring r;
            bool alive = true;
            for (int kb = 2 * first; kb < 2 * last; ++kb) {
                alive = bound.wait(full(r.stage), r.phase, kDevMmaWaitTimeout);
                if (!alive) break;
                fence_after();
                const uint32_t sw = base + r.stage * stage_bytes;
                const uint32_t w = desc_low(sw, BACK ? kTile / 2 : 0), t = desc_low(sw + kTile);
#pragma unroll
                for (int j = 0; j < 4; ++j) mma<1, false>(tmem, w + j * (BACK ? 128 : 2), t + j * 2, P.idesc, kb - 2 * first + j > 0);
                mma_commit<1>(empty(r.stage));
                r.next(P.stages);
            }
            if (alive) mma_commit<1>(sum_full);
        }
    } else {
        // A step is 128 contraction steps, two stages: a piece a thread.  Lanes of a warp hold the four pieces of eight rows, in an
        // order in which eight neighbouring lanes write to different banks.  Forward, a piece's halves belong to the two stages;
        // backward the first eight warps' rows are the one stage and the others' the other.
        const int t = lane % 4, row = 8 * warp + (lane / 8 + lane / 4 % 2 * 4), own = BACK ? warp / 8 : 0;
        uint4 ring[DEPTH];
        uint32_t s[DEPTH][SPB];
        uint32_t z[DEPTH][SPB];
        // Behind the last row it is read again: forward what comes of it is not written, backward it meets zeros.
        const int row0 = BACK ? row : n0 + row < P.rows ? n0 + row : P.rows - 1, end = P.rows - 1;
        const uint8_t *q_at = P.q + (BACK ? n0 / 2 : (int64_t)row0 * P.ldq) + 16 * t;
        const uint16_t *s_at = P.scale + (BACK ? 0 : (int64_t)row0 * P.ld_scale);
        const uint8_t *z_at = P.zero + (BACK || !ZERO ? 0 : (int64_t)row0 * P.ld_zero);
        auto group = [&](int block, int k) {                 // of the k-th part of a block; a block is as long as a group at least, or shorter
            if (SPB == 1) return block >> (P.group_log2 - 7);
            const int g = SPB * block + k;
            return g < P.groups ? g : P.groups - 1;
        };
        int own_group[SPB];
#pragma unroll
        for (int k = 0; k < SPB; ++k) own_group[k] = group(n0 / 128, k);
        auto fetch = [&](int step, int slot) {
            if (step >= last) return;
            const int n = 128 * step + row0 < end ? 128 * step + row0 : end;         // backward
            ring[slot] = load_piece(q_at + (BACK ? (uint64_t)(uint32_t)n * P.ldq : (uint64_t)(64u * (uint32_t)step)));
#pragma unroll
            for (int k = 0; k < SPB; ++k) {
                s[slot][k] = load_now(s_at + (BACK ? (uint64_t)(uint32_t)n * P.ld_scale + (uint32_t)own_group[k] : (uint64_t)(uint32_t)group(step, k)));
                if (ZERO) z[slot][k] = load_now(z_at + (BACK ? (uint64_t)(uint32_t)n * P.ld_zero + (uint32_t)own_group[k] : (uint64_t)(uint32_t)group(step, k)));
            }
        };
        // where the piece's four words go in a stage
        uint32_t place[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            place[j] = base + (BACK ? j / 2 * (kTile / 2) + row % 64 * 128 : row * 128) + 16 * ((4 * (j % 2) + t) ^ (row & 7));
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) fetch(first + d, d);
        Ring r;
        bool alive = true;
        for (int step0 = first; alive && step0 < last; step0 += DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (!alive || step0 + d >= last) break;
                int stage[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (!BACK || h == own) alive = alive && bound.wait(empty(r.stage), r.phase ^ 1u, kDevTmaWaitTimeout);
                    stage[h] = r.stage;
                    r.next(P.stages);
                }
                alive = __all_sync(0xffffffffu, alive);
                if (!alive) break;
                uint32_t words[4] = {ring[d].x, ring[d].y, ring[d].z, ring[d].w};
                if (PARTIAL && step0 + d == P.steps - 1) {
                    // what the carrier holds behind the last column becomes the zero point: a weight made of it could be infinite, and
                    // meets the tokens' zeros
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int left = P.tail - 32 * j - 8 * t, have = left < 0 ? 0 : left < 8 ? left : 8;
                        const uint32_t keep = ((1u << 4 * ((have + 1) / 2)) - 1u) | ((1u << 4 * (have / 2)) - 1u) << 16;
                        words[j] = (words[j] & keep) | ((ZERO ? z[d][j * SPB / 4] & 15u : 8u) * 0x11111111u & ~keep);
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t zero = int4_zero<E>(ZERO ? z[d][j * SPB / 4] & 15u : 8u), one = s[d][j * SPB / 4], scale = one | one << 16;
                    uint32_t v[4];
#pragma unroll
                    for (int p = 0; p < 4; ++p) v[p] = int4_scaled<E>(int4_pair<E>(words[j], p, zero), scale);
                    store_shared_v4(place[j] + (BACK ? (own ? stage[1] : stage[0]) : stage[j / 2]) * stage_bytes, make_uint4(v[0], v[1], v[2], v[3]));
                }
                fetch(step0 + d + DEPTH, d);
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) {
                    if (!BACK || !own) bar_arrive(full(stage[0]));
                    if (!BACK || own) bar_arrive(full(stage[1]));
                }
            }
        }
        // the partial sums go where the ring was: [token][128 rows]
        if (warp < 4 && __all_sync(0xffffffffu, bound.wait(sum_full, 0, kDevEpilogueWaitTimeout))) {
            fence_after();
            const uint32_t d = tmem + ((uint32_t)(32 * warp) << 16);
            uint32_t *sums = reinterpret_cast<uint32_t *>(smem_raw + (base - raw)) + 32 * warp + lane;
            for (int c = 0; c < P.tokens; c += 16) {
                uint32_t v[16];
                tmem_load16(d + c, v);
                tmem_wait_load();
#pragma unroll
                for (int i = 0; i < 16; ++i) sums[(c + i) * kRows] = v[i];
            }
            fence_before();
        }
    }
    __syncthreads();
    if (*abort_flag) {
        // no CTA of the cluster writes: its sums would lack this CTA's part.  Copies in flight get time to land.
        if (threadIdx.x < P.split) store_peer(peer_addr(smem_addr(misc) + 4, threadIdx.x), 1);
        const long long start = clock64();
        while (clock64() - start < 2000000LL) __nanosleep(1000);
    }
    __syncwarp();
    cluster_sync();
    if (warp == kLoaders) {
        fence_after();
        tmem_free<1>(tmem, P.tmem_columns);
    }
    // four columns of one token an item, dealt to the cluster's threads
    if (*abort_flag == 0) {
        const int64_t have = P.T - t0;
        const int items = (int)(have < P.tokens ? have : P.tokens) * (kRows / 4);
        const int j = 4 * (threadIdx.x % (kRows / 4));
        const int64_t n = n0 + j, left = P.N - n;
        if (left > 0)
            for (int it = rank * kThreads + threadIdx.x; it < items; it += P.split * kThreads) {
                const int token = it / (kRows / 4);
                float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int k = 0; k < kMaxSplit; ++k) {
                    if (k >= P.split) break;
                    const uint4 u = load_peer_v4(peer_addr(base, k) + 4u * (token * kRows + j));
                    v.x += __uint_as_float(u.x); v.y += __uint_as_float(u.y); v.z += __uint_as_float(u.z); v.w += __uint_as_float(u.w);
                }
                E *to = static_cast<E *>(P.out) + (t0 + token) * P.ld_out + n;
                if (P.vec_out && left >= 4) {
                    *reinterpret_cast<uint2 *>(to) = make_uint2(pack2<E>(v.x, v.y), pack2<E>(v.z, v.w));
                } else {
                    const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i < left) to[i] = from_float<E>(w[i]);
                }
            }
    }
    if (P.split > 1) {
        __syncwarp();
        cluster_sync();         // the sums stay until every CTA has read them
    }
}

template <typename E, bool BACK, bool ZERO, bool PARTIAL>
const void *kernel_of(int spb)
{
    return spb == 1   ? (const void *)&int4_stream_kernel<E, BACK, 1, ZERO, PARTIAL>
           : spb == 2 ? (const void *)&int4_stream_kernel<E, BACK, 2, ZERO, PARTIAL>
                      : (const void *)&int4_stream_kernel<E, BACK, 4, ZERO, PARTIAL>;
}

template <typename E>
const void *kernel_of(const lordba_int4_proj &p, bool backward)
{
    const int spb = p.group >= 128 ? 1 : 128 / p.group;
    if (backward) return p.zero ? kernel_of<E, true, true, false>(spb) : kernel_of<E, true, false, false>(spb);
    if (p.d_in % 128) return p.zero ? kernel_of<E, false, true, true>(spb) : kernel_of<E, false, false, true>(spb);
    return p.zero ? kernel_of<E, false, true, false>(spb) : kernel_of<E, false, false, false>(spb);
}

// Allowed its shared memory, once a device and kernel: the call takes as long as a launch.
bool allow(const void *func)
{
    static std::mutex mu;
    constexpr int kMost = 36;              // instantiations
    static const void *said[64][kMost];
    static int count[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
    std::lock_guard<std::mutex> lock(mu);
    for (int i = 0; i < count[dev]; ++i)
        if (said[dev][i] == func) return true;
    if (cudaFuncSetAttribute(func, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    if (count[dev] < kMost) said[dev][count[dev]++] = func;
    return true;
}

struct StreamPlan {
    int tokens, stages, split, steps;
    int64_t row_tiles, token_tiles;
    double us;
};

StreamPlan plan_stream(const lordba_int4_proj &p, int64_t T, bool backward)
{
    StreamPlan s = {};
    const int64_t N = backward ? p.d_in : p.d_out;
    s.tokens = T <= 16 ? 16 : T <= 32 ? 32 : T <= 64 ? 64 : 128;
    s.steps = (int)(((backward ? p.d_out : p.d_in) + 127) / 128);
    s.row_tiles = (N + kRows - 1) / kRows;
    s.token_tiles = (T + s.tokens - 1) / s.tokens;
    const int stage = kTile + s.tokens * 128, room = kSmem - kBarBytes - 1024;
    s.stages = room / stage < kMaxStages ? room / stage : kMaxStages;
    // Two CTAs share an SM.  A step takes one that is alone there 0.85 us, two at a time 1.25 us; around the steps 4 us, 0.4 us a CTA
    // that the sums are exchanged with, and 3 to 6 us for 128 tokens' sums (4096 x 4096, 17 tokens, clusters of 1, 2, 4, 6 and 8: 29.5, 17.6,
    // 11.8, 13.4 and 12.0 us; 4096 x 11008: 29.7, 24.8 and, of 3 and 4, 19.4 and 26.7 us).
    for (int n = 1; n <= kMaxSplit && n <= s.steps; ++n) {
        const int64_t fit = 2 * sm_count() / n, work = s.row_tiles * s.token_tiles;
        const double rounds = (double)((work + fit - 1) / fit), steps = (double)((s.steps + n - 1) / n);
        const bool alone = work * n <= sm_count();
        const double us = 4.0 + rounds * (steps * (alone ? 0.85 : 1.25) + 0.4 * n + s.tokens / 128.0 * (alone ? 3.2 : 6.5));
        if (s.split == 0 || us < s.us) { s.split = n; s.us = us; }
    }
    return s;
}

}  // namespace

bool int4_stream_takes(const lordba_int4_proj &p, int64_t T, bool backward)
{
    const StreamPlan s = plan_stream(p, T, backward);
    constexpr int64_t kFar = int64_t(1) << 31;           // pitches, and rows and columns with a tile's on top, are 32 bits
    return p.d_in < kFar / 2 && p.d_out < kFar / 2 && s.row_tiles <= 65535 && s.token_tiles <= 65535 && p.ldq < kFar && p.ld_scale < kFar && (!p.zero || p.ld_zero < kFar);
}

int launch_int4_stream(const lordba_int4_proj &p, int64_t T, int dtype, bool backward, cudaStream_t stream)
{
    const StreamPlan plan = plan_stream(p, T, backward);
    StreamArgs a;
    std::memset(&a, 0, sizeof(a));
    const int64_t K = backward ? p.d_out : p.d_in;
    if (!encode_map(&a.t, p.in, T, K, p.ld_in, 2, plan.tokens)) return LORDBA_ECUDA;
    a.q = p.q; a.scale = static_cast<const uint16_t *>(p.scale); a.zero = p.zero; a.out = p.out;
    a.ldq = (uint32_t)p.ldq; a.ld_scale = (uint32_t)p.ld_scale; a.ld_zero = (uint32_t)p.ld_zero; a.ld_out = p.ld_out;
    a.T = T;
    a.N = backward ? p.d_in : p.d_out;
    a.rows = (int)p.d_out;
    a.groups = (int)((p.d_in + p.group - 1) / p.group);
    while ((int64_t(1) << a.group_log2) < p.group) ++a.group_log2;
    a.steps = plan.steps;
    a.tail = (int)(p.d_in % 128);
    a.tokens = plan.tokens;
    a.stages = plan.stages;
    a.split = plan.split;
    a.tmem_columns = plan.tokens < 32 ? 32 : plan.tokens;
    a.vec_out = aligned(p.out, 8) && p.ld_out % 4 == 0;
    a.skip = test_skip_item();
    a.status = device_status_word();
    if (!a.status) return LORDBA_ECUDA;
    a.idesc = instr_desc(false, dtype == LORDBA_BF16, backward, false, kRows, plan.tokens);
    LaunchRec rec;
    std::memset(&rec, 0, sizeof(rec));
    rec.func = dtype == LORDBA_BF16 ? kernel_of<__nv_bfloat16>(p, backward) : kernel_of<__half>(p, backward);
    if (!allow(rec.func)) return LORDBA_ECUDA;
    rec.grid[0] = (unsigned)plan.split; rec.grid[1] = (unsigned)plan.row_tiles; rec.grid[2] = (unsigned)plan.token_tiles;
    rec.block = kThreads;
    const int used = plan.stages * (kTile + plan.tokens * 128), sums = plan.tokens * kRows * 4;
    rec.smem = (uint32_t)(kBarBytes + 1024 + (used > sums ? used : sums));
    rec.cluster = (uint32_t)plan.split;
    rec.pdl = 1;
    rec.n_args = 1;
    rec.arg_bytes[0] = sizeof(StreamArgs);
    return launch_record(rec, &a, nullptr, stream);
}

}  // namespace lordba
