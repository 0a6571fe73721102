// Products of some tens of tokens with 4-bit weights, in either direction, on tcgen05: the weights stream past the tokens
// and are widened on the way.
//
//   forward     y[t,n]  = sum_k x[t,k] w[n,k]       a CTA's 128 MMA rows are weight rows, the contraction runs along them
//   backward    dx[t,k] = sum_n dy[t,n] w[n,k]      they are 128 columns (a block of the carrier), the contraction runs over rows
//
// Eight warps fetch packed pieces of 16 bytes, several stages ahead in registers, widen them (u - zero, exactly; times the scale,
// rounded once to the type of x) and write them as the swizzled tiles that the tensor core reads; the tokens come through the copy
// engine.  The contraction is split over a cluster of up to eight CTAs, whose sums meet in distributed shared memory and are
// added in rank order.
//
// Bound: the widening.  A piece takes a lane 152 operations (a pair a shift, a choice of bits, a subtraction and a product), 5 us
// for 4096 x 11008 weights on all SMs, where they arrive in 3.5 us; it is done once for up to 128 tokens.
//
//   warps 0-7 widen (0-3 also move the sums), warp 8 issues MMAs and warp 9 the tokens' copies (one thread each)
#include <cstring>
#include <mutex>

#include "int4_common.cuh"
#include "product_internal.cuh"

namespace lordba {
namespace {

using namespace sm100;

constexpr int kRows = 128;                     // MMA rows: weight rows, or columns
constexpr int kTile = kRows * 128;             // bytes of a stage's weights: 64 contraction steps
constexpr int kLoaders = 8, kThreads = 32 * (kLoaders + 2);
constexpr int kMaxStages = 6, kMaxSplit = 8;
constexpr int kBarBytes = (2 * kMaxStages + 1) * 8 + 16;
constexpr int kSmem = 113 * 1024;              // of a CTA: two share an SM

struct StreamArgs {
    CUtensorMap t;
    const uint8_t *q;
    const uint16_t *scale;
    const uint8_t *zero;
    void *out;
    int64_t ldq, ld_scale, ld_zero, ld_out;
    int64_t T, N;            // of the output
    int rows, groups;        // of the weights
    int group_log2;
    int blocks;              // stages in all
    int tokens, stages, split, tmem_columns, vec_out;
    int skip;                // -1; the test-hooks build can name a stage whose copy is left out
    int *status;
    uint32_t idesc;
};

// SPB: scales of a block and row, 1, 2 or 4.  A step of the loaders is a block of 128 columns of 128 rows, two stages (forward), or
// of 64 rows, one stage (backward): PIECES of 16 bytes a thread.
template <typename E, bool BACK, int SPB, bool ZERO>
__global__ void __launch_bounds__(kThreads, 2)
int4_stream_kernel(const __grid_constant__ StreamArgs P)
{
    extern __shared__ uint8_t smem_raw[];
    constexpr int PIECES = BACK ? 1 : 2, STAGES_A_STEP = BACK ? 1 : 2, DEPTH = (BACK ? 2 : 1) * (SPB == 4 ? 2 : SPB == 2 ? 3 : 4);
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
    const int steps = P.blocks / STAGES_A_STEP, first = steps * rank / P.split, last = steps * (rank + 1) / P.split;

    if (threadIdx.x == 0) {
        for (int s = 0; s < P.stages; ++s) {
            bar_init(full(s), kLoaders + 1);
            bar_init(empty(s), 1);
        }
        bar_init(sum_full, 1);
        *abort_flag = 0;
        bar_init_fence();
    }
    if (warp == 8) tmem_alloc<1>(smem_addr(misc), P.tmem_columns);
    if (warp == 9 && lane == 0) prefetch_map(&P.t);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = *tmem_slot;
    grid_wait();
    grid_release();

    if (warp == 9) {
        if (lane == 0) {
            Ring r;
            for (int kb = first * STAGES_A_STEP; kb < last * STAGES_A_STEP; ++kb) {
                if (!bound.wait(empty(r.stage), r.phase ^ 1u, kDevTmaWaitTimeout)) break;
                bar_expect(full(r.stage), P.tokens * 128);
                if (kb - first * STAGES_A_STEP != P.skip) load_tile(base + r.stage * stage_bytes + kTile, &P.t, kb * 64, t0, full(r.stage));
                r.next(P.stages);
            }
        }
    } else if (warp == 8) {
        if (lane == 0) {
            Ring r;
            bool alive = true;
            for (int kb = first * STAGES_A_STEP; kb < last * STAGES_A_STEP; ++kb) {
                alive = bound.wait(full(r.stage), r.phase, kDevMmaWaitTimeout);
                if (!alive) break;
                fence_after();
                const uint32_t sw = base + r.stage * stage_bytes;
                const uint32_t w = desc_low(sw, BACK ? kTile / 2 : 0), t = desc_low(sw + kTile);
#pragma unroll
                for (int j = 0; j < 4; ++j) mma<1, false>(tmem, w + j * (BACK ? 128 : 2), t + j * 2, P.idesc, kb - first * STAGES_A_STEP + j > 0);
                mma_commit<1>(empty(r.stage));
                r.next(P.stages);
            }
            if (alive) mma_commit<1>(sum_full);
        }
    } else {
        // lanes of a warp: four pieces of a row; eight rows in an order in which eight neighbouring lanes write to different banks
        const int t = lane % 4, row = 8 * warp + (lane / 8 + lane / 4 % 2 * 4);          // and, forward, 64 rows on
        const int column = BACK ? n0 : 0;                    // where the tile's columns begin
        uint4 ring[DEPTH][PIECES];
        uint16_t s[DEPTH][PIECES][SPB];
        uint8_t z[DEPTH][PIECES][SPB];
        auto fetch = [&](int step, int slot) {
            if (step >= last) return;
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int64_t n = BACK ? 64 * (int64_t)step + row : (int64_t)n0 + row + 64 * i;
                const int64_t c = BACK ? column : 128 * (int64_t)step;
                ring[slot][i] = make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int k = 0; k < SPB; ++k) { s[slot][i][k] = 0; z[slot][i][k] = 0; }
                if (n < P.rows) {
                    ring[slot][i] = __ldg(reinterpret_cast<const uint4 *>(P.q + n * P.ldq + c / 2 + 16 * t));
#pragma unroll
                    for (int k = 0; k < SPB; ++k) {
                        const int g = (int)((c + 128 / SPB * k) >> P.group_log2), at = g < P.groups ? g : P.groups - 1;
                        s[slot][i][k] = __ldg(P.scale + n * P.ld_scale + at);
                        if (ZERO) z[slot][i][k] = __ldg(P.zero + n * P.ld_zero + at);
                    }
                }
            }
        };
        // word j of piece i as eight columns in a tile
        auto widen = [&](int slot, int i, int j, uint32_t to) {
            const uint4 &x = ring[slot][i];
            const uint32_t word = j == 0 ? x.x : j == 1 ? x.y : j == 2 ? x.z : x.w;
            const uint32_t zero = int4_zero<E>(ZERO ? z[slot][i][j * SPB / 4] & 15u : 8u), one = s[slot][i][j * SPB / 4], scale = one | one << 16;
            uint32_t v[4];
#pragma unroll
            for (int p = 0; p < 4; ++p) v[p] = int4_scaled<E>(int4_pair<E>(word, p, zero), scale);
            store_shared_v4(to, make_uint4(v[0], v[1], v[2], v[3]));
        };
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) fetch(first + d, d);
        Ring r;
        bool alive = true;
        for (int step0 = first; alive && step0 < last; step0 += DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (!alive || step0 + d >= last) break;
#pragma unroll
                for (int h = 0; h < STAGES_A_STEP; ++h) {
                    alive = alive && __all_sync(0xffffffffu, bound.wait(empty(r.stage), r.phase ^ 1u, kDevTmaWaitTimeout));
                    if (!alive) break;
                    const uint32_t sw = base + r.stage * stage_bytes + row * 128;
                    // row + 64 has the same place in the swizzle
#pragma unroll
                    for (int i = 0; i < PIECES; ++i)
#pragma unroll
                        for (int j = 0; j < (BACK ? 4 : 2); ++j)
                            widen(d, i, BACK ? j : 2 * h + j, sw + (BACK ? j / 2 * (kTile / 2) : i * 64 * 128) + 16 * ((4 * (j % 2) + t) ^ (row & 7)));
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) bar_arrive(full(r.stage));
                    r.next(P.stages);
                }
                fetch(step0 + d + DEPTH, d);
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
    if (warp == 8) {
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

template <typename E, bool BACK>
const void *kernel_of(int spb, bool zero)
{
    if (zero) return spb == 1   ? (const void *)&int4_stream_kernel<E, BACK, 1, true>
                     : spb == 2 ? (const void *)&int4_stream_kernel<E, BACK, 2, true>
                                : (const void *)&int4_stream_kernel<E, BACK, 4, true>;
    return spb == 1   ? (const void *)&int4_stream_kernel<E, BACK, 1, false>
           : spb == 2 ? (const void *)&int4_stream_kernel<E, BACK, 2, false>
                      : (const void *)&int4_stream_kernel<E, BACK, 4, false>;
}

const void *kernel_of(const lordba_int4_proj &p, int dtype, bool backward)
{
    const int spb = p.group >= 128 ? 1 : 128 / p.group;
    if (dtype == LORDBA_BF16) return backward ? kernel_of<__nv_bfloat16, true>(spb, p.zero) : kernel_of<__nv_bfloat16, false>(spb, p.zero);
    return backward ? kernel_of<__half, true>(spb, p.zero) : kernel_of<__half, false>(spb, p.zero);
}

// Allowed its shared memory, once a device and kernel: the call takes as long as a launch.
bool allow(const void *func)
{
    static std::mutex mu;
    static const void *said[64][32];
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
    if (count[dev] < 32) said[dev][count[dev]++] = func;
    return true;
}

struct StreamPlan {
    int tokens, stages, split, blocks;
    int64_t row_tiles, token_tiles;
    double us;
};

StreamPlan plan_stream(const lordba_int4_proj &p, int64_t T, bool backward)
{
    StreamPlan s = {};
    const int64_t N = backward ? p.d_in : p.d_out;
    s.tokens = T <= 16 ? 16 : T <= 32 ? 32 : T <= 64 ? 64 : 128;
    s.blocks = (int)(backward ? (p.d_out + 63) / 64 : (p.d_in + 127) / 128 * 2);
    s.row_tiles = (N + kRows - 1) / kRows;
    s.token_tiles = (T + s.tokens - 1) / s.tokens;
    const int stage = kTile + s.tokens * 128, room = kSmem - kBarBytes - 1024;
    s.stages = room / stage < kMaxStages ? room / stage : kMaxStages;
    // Two CTAs an SM; a cluster of n takes what no other CTAs' clusters leave.
    const int steps = backward ? s.blocks : s.blocks / 2;
    for (int n = 1; n <= kMaxSplit && n <= steps; ++n) {
        const int64_t fit = 2 * sm_count() / n, work = s.row_tiles * s.token_tiles;
        const double rounds = (double)((work + fit - 1) / fit), each = (double)((steps + n - 1) / n) * (backward ? 0.5 : 1.0);
        const double us = 3.0 + rounds * (1.0 + each * 0.45 + s.tokens / 128.0 * (2.0 + 1.0 / n) + 0.19 * (n - 1));
        if (s.split == 0 || us < s.us) { s.split = n; s.us = us; }
    }
    return s;
}

}  // namespace

double int4_stream_estimate(const lordba_int4_proj &p, int64_t T, bool backward)
{
    const StreamPlan s = plan_stream(p, T, backward);
    return s.row_tiles <= 65535 && s.token_tiles <= 65535 ? s.us : -1.0;
}

int launch_int4_stream(const lordba_int4_proj &p, int64_t T, int dtype, bool backward, cudaStream_t stream)
{
    const StreamPlan plan = plan_stream(p, T, backward);
    StreamArgs a;
    std::memset(&a, 0, sizeof(a));
    const int64_t K = backward ? p.d_out : p.d_in;
    if (!encode_map(&a.t, p.in, T, K, p.ld_in, 2, plan.tokens)) return LORDBA_ECUDA;
    a.q = p.q; a.scale = static_cast<const uint16_t *>(p.scale); a.zero = p.zero; a.out = p.out;
    a.ldq = p.ldq; a.ld_scale = p.ld_scale; a.ld_zero = p.ld_zero; a.ld_out = p.ld_out;
    a.T = T;
    a.N = backward ? p.d_in : p.d_out;
    a.rows = (int)p.d_out;
    a.groups = (int)((p.d_in + p.group - 1) / p.group);
    while ((int64_t(1) << a.group_log2) < p.group) ++a.group_log2;
    a.blocks = plan.blocks;
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
    rec.func = kernel_of(p, dtype, backward);
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
