// The product kernel for few rows (tokens): the weights stream through, on tcgen05 with the roles swapped.
//
//   D[t,n] = sum_k tokens[t,k] weights[n,k]: 128 weight rows are the MMA's 128 rows, 16 ... 128 tokens its
//   columns, so that nothing is padded to 128 tokens.
//
// Bound: HBM, the weights are read once.  What that takes is many loads in flight on every SM and an even
// share for each of them: a tile of 128 weight rows is split along the contraction over a cluster of up to
// eight CTAs, two CTAs fit an SM, each has a ring of 16 KB stages.  The CTAs of a cluster exchange their
// partial sums through distributed shared memory and add them in rank order (the result does not depend
// on timing), each the share of outputs that it then finishes and writes.
//
//   warp 0 copies, warp 1 MMAs (one thread), warps 2-5 move the sums from TMEM to shared memory; then all
//   warps add, finish and write.
#include <cstring>
#include <mutex>

#include "product_internal.cuh"

namespace lordba {
namespace {

using namespace sm100;

constexpr int kRows = 128;                    // weight rows a tile
constexpr int kWeightBytes = kRows * 128;     // of one stage and weight matrix
constexpr int kStreamThreads = 6 * 32;
constexpr int kMaxStages = 12;
constexpr int kMaxSplit = 8;
constexpr int kBarBytes = (2 * kMaxStages + 1) * 8 + 16;

struct StreamArgs {
    CUtensorMap w[2], t[2];
    Finish f;
    int k_blocks, parts;     // stages per operand pair; operand pairs summed into one accumulator
    int tokens;              // MMA columns: tokens of a tile, a multiple of 16
    int stages, split;
    int tmem_columns;
    int skip;                // -1; the test-hooks build can name a stage whose copies are left out
    int *status;
    uint32_t idesc;
};

template <bool INT8, bool GATED, bool W_MN>
__global__ void __launch_bounds__(kStreamThreads, 2)
product_stream_kernel(const __grid_constant__ StreamArgs P)
{
    extern __shared__ uint8_t smem_raw[];
    constexpr int kSums = GATED ? 2 : 1;
    constexpr int kBlockK = INT8 ? 128 : 64;
    const uint32_t raw = smem_addr(smem_raw);
    const uint32_t bars = raw;                                     // barriers first: the ring's size varies
    const uint32_t base = (raw + kBarBytes + 1023u) & ~1023u;
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (kMaxStages + s); };
    const uint32_t sum_full = bars + 8u * (2 * kMaxStages);
    uint8_t *misc = smem_raw + (2 * kMaxStages + 1) * 8;
    volatile uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(misc);
    volatile int *abort_flag = reinterpret_cast<int *>(misc + 4);
    const Bounded bound{abort_flag, P.status};

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int rank = (int)cluster_rank();
    const int stage_bytes = kSums * kWeightBytes + P.tokens * 128;
    const int n0 = blockIdx.y * kRows, t0 = blockIdx.z * P.tokens;
    const int blocks = P.k_blocks * P.parts;
    const int first = (int)((int64_t)blocks * rank / P.split), last = (int)((int64_t)blocks * (rank + 1) / P.split);

    if (threadIdx.x == 0) {
        for (int s = 0; s < P.stages; ++s) {
            bar_init(full(s), 1);
            bar_init(empty(s), 1);
        }
        bar_init(sum_full, 1);
        *abort_flag = 0;
        bar_init_fence();
    }
    if (warp == 1) tmem_alloc<1>(smem_addr(misc), P.tmem_columns);
    if (warp == 2 && lane == 0) {
        prefetch_map(&P.w[0]);
        prefetch_map(&P.t[0]);
        if (GATED) prefetch_map(&P.w[1]);
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = *tmem_slot;
    grid_wait();
    grid_release();

    if (warp == 0) {
        if (lane == 0) {
            Ring r;
            for (int kb = first; kb < last; ++kb) {
                if (!bound.wait(empty(r.stage), r.phase ^ 1u, kDevTmaWaitTimeout)) break;
                bar_expect(full(r.stage), stage_bytes);
                if (kb - first != P.skip) {
                    const int part = kb >= P.k_blocks ? 1 : 0;
                    const int k0 = (kb - part * P.k_blocks) * kBlockK;
                    const uint32_t sw = base + r.stage * stage_bytes;
#pragma unroll
                    for (int c = 0; c < kSums; ++c) {
                        const CUtensorMap *mw = &P.w[GATED ? c : part];
                        if (W_MN) {
                            load_tile(sw, mw, n0, k0, full(r.stage));
                            load_tile(sw + kWeightBytes / 2, mw, n0 + 64, k0, full(r.stage));
                        } else {
                            load_tile(sw + c * kWeightBytes, mw, k0, n0, full(r.stage));
                        }
                    }
                    load_tile(sw + kSums * kWeightBytes, &P.t[part], k0, t0, full(r.stage));
                }
                r.next(P.stages);
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            Ring r;
            bool alive = true;
            for (int kb = first; kb < last; ++kb) {
                alive = bound.wait(full(r.stage), r.phase, kDevMmaWaitTimeout);
                if (!alive) break;
                fence_after();
                const uint32_t sw = base + r.stage * stage_bytes;
                const uint32_t t = desc_low(sw + kSums * kWeightBytes);
#pragma unroll
                for (int c = 0; c < kSums; ++c) {
                    const uint32_t w = desc_low(sw + c * kWeightBytes, W_MN ? kWeightBytes / 2 : 0);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        mma<1, INT8>(tmem + c * P.tokens, w + j * (W_MN ? 128 : 2), t + j * 2, P.idesc, kb - first + j > 0);
                }
                mma_commit<1>(empty(r.stage));
                r.next(P.stages);
            }
            if (alive) mma_commit<1>(sum_full);
        }
    } else {
        // the partial sums go where the ring was: [sum][token][128 weight rows]
        const int quadrant = warp % 4;
        const bool alive = __all_sync(0xffffffffu, bound.wait(sum_full, 0, kDevEpilogueWaitTimeout));
        if (alive) {
            fence_after();
            const uint32_t d = tmem + ((uint32_t)(32 * quadrant) << 16);
            uint32_t *sums = reinterpret_cast<uint32_t *>(smem_raw + (base - raw)) + 32 * quadrant + lane;
            for (int c = 0; c < kSums * P.tokens; c += 16) {
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
    if (warp == 1) {
        fence_after();
        tmem_free<1>(tmem, P.tmem_columns);
    }

    // four weight rows of one token an item, the items dealt to the cluster's threads
    if (*abort_flag == 0) {
        const int64_t have = P.f.M - t0;
        const int items = (int)(have < P.tokens ? have : P.tokens) * (kRows / 4);
        for (int it = rank * kStreamThreads + threadIdx.x; it < items; it += P.split * kStreamThreads) {
            const int t = it / (kRows / 4), j = 4 * (it % (kRows / 4));
            if (n0 + j >= P.f.N) continue;
            uint32_t acc[2][4];
#pragma unroll
            for (int c = 0; c < kSums; ++c) {
                const uint32_t at = base + 4u * ((c * P.tokens + t) * kRows + j);
                uint4 v[kMaxSplit];
#pragma unroll
                for (int r = 0; r < kMaxSplit; ++r)
                    if (r < P.split) v[r] = load_peer_v4(peer_addr(at, r));
                uint32_t *a = acc[c];
                a[0] = v[0].x; a[1] = v[0].y; a[2] = v[0].z; a[3] = v[0].w;
#pragma unroll
                for (int r = 1; r < kMaxSplit; ++r)
                    if (r < P.split) {
                        const uint32_t w[4] = {v[r].x, v[r].y, v[r].z, v[r].w};
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            a[i] = INT8 ? a[i] + w[i] : __float_as_uint(__uint_as_float(a[i]) + __uint_as_float(w[i]));
                    }
            }
            finish_row<INT8, GATED, 4>(P.f, 0, t0 + t, n0 + j, acc[0], acc[GATED ? 1 : 0]);
        }
    }
    if (P.split > 1) {
        __syncwarp();
        cluster_sync();         // the sums stay until every CTA has read them
    }
}

template <bool INT8, bool GATED, bool W_MN>
int launch_stream(const StreamArgs &args, dim3 grid, int smem, cudaStream_t stream)
{
    const void *func = reinterpret_cast<const void *>(&product_stream_kernel<INT8, GATED, W_MN>);
    static std::mutex mu;
    static bool ready[64] = {false};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return LORDBA_ECUDA;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!ready[dev]) {
            if (cudaFuncSetAttribute(func, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024) != cudaSuccess) {
                cudaGetLastError();
                return LORDBA_ECUDA;
            }
            ready[dev] = true;
        }
    }
    LaunchRec rec;
    std::memset(&rec, 0, sizeof(rec));
    rec.func = func;
    rec.grid[0] = grid.x; rec.grid[1] = grid.y; rec.grid[2] = grid.z;
    rec.block = kStreamThreads;
    rec.smem = (uint32_t)smem;
    rec.cluster = grid.x;
    rec.pdl = 1;
    rec.n_args = 1;
    rec.arg_bytes[0] = sizeof(StreamArgs);
    return launch_record(rec, &args, nullptr, stream);
}

}  // namespace

int launch_product_stream(const Product &p, const Finish &f, cudaStream_t stream)
{
    const bool int8 = p.kind == kProductInt8, gated = p.form == Product::kGated, w_mn = p.b[0].mn_major;
    const int e = int8 ? 1 : 2, block_k = int8 ? 128 : 64, sums = gated ? 2 : 1;
    StreamArgs a;
    std::memset(&a, 0, sizeof(a));
    a.f = f;
    a.k_blocks = (int)((p.K + block_k - 1) / block_k);
    a.parts = p.form == Product::kSum ? 2 : 1;
    a.tokens = p.M <= 16 ? 16 : p.M <= 32 ? 32 : p.M <= 64 ? 64 : 128;
    for (int i = 0; i < 2; ++i) {
        const Operand &ot = p.a[i], &ow = p.b[i];
        if (ot.p && !encode_map(&a.t[i], ot.p, p.M, p.K, ot.ld, e, a.tokens)) return LORDBA_ECUDA;
        if (ow.p && !(w_mn ? encode_map(&a.w[i], ow.p, p.K, p.N, ow.ld, e, 64) : encode_map(&a.w[i], ow.p, p.N, p.K, ow.ld, e, kRows)))
            return LORDBA_ECUDA;
    }
    const int stage = sums * kWeightBytes + a.tokens * 128, exchange = sums * a.tokens * kRows * 4;
    const int fixed = kBarBytes + 1024;
    // two CTAs an SM where three stages and the exchange fit half of its shared memory, else one
    const int half = 113 * 1024 - fixed, whole = 227 * 1024 - fixed;
    const int per_sm = 3 * stage <= half && exchange <= half ? 2 : 1;
    const int room = per_sm == 2 ? half : whole;
    a.stages = room / stage < kMaxStages ? room / stage : kMaxStages;
    const int64_t row_tiles = (p.N + kRows - 1) / kRows, token_tiles = (p.M + a.tokens - 1) / a.tokens;
    if (row_tiles > 65535 || token_tiles > 65535) return LORDBA_EUNSUPPORTED;
    // The split with the least rounds of CTAs x stages a CTA walks; six stages' worth of time go to a CTA's
    // start, the exchange and the epilogue.
    const int64_t slots = (int64_t)sm_count() * per_sm, work = row_tiles * token_tiles;
    const int blocks = a.k_blocks * a.parts;
    int64_t best = 0;
    for (int s = 1; s <= kMaxSplit && s <= blocks; ++s) {
        const int64_t cost = (work * s + slots - 1) / slots * ((blocks + s - 1) / s + 6);
        if (a.split == 0 || cost < best) { a.split = s; best = cost; }
    }
    a.tmem_columns = 32;
    while (a.tmem_columns < sums * a.tokens) a.tmem_columns *= 2;
    a.skip = test_skip_item();
    a.status = device_status_word();
    if (!a.status) return LORDBA_ECUDA;
    a.idesc = instr_desc(int8, p.kind == kProductBf16, w_mn, false, kRows, a.tokens);
    const int ring = a.stages * stage;
    const int smem = fixed + (ring > exchange ? ring : exchange);
    const dim3 grid((unsigned)a.split, (unsigned)row_tiles, (unsigned)token_tiles);
    if (int8) return gated ? launch_stream<true, true, false>(a, grid, smem, stream) : launch_stream<true, false, false>(a, grid, smem, stream);
    return gated ? launch_stream<false, true, false>(a, grid, smem, stream) : launch_stream<false, false, true>(a, grid, smem, stream);
}

}  // namespace lordba
