// The product kernel for few rows (tokens): the weights stream through, on tcgen05 with the roles swapped.
//
// (and for sums so long that their few results leave SMs idle: the split along the contraction fills them)
//
//   D[t,n] = sum_k tokens[t,k] weights[n,k]: 128 weight rows are the MMA's 128 rows, 16 ... 128 tokens its
//   columns, so that nothing is padded to 128 tokens.
//
// Bound: HBM, the weights are read once.  What that takes is many loads in flight on every SM and an even
// share for each of them: a tile of 128 weight rows is split along the contraction over a cluster of up to
// eight CTAs, two CTAs fit an SM, each has a ring of stages (16 KB a weight matrix and the tokens' part).  The CTAs of a cluster exchange their
// partial sums through distributed shared memory and add them in rank order (the result does not depend
// on timing), each the share of outputs that it then finishes and writes.
//
// Measured, one call after the other on weights from HBM: gated 8 x 4096 -> 11008 in bf16 32 us (180 MB, 5.7 TB/s, 86 % of
// what a copy reaches), 64 tokens 36 us; 8-bit one token x 4096 -> 11008 11.6 us (45 MB), 4096 -> 4096 7.5 us (17 MB): what
// does not shrink with the weights is 5 us of latencies (launch, first stages, exchange, store).
//
//   warps 0-3 move the sums from TMEM to shared memory, warp 4 issues MMAs and warp 5 copies (one thread
//   each); then all warps add, finish and write.
//
// Operands whose base or pitch is not a multiple of 16 bytes are out of the copy engine's reach.  Copying
// them first would move each weight three times; instead (LOOSE) warps 0-3 and 6-9 fetch the aligned pieces
// that hold a stage into a second ring, several stages ahead (cp.async), and shift them into place.
#include <atomic>
#include <cstring>
#include <mutex>

#include "product_internal.cuh"

namespace lordba {
namespace {

using namespace sm100;

constexpr int kRows = 128;                    // weight rows a tile
constexpr int kWeightBytes = kRows * 128;     // of one stage and weight matrix
__host__ __device__ constexpr int threads_of(bool loose) { return loose ? 10 * 32 : 6 * 32; }
constexpr int kMaxStages = 12;
constexpr int kMaxSplit = 8;
constexpr int kBarBytes = (2 * kMaxStages + 1) * 8 + 16;
constexpr int kHalf = 113 * 1024, kWhole = 227 * 1024;      // shared memory of a CTA where two, or one, share an SM

struct Rows {              // a row-major matrix in bytes
    const uint8_t *p;
    int64_t ld, rows, cols;
};

struct StreamArgs {
    CUtensorMap w[2], t[4];   // t[2 + i]: the rest of t[i], where halves = 2
    Rows rw[2], rt[4];       // the same operands as they lie in memory
    Finish f;
    int k_blocks, parts;     // stages per operand pair; operand pairs summed into one accumulator
    int tokens;              // of a tile: a multiple of 16
    int halves;              // 2: the tokens' entries come as two terms, each term MMA columns of its own
    int token_tiles;         // of one problem (T_MN: two problems, with the tokens t[0] and t[1])
    int problems;
    int groups;              // more than 1: so many clusters share a tile's contraction and write their sums to
    uint32_t *raw;           // raw, [group][problem or gate, up][M][raw_ld], for finish_kernel to add
    int64_t raw_ld;          // N rounded up to 4
    uint32_t *whole;         // [blockIdx.z][row tile]: whether the cluster's sums are complete; every cluster says so
    int stages, split;
    int raw_stages;          // LOOSE: stages fetched ahead (2 ... 6)
    int tmem_columns;
    int skip;                // -1; the test-hooks build can name a stage whose copies are left out
    int *status;
    uint32_t idesc;
};

// ---- LOOSE: rows of BOXES x 128 bytes from row y and byte x of a matrix on -----------------------------------
// A warp fetches and shifts the same rows, so the two steps need no barrier between warps.  What lies past the
// matrix's end in either direction is fetched as zeros, or masked where it shares a piece with valid bytes.
constexpr int kLoaders = 8;                                                 // warps
template <int BOXES> constexpr int kRawPitch = BOXES * 128 + 16;             // one more piece than the row's share

// A lane's share of a matrix: up to four rows, kStep apart.  Their distance is a multiple of 16 rows, so they
// all lie alike against the 16-byte grid.
template <int BOXES>
struct Share {
    static constexpr int kAcross = 8 * BOXES, kPer = 32 / kAcross, kStep = kLoaders * kPer;
    uintptr_t at;          // first row's byte x0, rounded down, plus the lane's piece
    int64_t stride;        // to the next row
    int64_t left;          // bytes from `at` to the end of the row
    uint32_t raw, dst;     // offsets of the first row's piece in a raw and in an ordinary stage
    uint32_t by;
    int first, rows;       // first row in the tile; rows the tile has of the matrix, counted from it
    bool edge;             // the lane also fetches the piece after its own

    // the part of `tile_rows` rows from row y and byte x on
    __device__ __forceinline__ Share(int loader, int lane, const Rows &m, int64_t x, int64_t y, int tile_rows)
    {
        const int piece = lane % kAcross;
        first = loader * kPer + lane / kAcross;
        const uintptr_t row = reinterpret_cast<uintptr_t>(m.p) + (y + first) * m.ld;
        by = (uint32_t)(row + x) & 15u;
        at = row + x - by + 16 * piece;
        left = (int64_t)(row + m.cols - at);
        stride = m.ld * kStep;
        raw = first * kRawPitch<BOXES> + 16 * piece;
        dst = (piece / 8) * tile_rows * 128 + first * 128 + (((piece % 8) ^ (first & 7)) * 16);     // kStep is a multiple of 8
        edge = piece == kAcross - 1;
        const int64_t have = m.rows - y < tile_rows ? m.rows - y : tile_rows;
        rows = (int)have;
    }
    // `dx` bytes on along the row, `dy` rows down (both from the share's place; dy a multiple of 16)
    __device__ __forceinline__ void fetch(uint32_t stage, int64_t dx, int64_t dy_bytes, int rows_now, int tile_rows) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (first + i * kStep >= tile_rows) break;
            const bool in = first + i * kStep < rows_now;
            const uintptr_t from = at + dx + dy_bytes + i * stride;
            const uint32_t to = stage + raw + i * kStep * kRawPitch<BOXES>;
            fetch16(to, from, in && dx < left);
            if (edge) fetch16(to + 16, from + 16, in && dx + 16 < left);
        }
    }
    __device__ __forceinline__ void shift(uint32_t stage, uint32_t to, int64_t dx, int tile_rows) const
    {
        const int64_t valid64 = left - by - dx;                    // valid bytes of the joined piece
        const int valid = valid64 >= 16 ? 16 : valid64 > 0 ? (int)valid64 : 0;
        uint32_t keep[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) keep[j] = valid >= 4 * j + 4 ? 0xffffffffu : valid <= 4 * j ? 0u : (1u << 8 * (valid - 4 * j)) - 1u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (first + i * kStep >= tile_rows) break;
            const uint32_t from = stage + raw + i * kStep * kRawPitch<BOXES>;
            const uint4 v = join_pieces(load_shared_v4(from), load_shared_v4(from + 16), by);
            store_shared_v4(to + dst + i * kStep * 128, make_uint4(v.x & keep[0], v.y & keep[1], v.z & keep[2], v.w & keep[3]));
        }
    }
};

// ---- epilogue: four weight rows (columns of the output) of one token ------------------------------------------
// Neighbouring lanes hold neighbouring columns, so whatever the alignment a warp's accesses are whole lines.
__device__ __forceinline__ void load4(const void *p, int64_t at, int n, int vec, int dtype, float v[4])
{
    const uint16_t *q = static_cast<const uint16_t *>(p) + at;
    uint2 w;
    if (vec && n >= 4) {
        w = *reinterpret_cast<const uint2 *>(q);
    } else {
        uint32_t x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = i < n ? q[i] : 0u;
        w = make_uint2(x[0] | x[1] << 16, x[2] | x[3] << 16);
    }
    const float2 lo = unpack2_any(w.x, dtype), hi = unpack2_any(w.y, dtype);
    v[0] = lo.x; v[1] = lo.y; v[2] = hi.x; v[3] = hi.y;
}

__device__ __forceinline__ void store4(void *p, int64_t at, int n, int vec, int dtype, const float v[4])
{
    if (dtype == LORDBA_F32) {
        float *q = static_cast<float *>(p) + at;
        if (vec && n >= 4) {
            *reinterpret_cast<float4 *>(q) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < n) q[i] = v[i];
        }
        return;
    }
    uint16_t *q = static_cast<uint16_t *>(p) + at;
    const uint32_t w[2] = {pack2_any(v[0], v[1], dtype), pack2_any(v[2], v[3], dtype)};
    if (vec && n >= 4) {
        *reinterpret_cast<uint2 *>(q) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) q[i] = (uint16_t)(w[i / 2] >> 16 * (i % 2));
    }
}

template <bool INT8, bool GATED>
__device__ __forceinline__ void finish4(const Finish &F, int problem, int64_t m, int64_t n, const uint32_t acc0[4], const uint32_t acc1[4])
{
    const int left = (int)(F.N - n < 4 ? F.N - n : 4);
    float v[4], w[4];
    products_of<INT8, GATED, 4>(F, m, n, left, acc0, acc1, v, w);
    if (GATED) {
        if (F.add[0]) {
            float a[4], b[4];
            load4(F.add[0], m * F.ld_add + n, left, F.vec_add, F.dtype, a);
            load4(F.add[1], m * F.ld_add + n, left, F.vec_add, F.dtype, b);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] += a[i]; w[i] += b[i]; }
        }
        if (F.pre[0]) {
            store4(F.pre[0], m * F.ld_pre + n, left, F.vec_pre, F.dtype, v);
            store4(F.pre[1], m * F.ld_pre + n, left, F.vec_pre, F.dtype, w);
        }
        gate<4>(F.act, v, w);
    }
    store4(F.out[problem], m * F.ldo + n, left, F.vec_out, F.dtype, v);
}

template <bool INT8>
__device__ __forceinline__ uint4 add4(uint4 a, uint4 b)
{
    if (INT8) return make_uint4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
    return make_uint4(__float_as_uint(__uint_as_float(a.x) + __uint_as_float(b.x)), __float_as_uint(__uint_as_float(a.y) + __uint_as_float(b.y)),
                      __float_as_uint(__uint_as_float(a.z) + __uint_as_float(b.z)), __float_as_uint(__uint_as_float(a.w) + __uint_as_float(b.w)));
}

// W_MN, T_MN: the contraction runs along the rows of the weights (the tokens).  T_MN is the gradients of weights:
// the "tokens" are rows of the result, the entries of dgate or dup, and the contraction is over the real tokens.
template <bool INT8, bool GATED, bool W_MN, bool T_MN, bool LOOSE>
__global__ void __launch_bounds__(threads_of(LOOSE), LOOSE ? 1 : 2)
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
    constexpr int kHalves = W_MN && !T_MN ? 2 : 1;                // at most
    const int halves = kHalves > 1 ? P.halves : 1, columns = halves * P.tokens;
    const int stage_bytes = kSums * kWeightBytes + columns * 128;
    const int z = (int)blockIdx.z / P.token_tiles;
    const int t0 = ((int)blockIdx.z - z * P.token_tiles) * P.tokens, n0 = blockIdx.y * kRows;
    const int group = z / P.problems, problem = z - group * P.problems;
    const int blocks = P.k_blocks * P.parts;
    const int slice = group * P.split + rank, slices = P.groups * P.split;
    const int first = (int)((int64_t)blocks * slice / slices), last = (int)((int64_t)blocks * (slice + 1) / slices);

    if (threadIdx.x == 0) {
        for (int s = 0; s < P.stages; ++s) {
            bar_init(full(s), LOOSE ? 32 * kLoaders : 1);
            bar_init(empty(s), 1);
        }
        bar_init(sum_full, 1);
        *abort_flag = 0;
        bar_init_fence();
    }
    if (warp == 4) tmem_alloc<1>(smem_addr(misc), P.tmem_columns);
    if (!LOOSE && warp == 5 && lane == 0) {
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

    if (warp == 5) {
        if (!LOOSE && lane == 0) {
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
                    if (T_MN) {
                        for (int b = 0; b < P.tokens; b += 64)
                            load_tile(sw + kWeightBytes + b * 128, &P.t[problem], t0 + b, k0, full(r.stage));
                    } else {
                        load_tile(sw + kSums * kWeightBytes, &P.t[part], k0, t0, full(r.stage));
                    }
                    if (halves > 1) load_tile(sw + kSums * kWeightBytes + P.tokens * 128, &P.t[2 + part], k0, t0, full(r.stage));
                }
                r.next(P.stages);
            }
        }
    } else if (warp == 4) {
        if (lane == 0) {
            Ring r;
            bool alive = true;
            for (int kb = first; kb < last; ++kb) {
                alive = bound.wait(full(r.stage), r.phase, kDevMmaWaitTimeout);
                if (!alive) break;
                fence_after();
                const uint32_t sw = base + r.stage * stage_bytes;
                const uint32_t t = desc_low(sw + kSums * kWeightBytes, T_MN ? 64 * 128 : 0);
#pragma unroll
                for (int c = 0; c < kSums; ++c) {
                    const uint32_t w = desc_low(sw + c * kWeightBytes, W_MN ? kWeightBytes / 2 : 0);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        mma<1, INT8>(tmem + c * columns, w + j * (W_MN ? 128 : 2), t + j * (T_MN ? 128 : 2), P.idesc, kb - first + j > 0);
                }
                mma_commit<1>(empty(r.stage));
                r.next(P.stages);
            }
            if (alive) mma_commit<1>(sum_full);
        }
    } else {
        if (LOOSE) {
            const int loader = warp < 4 ? warp : warp - 2;
            const uint32_t raw0 = base + P.stages * stage_bytes;
            const int raw_weight = W_MN ? 64 * kRawPitch<2> : kRows * kRawPitch<1>;
            const int raw_bytes = kSums * raw_weight + columns * kRawPitch<1>;
            constexpr int kBoxes = W_MN ? 2 : 1, kBoxRows = W_MN ? 64 : kRows;
            // of a sum of two products the second has operands of its own
            const Share<kBoxes> w0(loader, lane, P.rw[0], W_MN ? 2 * (int64_t)n0 : 0, W_MN ? 0 : n0, kBoxRows);
            const Share<kBoxes> w1(loader, lane, P.rw[GATED || P.parts > 1 ? 1 : 0], W_MN ? 2 * (int64_t)n0 : 0, W_MN ? 0 : n0, kBoxRows);
            const Share<1> tok0(loader, lane, P.rt[0], 0, t0, P.tokens);
            const Share<1> tok1(loader, lane, P.rt[W_MN && P.parts > 1 ? 1 : 0], 0, t0, P.tokens);
            const Share<1> rest0(loader, lane, P.rt[halves > 1 ? 2 : 0], 0, t0, P.tokens);
            const Share<1> rest1(loader, lane, P.rt[halves > 1 ? 3 : 0], 0, t0, P.tokens);
            const int raw_rest = kSums * raw_weight + P.tokens * kRawPitch<1>, rest_at = kSums * kWeightBytes + P.tokens * 128;
            const int64_t contraction = W_MN ? P.rw[0].rows : 0, ld = P.rw[0].ld;
            auto fetch = [&](int kb, int slot) {
                const uint32_t raw = raw0 + slot * raw_bytes;
                if (kb < last) {
                    const bool second = W_MN && kb >= P.k_blocks;
                    const int64_t at = kb - (second ? P.k_blocks : 0);
                    if (W_MN) {
                        const int64_t have = contraction - kBlockK * at;
                        const int rows_now = (int)(have < kBoxRows ? have : kBoxRows);
                        if (second) w1.fetch(raw, 0, kBlockK * at * ld, rows_now, kBoxRows);
                        else w0.fetch(raw, 0, kBlockK * at * ld, rows_now, kBoxRows);
                    } else {
                        w0.fetch(raw, 128 * at, 0, w0.rows, kBoxRows);
                        if (GATED) w1.fetch(raw + raw_weight, 128 * at, 0, w1.rows, kBoxRows);
                    }
                    if (second) tok1.fetch(raw + kSums * raw_weight, 128 * at, 0, tok1.rows, P.tokens);
                    else tok0.fetch(raw + kSums * raw_weight, 128 * at, 0, tok0.rows, P.tokens);
                    if (halves > 1) {
                        if (second) rest1.fetch(raw + raw_rest, 128 * at, 0, rest1.rows, P.tokens);
                        else rest0.fetch(raw + raw_rest, 128 * at, 0, rest0.rows, P.tokens);
                    }
                }
                fetch_commit();        // also where there is nothing left: the groups are counted
            };
            for (int i = 0; i < P.raw_stages; ++i) fetch(first + i, i);
            Ring r;
            int slot = 0;
            for (int kb = first; kb < last; ++kb) {
                fetch_wait(P.raw_stages - 1);
                __syncwarp();
                const bool go = __all_sync(0xffffffffu, bound.wait(empty(r.stage), r.phase ^ 1u, kDevTmaWaitTimeout));
                if (!go) break;
                const uint32_t sw = base + r.stage * stage_bytes, raw = raw0 + slot * raw_bytes;
                const bool second = W_MN && kb >= P.k_blocks;
                const int64_t at = kb - (second ? P.k_blocks : 0);
                if (W_MN) {
                    if (second) w1.shift(raw, sw, 0, kBoxRows);
                    else w0.shift(raw, sw, 0, kBoxRows);
                } else {
                    w0.shift(raw, sw, 128 * at, kBoxRows);
                    if (GATED) w1.shift(raw + raw_weight, sw + kWeightBytes, 128 * at, kBoxRows);
                }
                if (second) tok1.shift(raw + kSums * raw_weight, sw + kSums * kWeightBytes, 128 * at, P.tokens);
                else tok0.shift(raw + kSums * raw_weight, sw + kSums * kWeightBytes, 128 * at, P.tokens);
                if (halves > 1) {
                    if (second) rest1.shift(raw + raw_rest, sw + rest_at, 128 * at, P.tokens);
                    else rest0.shift(raw + raw_rest, sw + rest_at, 128 * at, P.tokens);
                }
                fence_proxy_async();
                if (kb - first != P.skip) bar_arrive(full(r.stage));
                __syncwarp();
                fetch(kb + P.raw_stages, slot);
                slot = slot + 1 == P.raw_stages ? 0 : slot + 1;
                r.next(P.stages);
            }
            fetch_wait(0);
            __syncwarp();
        }
        // the partial sums go where the ring was: [sum][half][token][128 weight rows]
        const int quadrant = warp;
        const bool alive = warp < 4 && __all_sync(0xffffffffu, bound.wait(sum_full, 0, kDevEpilogueWaitTimeout));
        if (alive) {
            fence_after();
            const uint32_t d = tmem + ((uint32_t)(32 * quadrant) << 16);
            uint32_t *sums = reinterpret_cast<uint32_t *>(smem_raw + (base - raw)) + 32 * quadrant + lane;
            for (int c = 0; c < kSums * columns; c += 16) {
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
    if (warp == 4) {
        fence_after();
        tmem_free<1>(tmem, P.tmem_columns);
    }

    if (P.groups > 1 && rank == 0 && threadIdx.x == 0) P.whole[blockIdx.z * gridDim.y + blockIdx.y] = *abort_flag == 0;

    // four weight rows of one token an item, the items dealt to the cluster's threads, kBatch of a thread's at
    // a time: their sums are all on the way before the first is finished
    if (*abort_flag == 0) {
        constexpr int kBatch = GATED ? 2 : 4;
        const int64_t have = P.f.M - t0;
        const int items = (int)(have < P.tokens ? have : P.tokens) * (kRows / 4), step = P.split * threads_of(LOOSE);
        const int j = 4 * (threadIdx.x % (kRows / 4));             // a thread's items share their weight rows
        if (n0 + j < P.f.N)
            for (int it = rank * threads_of(LOOSE) + threadIdx.x; it < items; it += kBatch * step) {
                uint4 acc[kBatch][2];
#pragma unroll
                for (int r = 0; r < kMaxSplit; ++r) {
                    if (r >= P.split) break;
                    const uint32_t from = peer_addr(base, r) + 4u * j;
#pragma unroll
                    for (int k = 0; k < kBatch; ++k) {
                        const int i = it + k * step;
                        if (i < items)         // a predicate of the loads: a way out of the loop would keep them from being batched
#pragma unroll
                        for (int c = 0; c < kSums; ++c) {
                            const uint32_t at = from + 4u * ((c * columns + i / (kRows / 4)) * kRows);
                            uint4 v = load_peer_v4(at);
                            if (kHalves > 1 && halves > 1) v = add4<INT8>(v, load_peer_v4(at + 4u * P.tokens * kRows));
                            acc[k][c] = r == 0 ? v : add4<INT8>(acc[k][c], v);
                        }
                    }
                }
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    if (it + k * step >= items) break;
                    if (P.groups > 1) {
                        const int64_t row = t0 + (it + k * step) / (kRows / 4);
#pragma unroll
                        for (int c = 0; c < kSums; ++c)
                            *reinterpret_cast<uint4 *>(P.raw + (((int64_t)group * (GATED ? 2 : P.problems) + (GATED ? c : problem)) * P.f.M + row) *
                                                                   P.raw_ld + n0 + j) = acc[k][c];
                        continue;
                    }
                    const uint32_t g[4] = {acc[k][0].x, acc[k][0].y, acc[k][0].z, acc[k][0].w};
                    const uint4 w = acc[k][GATED ? 1 : 0];
                    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
                    finish4<INT8, GATED>(P.f, problem, t0 + (it + k * step) / (kRows / 4), n0 + j, g, u);
                }
            }
    }
    if (P.split > 1) {
        __syncwarp();
        cluster_sync();         // the sums stay until every CTA has read them
    }
}

// What the groups of a product left: their sums, and whether each cluster's are complete.
struct Joint {
    const uint32_t *raw, *whole;
    int64_t ld;                                  // of raw
    int groups, problems, tokens, token_tiles, row_tiles;
};

// Adds the groups' sums in group order and finishes.  A thread: four columns of a row.  Where a group gave up a wait
// its sums are not there, and the results stay as they were.
template <bool INT8, bool GATED>
__global__ void __launch_bounds__(256)
finish_kernel(const __grid_constant__ Finish F, const __grid_constant__ Joint J)
{
    const int64_t n = 4 * ((int64_t)blockIdx.x * 64 + threadIdx.x % 64);      // a warp's columns lie in one row tile
    const int planes = GATED ? 2 : J.problems, problem = GATED ? 0 : blockIdx.z, lane = threadIdx.x % 32;
    const bool in = n < F.N;
    grid_wait();
    grid_release();
    if (n - 4 * lane >= F.N) return;
    for (int64_t m = (int64_t)blockIdx.y * 4 + threadIdx.x / 64; m < F.M; m += (int64_t)gridDim.y * 4) {
        // the groups' words, a lane each
        const int64_t word = (((int64_t)lane * J.problems + problem) * J.token_tiles + (int)m / J.tokens) * J.row_tiles + n / kRows;
        const bool complete = lane >= J.groups || J.whole[word] != 0;
        uint4 acc[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
        if (in) {
#pragma unroll
            for (int c = 0; c < (GATED ? 2 : 1); ++c) {
                const uint4 *p = reinterpret_cast<const uint4 *>(J.raw + ((GATED ? c : problem) * F.M + m) * J.ld + n);
                const int64_t next = planes * F.M * J.ld / 4;
                acc[c] = __ldcs(p);
#pragma unroll 4
                for (int g = 1; g < J.groups; ++g) acc[c] = add4<INT8>(acc[c], __ldcs(p + g * next));
            }
        }
        if (!__all_sync(0xffffffffu, complete) || !in) continue;
        const uint4 w = acc[GATED ? 1 : 0];
        const uint32_t g[4] = {acc[0].x, acc[0].y, acc[0].z, acc[0].w}, u[4] = {w.x, w.y, w.z, w.w};
        finish4<INT8, GATED>(F, problem, m, n, g, u);
    }
}

// The instantiations, by number.
enum Form { kLinear8, kGated8, kGated16, kSum16, kPair16, kLinear16 };

Form form_of(const Product &p)
{
    if (p.kind == kProductInt8) return p.form == Product::kGated ? kGated8 : kLinear8;
    if (p.form == Product::kSingle) return p.b[0].mn_major ? kSum16 : kLinear16;      // a sum of one product
    return p.form == Product::kGated ? kGated16 : p.form == Product::kPair ? kPair16 : kSum16;
}

const void *kernel_of(Form form, bool loose)
{
    switch (form) {
        case kLinear8: return loose ? (const void *)&product_stream_kernel<true, false, false, false, true>
                                    : (const void *)&product_stream_kernel<true, false, false, false, false>;
        case kGated8: return loose ? (const void *)&product_stream_kernel<true, true, false, false, true>
                                   : (const void *)&product_stream_kernel<true, true, false, false, false>;
        case kGated16: return loose ? (const void *)&product_stream_kernel<false, true, false, false, true>
                                    : (const void *)&product_stream_kernel<false, true, false, false, false>;
        case kSum16: return loose ? (const void *)&product_stream_kernel<false, false, true, false, true>
                                  : (const void *)&product_stream_kernel<false, false, true, false, false>;
        case kLinear16: return loose ? (const void *)&product_stream_kernel<false, false, false, false, true>
                                     : (const void *)&product_stream_kernel<false, false, false, false, false>;
        default: return (const void *)&product_stream_kernel<false, false, true, true, false>;
    }
}

// Clusters of 1 ... 8 CTAs, one CTA an SM, that fit the device at once ([split]; 0: none, or the query failed).  For a
// kernel that allocates TMEM the query never counts more than one CTA an SM, whatever its size; two of this kernel's
// were seen to run side by side where its shared memory allows it, so the caller multiplies.  The query is slow, so its
// answers are kept for each device and kernel; a failure is not kept, the next call asks again.
struct Resident {
    int clusters[kMaxSplit + 1];
};

Resident resident(Form form, bool loose)
{
    static std::mutex mu;
    static Resident known[64][2 * (kLinear16 + 1)];
    static std::atomic<bool> answered[64][2 * (kLinear16 + 1)];
    Resident r = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return r;
    Resident &kept = known[dev][2 * form + loose];
    std::atomic<bool> &done = answered[dev][2 * form + loose];
    if (done.load(std::memory_order_acquire)) return kept;
    std::lock_guard<std::mutex> lock(mu);
    if (done.load(std::memory_order_relaxed)) return kept;
    const void *func = kernel_of(form, loose);
    bool all = true;
    for (int split = 1; split <= kMaxSplit; ++split) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)split, 1, 1);
        cfg.blockDim = dim3(threads_of(loose), 1, 1);
        cfg.dynamicSmemBytes = kWhole;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = (unsigned)split; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        if (test_fail_queries() || cudaFuncSetAttribute(func, cudaFuncAttributeMaxDynamicSharedMemorySize, kWhole) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&r.clusters[split], func, &cfg) != cudaSuccess) {
            cudaGetLastError();
            r.clusters[split] = 0;
            all = false;
        }
    }
    if (all) {
        kept = r;
        done.store(true, std::memory_order_release);
    }
    return r;
}

struct StreamPlan {
    bool loose;
    int tokens, halves, k_blocks, parts, stages, raw_stages, split, groups, smem;
    int64_t row_tiles, token_tiles;
    size_t raw_bytes, whole_bytes;      // of the sums that groups leave, and of the words that say whether they are complete
    double us;             // estimate
};

StreamPlan plan_stream(const Product &p)
{
    const Form form = form_of(p);
    const bool int8 = p.kind == kProductInt8, gated = p.form == Product::kGated, w_mn = p.b[0].mn_major;
    const int e = int8 ? 1 : 2, block_k = int8 ? 128 : 64, sums = gated ? 2 : 1;
    StreamPlan s = {};
    s.k_blocks = (int)((p.K + block_k - 1) / block_k);
    s.parts = p.form == Product::kSum ? 2 : 1;
    const int problems = p.form == Product::kPair ? 2 : 1;
    s.tokens = p.M <= 16 ? 16 : p.M <= 32 ? 32 : p.M <= 64 ? 64 : 128;
    if (problems > 1 && s.tokens < 64) s.tokens = 64;        // whole boxes of 64 columns
    s.halves = p.lo[0].p ? 2 : 1;
    s.loose = !(taken_as_is(p.a[0], e) && taken_as_is(p.a[1], e) && taken_as_is(p.b[0], e) && taken_as_is(p.b[1], e));
    if ((s.loose || s.halves > 1) && problems > 1) return s;         // not built: the tile kernel's
    s.row_tiles = (p.N + kRows - 1) / kRows;
    s.token_tiles = (p.M + s.tokens - 1) / s.tokens;
    const int columns = s.halves * s.tokens, stage = sums * kWeightBytes + columns * 128, exchange = sums * columns * kRows * 4;
    const int fixed = kBarBytes + 1024, half = kHalf - fixed, whole = kWhole - fixed;
    const int raw = sums * (w_mn ? 64 * kRawPitch<2> : kRows * kRawPitch<1>) + columns * kRawPitch<1>;       // LOOSE: of a stage
    const int64_t work = s.row_tiles * s.token_tiles * problems;
    const int blocks = s.k_blocks * s.parts;
    const double hbm = (double)p.N * (double)p.K * e * sums * s.parts / 9.0e6;
    const double plane = (double)p.M * (double)((p.N + 3) / 4 * 16) * sums * problems;       // bytes of a group's sums
    const Resident res = resident(form, s.loose);
    // Two CTAs an SM where two stages and the exchange fit half of its shared memory, or one; the split over a
    // cluster, and over clusters, that takes the least time.  A CTA draws its stages at what its ring holds in 0.84 us,
    // at most 174 KB/us an SM (LOOSE: it shifts 12 - 18); an end of 128 columns takes it 3.2 us (gated 1.7 times
    // that), 1.1 of them shared by the cluster, besides 2.5 us of latencies and 0.19 a CTA it exchanges with; the weights'
    // way from HBM comes on top (9 TB/s: what is not hidden of it), and 0.3 us where no CTA of the next kernel has room.
    // Fitted to 52 sizes (896 ... 11008, 1 ... 256 tokens) x 16 plans, off by 3 % near the best ones: what it chooses takes
    // 2 % more than the best plan, where rules without the rings' depth took 8 % (8-bit 4096 x 4096, 64 tokens: clusters of
    // four 9.1, of six 10 us; gated 4096 x 11008, 64 tokens: two CTAs an SM of two stages 36 us, one of five 42).  The
    // worst choices found: gated 2560 x 6912, 64 tokens, 22 us where 18 were possible; dx of 4096 x 11008, one token, 38 and 33 us.
    // Groups write their sums and another kernel reads them.
    for (int per_sm = s.loose ? 1 : 2; per_sm >= 1; --per_sm) {
        const int room = per_sm == 2 ? half : whole;
        int stages, raw_stages = 0, used;
        if (s.loose) {
            stages = 3 * stage + 3 * raw <= room ? 3 : 2;
            raw_stages = (room - stages * stage) / raw < 6 ? (room - stages * stage) / raw : 6;
            used = stages * stage + raw_stages * raw;
        } else {
            stages = room / stage < kMaxStages ? room / stage : kMaxStages;
            used = stages * stage;
        }
        if (stages < 2 || exchange > room) continue;
        for (int n = 1; n <= kMaxSplit && n <= blocks; ++n) {
            const int fit = per_sm * res.clusters[n];
            if (fit < 1) continue;
            for (int g = 1; g <= 16 && n * g * (g > 1 ? 4 : 1) <= blocks && (g == 1 || g * plane < 64e6); g *= 2) {
                const double rounds = (double)((work * g + fit - 1) / fit), steps = (double)((blocks + n * g - 1) / (n * g));
                const double most = 174e3 / (per_sm == 2 && work * n * g > sm_count() ? 2 : 1), ring = (double)stages * stage / 0.84;
                const double stage_us = stage / (s.loose ? (w_mn ? 12e3 : 18e3) : ring < most ? ring : most);
                const double finish = 2.5 + columns / 128.0 * (gated ? 1.7 : 1.0) * (3.2 + 1.1 / n) + 0.19 * (n - 1);
                const double us = (s.loose ? 2.0 : 1.0) + hbm + rounds * (steps * stage_us + finish) + (per_sm == 1 ? 0.3 : 0.0) +
                                  (g > 1 ? 4.0 + 2 * g * plane / 4.0e6 : 0.0);
                if (s.split == 0 || us < s.us * (g > 1 ? 0.9 : 1.0)) {
                    s.split = n;
                    s.groups = g;
                    s.us = us;
                    s.stages = stages;
                    s.raw_stages = raw_stages;
                    s.smem = fixed + (used > exchange ? used : exchange);
                }
            }
        }
    }
    if (s.groups > 1) {
        s.raw_bytes = (size_t)s.groups * (size_t)plane;
        s.whole_bytes = (size_t)(s.groups * work) * 4;
    }
    return s;
}

}  // namespace

double stream_estimate(const Product &p)
{
    const StreamPlan s = plan_stream(p);
    return s.split > 0 && s.row_tiles <= 65535 && s.token_tiles <= 65535 / 32 ? s.us : -1.0;
}

size_t stream_workspace_bytes(const Product &p)
{
    const StreamPlan s = plan_stream(p);
    return s.raw_bytes + s.whole_bytes;
}

int launch_product_stream(const Product &p, const Finish &f, void *workspace, cudaStream_t stream)
{
    const bool int8 = p.kind == kProductInt8, gated = p.form == Product::kGated, w_mn = p.b[0].mn_major;
    const int e = int8 ? 1 : 2;
    const StreamPlan plan = plan_stream(p);
    if (plan.split == 0) return LORDBA_ECUDA;
    if (plan.row_tiles > 65535 || plan.token_tiles > 65535 / 32) return LORDBA_EUNSUPPORTED;
    const bool t_mn = p.a[0].mn_major;
    StreamArgs a;
    std::memset(&a, 0, sizeof(a));
    a.f = f;
    a.k_blocks = plan.k_blocks;
    a.parts = plan.parts;
    a.tokens = plan.tokens;
    a.halves = plan.halves;
    a.token_tiles = (int)plan.token_tiles;
    a.problems = p.form == Product::kPair ? 2 : 1;
    a.groups = plan.groups;
    a.raw = static_cast<uint32_t *>(workspace);
    a.raw_ld = (p.N + 3) / 4 * 4;
    a.whole = reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(workspace) + plan.raw_bytes);
    a.stages = plan.stages;
    a.raw_stages = plan.raw_stages;
    a.split = plan.split;
    for (int i = 0; i < 2; ++i) {
        const Operand &ot = p.a[i], &ow = p.b[i];
        const int64_t w_rows = w_mn ? p.K : p.N, w_cols = w_mn ? p.N : p.K;
        a.rt[i] = Rows{static_cast<const uint8_t *>(ot.p), ot.ld * e, p.M, p.K * e};
        a.rw[i] = Rows{static_cast<const uint8_t *>(ow.p), ow.ld * e, w_rows, w_cols * e};
        const Operand &ol = p.lo[i];
        a.rt[2 + i] = Rows{static_cast<const uint8_t *>(ol.p), ol.ld * e, p.M, p.K * e};
        if (plan.loose) continue;
        if (ol.p && !encode_map(&a.t[2 + i], ol.p, p.M, p.K, ol.ld, e, a.tokens)) return LORDBA_ECUDA;
        if (ot.p && !(t_mn ? encode_map(&a.t[i], ot.p, p.K, p.M, ot.ld, e, 64) : encode_map(&a.t[i], ot.p, p.M, p.K, ot.ld, e, a.tokens)))
            return LORDBA_ECUDA;
        if (ow.p && !encode_map(&a.w[i], ow.p, w_rows, w_cols, ow.ld, e, w_mn ? 64 : kRows)) return LORDBA_ECUDA;
    }
    a.tmem_columns = 32;
    while (a.tmem_columns < (gated ? 2 : 1) * a.halves * a.tokens) a.tmem_columns *= 2;
    a.skip = test_skip_item();
    a.status = device_status_word();
    if (!a.status) return LORDBA_ECUDA;
    a.idesc = instr_desc(int8, p.kind == kProductBf16, w_mn, t_mn, kRows, a.halves * a.tokens);
    LaunchRec rec;
    std::memset(&rec, 0, sizeof(rec));
    rec.func = kernel_of(form_of(p), plan.loose);
    rec.grid[0] = (unsigned)plan.split; rec.grid[1] = (unsigned)plan.row_tiles; rec.grid[2] = (unsigned)(plan.token_tiles * a.problems * plan.groups);
    rec.block = threads_of(plan.loose);
    rec.smem = (uint32_t)plan.smem;
    rec.cluster = (uint32_t)plan.split;
    rec.pdl = 1;
    rec.n_args = 1;
    rec.arg_bytes[0] = sizeof(StreamArgs);
    const int rc = launch_record(rec, &a, nullptr, stream);
    if (rc != LORDBA_OK || plan.groups == 1) return rc;
    const int64_t gx = (p.N + 255) / 256, gy = (p.M + 3) / 4, most = gx >= 148 * 32 ? 1 : 148 * 32 / gx;
    const dim3 grid((unsigned)gx, (unsigned)(gy < most ? gy : most), (unsigned)a.problems);
    const auto kernel = int8 ? (gated ? finish_kernel<true, true> : finish_kernel<true, false>)
                             : (gated ? finish_kernel<false, true> : finish_kernel<false, false>);
    const Joint joint{a.raw, a.whole, a.raw_ld, plan.groups, a.problems, plan.tokens, a.token_tiles, (int)plan.row_tiles};
    return launch_kernel(kernel, grid, 256, 0, stream, f, joint);
}

}  // namespace lordba
