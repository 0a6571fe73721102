// Distillation from a teacher's top logits: the loss of a row, its log-sum, and the gradient to the student's logits.
//
// Bound: HBM.  A row's logits are read once, and for the gradient written once.  Eight 16-byte pieces a thread are on the way before
// the first is looked at.  A row that fits stays in a CTA's registers in between, or, where rows are few, in those of a cluster of
// up to eight, which exchange maxima and sums through distributed shared memory; a longer one goes by against a running maximum,
// and for the gradient comes a second time, from L2.  A thousand threads an SM, in CTAs as small as a row allows: while some
// wait for a row to arrive or for one another, others calculate or write.
//
// Persistent CTAs that had the copy engine fetch rows ahead, with a row's exponentials kept in registers between the passes,
// were slower (4096 x 131072 in bf16 1190 us, this 438; 2048 x 32000 128 and 68): a row is a chain of latencies for the warps that
// share it, and what hides it is many rows at a time.  The fullest unit is the one of the exponentials (59 % of its rate, 2048 x 32000), and warps
// wait most for a row to arrive; no unit alone bounds it.
//
// Pieces lie on 16-byte boundaries whatever the row's alignment is: the first and last are masked, and results that lie
// otherwise are joined from the pieces of neighbouring lanes.
//
// The exponentials are powers of two of  (z - max) log2(e)/temperature : a difference and a product (of two at a time) and one
// instruction each.  The difference comes first: a product of max and the factor, subtracted in one multiply-add, would leave its rounding
// in every exponent, and of very low numbers (a mask's) an infinity.
//
// The teacher's part of a row (softmax of the top entries, the student's logits there) is a chain of latencies too: for many rows a
// kernel of its own goes through it first.
#include <cstring>
#include <type_traits>

#include "block_checks.h"
#include "product_internal.cuh"

namespace lordba {
namespace {

using namespace sm100;

constexpr int kHeld = 8;                  // pieces a thread keeps
constexpr int kMaxSplit = 8, kMaxThreads = 512;
// Rows up to which each does its teacher's part itself: a chain of accesses that wait for one another, 2 us where the GPU is
// idle, but more than twice that among other rows' traffic, where a kernel of its own before (one more launch, 1.5 us) pays.
constexpr int64_t kDistillAlone = 128;
constexpr float kLog2E = 1.4426950408889634f;
enum Mode { kLoss, kStep, kBack };

struct DistillArgs {
    const void *logits, *ids, *teacher;
    const float *weight;
    float *loss, *lse;
    void *dlogits;
    int64_t ld_logits, ld_ids, ld_teacher, ld_dlogits, vocab;
    int top, ids64, teacher_dtype;
    int split, split_log2, part;          // CTAs a row, a power of two; classes of one
    int table;                            // entries of the hash table of classes: a power of two, at least twice `top`
    float temperature, inverse, scale;    // scale: log2(e) / temperature
    uint4 *entries;                       // of all rows, as the teacher's kernel leaves them, or null
    uint2 *heads;
};

__device__ __forceinline__ float exp2_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A sum of 2^(scale (z - max)) and the max it is relative to.
struct Stat {
    float max, sum;
};

// One of the teacher's top classes: its probability there and the logarithm of it, the student's logit.
struct __align__(16) Entry {
    int id;
    float p, log, z;
};
struct Head {
    float sum;
    int twice;
};

// The logits of a piece.
template <typename E>
__device__ __forceinline__ void unpack_chunk(uint4 w, Two v[8 / sizeof(E)])
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i) v[i] = two(__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack2<E>(u[i]);
            v[i] = two(f.x, f.y);
        }
    }
}
// What does not belong to the group's part of the row becomes minus infinity.
template <typename E>
__device__ __noinline__ uint4 mask_chunk(uint4 w, int chunk, int off, int count)
{
    constexpr int N = 16 / sizeof(E);
    uint32_t u[4] = {w.x, w.y, w.z, w.w};
    const int base = chunk * N - off / (int)sizeof(E);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (base + i >= 0 && base + i < count) continue;
        if (sizeof(E) == 4) u[i] = 0xff800000u;
        else {
            const uint32_t low = std::is_same_v<E, __half> ? 0xfc00u : 0xff80u;
            u[i / 2] = i % 2 ? (u[i / 2] & 0xffffu) | low << 16 : (u[i / 2] & 0xffff0000u) | low;
        }
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}
// The larger of each entry, where one is NaN the other.
template <typename E>
__device__ __forceinline__ void top_of_chunk(uint4 w, uint32_t top[sizeof(E) == 4 ? 1 : 2])
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) top[0] = __float_as_uint(fmaxf(__uint_as_float(top[0]), __uint_as_float(u[i])));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (std::is_same_v<E, __half>) asm("max.f16x2 %0, %0, %1;" : "+r"(top[i % 2]) : "r"(u[i]));
            else asm("max.bf16x2 %0, %0, %1;" : "+r"(top[i % 2]) : "r"(u[i]));
        }
    }
}

template <typename E>
__device__ __forceinline__ uint4 pack_chunk(const Two v[8 / sizeof(E)])
{
    const float2 a = halves(v[0]), b = halves(v[1]);
    if constexpr (sizeof(E) == 4) return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
    else {
        const float2 c = halves(v[2]), d = halves(v[3]);
        return make_uint4(pack2<E>(a.x, a.y), pack2<E>(b.x, b.y), pack2<E>(c.x, c.y), pack2<E>(d.x, d.y));
    }
}
// Bytes [from, to) of a piece to the address that its first byte has, element by element.
template <typename E>
__device__ __noinline__ void store_part(uint8_t *at, uint4 w, int from, int to)
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 16 / (int)sizeof(E); ++i) {
        const int b = i * (int)sizeof(E);
        if (b < from || b >= to) continue;
        if (sizeof(E) == 4) *reinterpret_cast<uint32_t *>(at + b) = u[i];
        else *reinterpret_cast<uint16_t *>(at + b) = (uint16_t)(u[i / 2] >> 16 * (i % 2));
    }
}
// A warp's 32 neighbouring pieces to memory.  `at`: where the lane's piece goes; by: at's distance from the last 16-byte
// boundary, the same for all lanes; begin, end: the bytes of the piece that exist.  Off the boundaries a lane joins the end
// of its piece and the beginning of its neighbour's.
template <typename E>
__device__ __forceinline__ void store_chunks(uint8_t *at, uint4 w, int by, int begin, int end, int lane)
{
    if (by == 0) {
        if (begin == 0 && end == 16) *reinterpret_cast<uint4 *>(at) = w;
        else if (begin < end) store_part<E>(at, w, begin, end);
        return;
    }
    uint4 next;
    next.x = __shfl_down_sync(0xffffffffu, w.x, 1); next.y = __shfl_down_sync(0xffffffffu, w.y, 1);
    next.z = __shfl_down_sync(0xffffffffu, w.z, 1); next.w = __shfl_down_sync(0xffffffffu, w.w, 1);
    const bool whole = begin == 0 && end == 16;
    const unsigned all = __ballot_sync(0xffffffffu, whole);
    const bool before = lane > 0 && (all >> (lane - 1) & 1u), after = lane < 31 && (all >> (lane + 1) & 1u);
    if (whole && after) *reinterpret_cast<uint4 *>(at + 16 - by) = join_pieces(w, next, 16 - by);
    // what no neighbour takes along
    const int head = whole && before ? 16 - by : begin, tail = whole && after ? 16 - by : end;
    if (head < tail) store_part<E>(at, w, head, tail);
}

// The teacher's entries of a row, by one warp, into shared memory.  sum: 0 where no entry has a chance; twice: whether a
// class stands there twice (a hash table of `slots` classes says so).
template <typename E>
__device__ __forceinline__ Head teacher_of(const DistillArgs &A, int64_t t, Entry *top, int *table, int slots, int lane)
{
    const E *z = static_cast<const E *>(A.logits) + t * A.ld_logits;
    for (int i = lane; i < slots; i += 32) table[i] = -1;
    __syncwarp();
    float most = -INFINITY;
    bool met = false;
#pragma unroll 2
    for (int j = lane; j < A.top; j += 32) {
        const int64_t k = A.ids64 ? static_cast<const int64_t *>(A.ids)[t * A.ld_ids + j] : (int64_t)static_cast<const int32_t *>(A.ids)[t * A.ld_ids + j];
        const int64_t at = t * A.ld_teacher + j;
        float v = A.teacher_dtype == LORDBA_F32    ? static_cast<const float *>(A.teacher)[at]
                  : A.teacher_dtype == LORDBA_BF16 ? to_float(static_cast<const __nv_bfloat16 *>(A.teacher)[at])
                                                   : to_float(static_cast<const __half *>(A.teacher)[at]);
        const bool in = k >= 0 && k < A.vocab;
        if (!in) v = -INFINITY;
        top[j] = Entry{in ? (int)k : -1, 0.0f, v, in ? to_float(z[k]) : 0.0f};
        most = fmaxf(most, v);
        for (uint32_t h = (uint32_t)k * 2654435769u; in; ++h) {
            const int was = atomicCAS(&table[h & (slots - 1)], -1, (int)k);
            met |= was == (int)k;
            if (was == -1 || was == (int)k) break;
        }
    }
    for (int o = 16; o; o /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    float sum = 0.0f;                      // a NaN comes through here
    for (int j = lane; j < A.top; j += 32) {
        const float v = top[j].log, x = v == -INFINITY ? v : __fdiv_rn(v - most, A.temperature), e = expf(x);
        top[j].log = x;
        top[j].p = e;
        sum += e;
    }
    for (int o = 16; o; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float log_sum = logf(sum), inverse = 1.0f / sum;
    for (int j = lane; j < A.top; j += 32) {
        top[j].p = top[j].log == -INFINITY ? 0.0f : top[j].p * inverse;
        top[j].log -= log_sum;
    }
    const Head h{sum, (int)__any_sync(0xffffffffu, met)};
    __syncwarp();
    return h;
}

// The teacher's part of every row, a warp each, for the kernel below.
template <typename E>
__global__ void __launch_bounds__(128)
distill_teacher_kernel(const __grid_constant__ DistillArgs A, int64_t T)
{
    extern __shared__ __align__(16) uint8_t own[];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int64_t t = (int64_t)blockIdx.x * 4 + warp;
    Entry *top = reinterpret_cast<Entry *>(own) + warp * A.top;
    int *table = reinterpret_cast<int *>(own + 4 * A.top * sizeof(Entry)) + warp * A.table;
    grid_wait();
    grid_release();
    if (t >= T) return;
    const Head h = teacher_of<E>(A, t, top, table, A.table, lane);
    for (int j = lane; j < A.top; j += 32) A.entries[t * A.top + j] = *reinterpret_cast<const uint4 *>(top + j);
    if (lane == 0) A.heads[t] = make_uint2(__float_as_uint(h.sum), (uint32_t)h.twice);
}

// Loss and lse of a row, by one warp.
__device__ __forceinline__ void loss_of(const DistillArgs &A, int64_t t, const Entry *top, Stat all, float weight, bool live, int lane)
{
    // log p - log q from what is left of both maxima: neither lse nor a logit of its size enters
    const float log_sum = logf(all.sum);
    float loss = 0.0f;
    for (int j = lane; j < A.top; j += 32)
        if (top[j].p != 0.0f) loss += top[j].p * (top[j].log - ((top[j].z - all.max) * A.inverse - log_sum));
    for (int o = 16; o; o /= 2) loss += __shfl_xor_sync(0xffffffffu, loss, o);
    if (lane == 0) {
        A.lse[t] = all.max * A.inverse + log_sum;
        A.loss[t] = live ? weight * A.temperature * A.temperature * loss : 0.0f;
    }
}

// The gradients of the teacher's entries, every `by`-th from `at` on, over what was put there.  probability: the student's, of a logit.
template <typename E, typename F>
__device__ __forceinline__ void patch_row(const DistillArgs &A, int64_t t, int first, int count, const Entry *top, bool twice, float factor,
                                          F probability, int at, int by)
{
    E *dz = static_cast<E *>(A.dlogits) + t * A.ld_dlogits;
    for (int j = at; j < A.top; j += by) {
        const Entry e = top[j];
        if (e.id < first || e.id >= first + count) continue;
        float p = e.p;
        if (twice) {                       // a class that stands there twice: both write the same value
            p = 0.0f;
            for (int k = 0; k < A.top; ++k) p += top[k].id == e.id ? top[k].p : 0.0f;
        }
        dz[e.id] = from_float<E>(factor * (probability(e.z) - p));
    }
}

// The sides of LANES neighbouring lanes joined, in every one of them the same bits.
template <int LANES>
__device__ __forceinline__ Stat over_lanes(Stat s, float scale)
{
    float m = s.max;
    if constexpr (LANES == 32) asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(s.max));
    else
#pragma unroll
        for (int o = LANES / 2; o; o /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    float sum = s.sum * exp2_of((s.max - (m == -INFINITY ? 0.0f : m)) * scale);
#pragma unroll
    for (int o = LANES / 2; o; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return Stat{m, sum};
}


// ALONE: the row's first warp does the teacher's part itself; otherwise distill_teacher_kernel has done it for all rows.  HELD:
// the registers have room for the CTA's part of the row; otherwise it goes by, half of the pieces at a time, whose successors are asked
// for at once, against a running maximum, and for the gradient once more (it comes from L2 then).
template <typename E, int MODE, int THREADS, bool ALONE, bool HELD>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS)
distill_kernel(const __grid_constant__ DistillArgs A)
{
    extern __shared__ __align__(16) uint8_t own[];
    constexpr int N = 16 / (int)sizeof(E), kWarps = THREADS / 32, kHalf = kHeld / 2;
    constexpr uint32_t kLow = sizeof(E) == 4 ? 0xff800000u : std::is_same_v<E, __half> ? 0xfc00fc00u : 0xff80ff80u;
    __shared__ Stat part[kWarps], peers[kMaxSplit];
    __shared__ Head head;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int64_t t = blockIdx.x >> A.split_log2;
    const int rank = blockIdx.x & (A.split - 1);
    Entry *top = reinterpret_cast<Entry *>(own);

    // the CTA's part of the row, and the 16-byte pieces that hold it
    const int first = rank * A.part, count = (int)A.vocab - first < A.part ? (int)A.vocab - first : A.part;
    const uintptr_t row = reinterpret_cast<uintptr_t>(static_cast<const E *>(A.logits) + t * A.ld_logits + first);
    const int off = (int)(row & 15), last = off + count * (int)sizeof(E), chunks = (last + 15) / 16;
    const uint4 *in = reinterpret_cast<const uint4 *>(row - off) + tid;
    const int pieces = (chunks - (tid - lane) + THREADS - 1) / THREADS;      // of the warp's first lane
    const bool edges = off || last % 16;
    auto mask = [&](uint4 w, int c) {
        if (edges && (c == 0 || c == chunks - 1)) w = mask_chunk<E>(w, c, off, count);
        return w;
    };
    // Logits too wait for the end of all kernels before.  Reading them while the teacher's kernel still runs gained a microsecond for the loss of
    // 2048 x 32000 and lost ten of 4096 x 131072 with gradient.
    grid_wait();
    grid_release();
    if (MODE != kBack && A.split > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");    // this CTA runs
    auto piece = [&](int i) { return tid + THREADS * i < chunks ? __ldcg(in + THREADS * i) : make_uint4(kLow, kLow, kLow, kLow); };
    // for the last time: other rows may take its place in L2
    auto last_piece = [&](int i) { return MODE != kStep ? piece(i) : tid + THREADS * i < chunks ? __ldcs(in + THREADS * i) : make_uint4(kLow, kLow, kLow, kLow); };
    uint4 raw[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) raw[i] = piece(i);
    const float weight = A.weight ? A.weight[t] : 1.0f;
    if constexpr (ALONE) {
        if (warp == 0) {
            const Head h = teacher_of<E>(A, t, top, reinterpret_cast<int *>(top + A.top), A.table, lane);
            if (lane == 0) head = h;
        }
    } else {
        for (int j = tid; j < A.top; j += THREADS) *reinterpret_cast<uint4 *>(top + j) = __ldcg(A.entries + t * A.top + j);
        if (tid == 0) {
            const uint2 h = __ldcg(A.heads + t);
            head = Head{__uint_as_float(h.x), (int)h.y};
        }
    }
    Stat all = {0.0f, 1.0f};
    if (MODE != kBack) {
        uint32_t most[2] = {kLow, kLow};
        Stat s;
        auto largest = [&] {
            if constexpr (sizeof(E) == 4) return __uint_as_float(most[0]);
            else {
                const float2 x = unpack2<E>(most[0]), y = unpack2<E>(most[1]);
                return fmaxf(fmaxf(x.x, x.y), fmaxf(y.x, y.y));
            }
        };
        const Two scales = two(A.scale, A.scale);
        Two minuses, sums[2] = {two(0.0f, 0.0f), two(0.0f, 0.0f)};
        // sums are relative to the largest logit so far itself, or to 0 where that is minus infinity
        auto relative_to = [&](float max) {
            const float minus = max == -INFINITY ? 0.0f : -max;
            minuses = two(minus, minus);
            return minus;
        };
        auto add = [&](uint4 w) {
            Two v[N / 2];
            unpack_chunk<E>(w, v);
#pragma unroll
            for (int j = 0; j < N / 2; ++j) {
                const float2 x = halves(mul_two(add_two(v[j], minuses), scales));
                sums[j % 2] = add_two(sums[j % 2], two(exp2_of(x.x), exp2_of(x.y)));
            }
        };
        if constexpr (!HELD) {
            s.max = -INFINITY;
            for (int base = 0; base < pieces; base += kHeld) {
#pragma unroll
                for (int h = 0; h < kHeld; h += kHalf) {
                    if (base + h >= pieces) break;
#pragma unroll
                    for (int i = h; i < h + kHalf; ++i) {
                        raw[i] = mask(raw[i], tid + THREADS * (base + i));
                        top_of_chunk<E>(raw[i], most);
                    }
                    const float was = s.max;
                    s.max = largest();
                    const float kept = exp2_of((was + relative_to(s.max)) * A.scale);          // 1 where the maximum stays
#pragma unroll
                    for (int j = 0; j < 2; ++j) sums[j] = mul_two(sums[j], two(kept, kept));
#pragma unroll
                    for (int i = h; i < h + kHalf; ++i) {
                        add(raw[i]);
                        raw[i] = piece(base + kHeld + i);
                    }
                }
            }
            if (MODE == kStep) {
#pragma unroll
                for (int i = 0; i < kHeld; ++i) raw[i] = last_piece(i);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kHeld; ++i) {
                if (i >= pieces) break;
                raw[i] = mask(raw[i], tid + THREADS * i);
                top_of_chunk<E>(raw[i], most);
            }
            s.max = largest();
            relative_to(s.max);
#pragma unroll
            for (int i = 0; i < kHeld; ++i) {
                if (i >= pieces) break;
                add(raw[i]);
            }
        }
        const float2 sum = halves(add_two(sums[0], sums[1]));
        s.sum = sum.x + sum.y;
        s = over_lanes<32>(s, A.scale);
        if (lane == 0) part[warp] = s;
        __syncthreads();
        s = over_lanes<kWarps>(part[lane % kWarps], A.scale);
        if (A.split > 1) {
            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
            if (warp == 0 && lane < A.split) {
                const uint32_t to = peer_addr(smem_addr(&peers[rank]), lane);
                store_peer(to, __float_as_uint(s.max));
                store_peer(to + 4, __float_as_uint(s.sum));
            }
            __syncwarp();
            // what the first warps have pushed is all that the peers must see
            if (warp == 0) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
            else asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
            s = over_lanes<kMaxSplit>(lane % kMaxSplit < A.split ? peers[lane % kMaxSplit] : Stat{-INFINITY, 0.0f}, A.scale);
        }
        all = s;
    } else {
        __syncthreads();
    }
    const bool live = weight != 0.0f && head.sum != 0.0f;
    if (MODE != kBack && rank == 0 && warp == 0) loss_of(A, t, top, all, weight, live, lane);
    if (MODE == kLoss) return;
    // The student's probabilities: 2^((z - max) log2(e)/temperature - log2(sum)), or from lse 2^((z/temperature - lse) log2(e)).  As in the sums the
    // large numbers meet first, and what is left of them is scaled.
    const float less = MODE != kBack ? -all.max : -A.lse[t], log_sum = MODE != kBack ? -log2f(all.sum) : 0.0f;
    auto exponents = [&](Two v) {
        if constexpr (MODE != kBack) return fma_two(add_two(v, two(less, less)), two(A.scale, A.scale), two(log_sum, log_sum));
        else return mul_two(fma_two(v, two(A.inverse, A.inverse), two(less, less)), two(kLog2E, kLog2E));
    };
    auto probability = [&](float z) { return exp2_of(halves(exponents(two(z, z))).x); };
    const float factor = weight * A.temperature;
    const Two times = two(factor, factor);
    uint8_t *to = reinterpret_cast<uint8_t *>(static_cast<E *>(A.dlogits) + t * A.ld_dlogits + first) - off + 16 * tid;
    const int by = (int)(reinterpret_cast<uintptr_t>(to) & 15);
    const bool plain = by == 0 && !edges;             // whole pieces alone
    auto put = [&](uint4 w, int c) {
        Two v[N / 2];
        unpack_chunk<E>(w, v);
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
            const float2 x = halves(exponents(v[j]));
            v[j] = mul_two(two(exp2_of(x.x), exp2_of(x.y)), times);
        }
        w = pack_chunk<E>(v);
        if (!live) w = make_uint4(0, 0, 0, 0);                        // whatever stood there
        uint8_t *at = to + 16 * (c - tid);
        if (plain) {
            if (c < chunks) __stcs(reinterpret_cast<uint4 *>(at), w);
        } else {
            store_chunks<E>(at, w, by, c == 0 ? off : 0, last - 16 * c < 16 ? last - 16 * c : 16, lane);
        }
    };
    for (int base = 0; base < (HELD ? 1 : pieces); base += kHeld) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            if (base + i >= pieces) break;
            put(raw[i], tid + THREADS * (base + i));
            if (!HELD) raw[i] = last_piece(base + kHeld + i);
        }
    }
    if (!live) return;
    __syncthreads();                       // the teacher's entries' gradients go over what was put there
    if (warp * 32 < A.top) patch_row<E>(A, t, first, count, top, head.twice, factor, probability, tid, THREADS);
}

template <typename E, int MODE, bool ALONE, bool HELD>
const void *kernel_of(int threads)
{
    return threads == 64    ? reinterpret_cast<const void *>(&distill_kernel<E, MODE, 64, ALONE, HELD>)
           : threads == 128 ? reinterpret_cast<const void *>(&distill_kernel<E, MODE, 128, ALONE, HELD>)
           : threads == 256 ? reinterpret_cast<const void *>(&distill_kernel<E, MODE, 256, ALONE, HELD>)
                            : reinterpret_cast<const void *>(&distill_kernel<E, MODE, 512, ALONE, HELD>);
}
template <typename E, int MODE, bool ALONE>
const void *kernel_of(int threads, bool held)
{
    if constexpr (MODE == kLoss) return kernel_of<E, MODE, ALONE, false>(threads);
    else if (held) return kernel_of<E, MODE, ALONE, true>(threads);
    else if constexpr (MODE == kBack && !ALONE) return kernel_of<E, MODE, ALONE, false>(threads);
    else return reinterpret_cast<const void *>(&distill_kernel<E, MODE, kMaxThreads, ALONE, false>);
}

template <typename E, int MODE>
int launch_row(DistillArgs &A, int64_t T, cudaStream_t stream)
{
    // Of a row, or a CTA's part (whole 16 bytes of it): one more where it begins inside a piece.
    const bool inside = reinterpret_cast<uintptr_t>(A.logits) % 16 || (T > 1 && A.ld_logits * sizeof(E) % 16);
    auto part_of = [&](int split) { return (A.vocab + 8 * split - 1) / (8 * split) * 8; };
    auto pieces_of = [&](int split) {
        const int64_t part = part_of(split);
        return ((part < A.vocab ? part : A.vocab) * (int64_t)sizeof(E) + 15) / 16 + inside;
    };
    // With a row for every SM, one CTA each (two an SM, 512 threads) goes over rows that it cannot hold, unless a cluster holds them and
    // is filled: in CTAs of 256 threads then, where eight are enough.  Steps of 4096 x 131072 in bf16, inputs that change from call to
    // call, 438 us, gone by 429, held in CTAs of 512 threads 474; of 1024 x 131072 in f32 held 220, gone by 248; of 1500 x 160000 gone by
    // 215, held (not filled) 288; of 2048 x 50257 109 and 113.  Backward, which takes one pass, rows go by: 346, held 339; f32 182 and 170; 166 and 180;
    // 79 and 83; rows that a CTA could hold go by small CTAs as well where there are many of 16 KB and more (2048 x 32000 58 and 61).
    constexpr int64_t kRoom = kMaxThreads * kHeld;
    const bool many = T >= sm_count() && T > kDistillAlone;
    int split = 1;
    while (split < kMaxSplit && pieces_of(split) > kRoom) split *= 2;
    const bool filled = MODE == kStep && pieces_of(split) * 8 >= kRoom * 7;
    const bool small = MODE == kBack && T >= 4 * sm_count() && pieces_of(1) > 1024;
    const bool held = MODE != kLoss && pieces_of(split) <= kRoom && (!many || filled || (split == 1 && !small));
    if (!held && (MODE == kLoss || many)) split = 1;
    if (held && many && split > 1 && split < kMaxSplit) split *= 2;
    while (split < kMaxSplit && pieces_of(split) > 1 << 26) split *= 2;          // a part's bytes are counted in 32 bits
    // more CTAs a row while there are SMs without one and a CTA keeps a few kilobytes
    while (split < kMaxSplit && T * split * 2 <= sm_count() && pieces_of(1) >= 256 * split) split *= 2;
    if (T * split > 0x7fffffff) return LORDBA_EUNSUPPORTED;
    A.split = split;
    A.split_log2 = 0;
    while ((1 << A.split_log2) < split) ++A.split_log2;
    A.part = (int)part_of(split);
    const int64_t mine = pieces_of(split);
    // The smallest CTA that holds its part.  Of many rows that nothing of is held, small ones of several rounds: the gradient from lse of 2048 x 32000
    // 58 us, of one round 69, its loss 41 and 43; the loss of 4096 x 131072 182, with 512 threads 197.
    const int rounds = !many || held ? 1 : MODE == kLoss ? 4 : 2, most = MODE == kLoss && many ? kMaxThreads / 2 : kMaxThreads;
    int threads = 64;
    while (threads < most && mine > (int64_t)threads * kHeld * rounds) threads *= 2;
    const bool alone = T <= kDistillAlone;
    LaunchRec rec;
    std::memset(&rec, 0, sizeof(rec));
    rec.func = alone ? kernel_of<E, MODE, true>(threads, held) : kernel_of<E, MODE, false>(threads, held);
    rec.grid[0] = (unsigned)(T * split);
    rec.grid[1] = rec.grid[2] = 1;
    rec.block = (uint32_t)threads;
    rec.smem = (uint32_t)(A.top * sizeof(Entry) + (alone ? 4 * A.table : 0));
    rec.cluster = MODE == kBack ? 1 : (uint32_t)split;
    rec.pdl = 1;
    rec.n_args = 1;
    rec.arg_bytes[0] = sizeof(DistillArgs);
    return launch_record(rec, &A, nullptr, stream);
}

template <typename E, int MODE>
int launch_mode(DistillArgs &A, int64_t T, cudaStream_t stream)
{
    if (T > kDistillAlone) {
        const unsigned smem = 4u * (unsigned)(A.top * sizeof(Entry) + 4 * A.table);
        const int rc = launch_kernel(distill_teacher_kernel<E>, dim3((unsigned)((T + 3) / 4), 1, 1), 128, smem, stream, A, T);
        if (rc != LORDBA_OK) return rc;
    }
    return launch_row<E, MODE>(A, T, stream);
}

template <typename E>
int launch_typed(DistillArgs &A, int64_t T, bool backward, cudaStream_t stream)
{
    if (backward) return launch_mode<E, kBack>(A, T, stream);
    return A.dlogits ? launch_mode<E, kStep>(A, T, stream) : launch_mode<E, kLoss>(A, T, stream);
}

}  // namespace

size_t distill_bytes(const lordba_distill &d, int64_t T)
{
    return T <= kDistillAlone ? 0 : ((size_t)T * ((size_t)d.top * sizeof(Entry) + sizeof(uint2)) + 255) / 256 * 256;
}

int launch_distill(const lordba_distill &d, int64_t T, int dtype, bool backward, void *workspace, cudaStream_t stream)
{
    DistillArgs A;
    std::memset(&A, 0, sizeof(A));
    A.logits = d.logits; A.ids = d.ids; A.teacher = d.teacher; A.weight = d.weight;
    A.loss = d.loss; A.lse = d.lse; A.dlogits = d.dlogits;
    A.ld_logits = d.ld_logits; A.ld_ids = d.ld_ids; A.ld_teacher = d.ld_teacher; A.ld_dlogits = d.ld_dlogits;
    A.vocab = d.vocab;
    A.top = (int)d.top;
    A.ids64 = d.flags & LORDBA_DISTILL_IDS_64;
    A.teacher_dtype = d.teacher_dtype;
    A.entries = static_cast<uint4 *>(workspace);
    A.heads = reinterpret_cast<uint2 *>(A.entries + T * d.top);
    A.table = 32;
    while (A.table < 2 * A.top) A.table *= 2;
    A.temperature = d.temperature;
    A.inverse = 1.0f / d.temperature;
    A.scale = (float)(1.4426950408889634 / (double)d.temperature);
    switch (dtype) {
        case LORDBA_BF16: return launch_typed<__nv_bfloat16>(A, T, backward, stream);
        case LORDBA_F16: return launch_typed<__half>(A, T, backward, stream);
        default: return launch_typed<float>(A, T, backward, stream);
    }
}

}  // namespace lordba
