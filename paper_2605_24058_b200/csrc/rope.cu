// Norms of queries and keys for each head, the rotation by position, and the gradients of both: one launch for queries
// and keys (the gradients of the norms' weights add the join of their partial sums).
//
// Bound: HBM, each head vector is read once and written once.  A head vector of d entries lies in ceil(d / 16) lanes of a
// warp, in registers from its load to its store; a lane holds eight of the pairs that are rotated together, so norm and
// rotation need nothing of another lane but the sum of squares.  A warp takes 32 / width heads of a token at a time and
// walks over the token's heads: the token's angles are worked out once for all of them.
//
// Angles.  f = position * inv_freq / (2 pi), in turns, less its whole turns.  A product in 32 bits would be off by 8e-3 already at position
// 131072, one in 64 bits by 2^-17 of a turn at 2^40: frequencies are taken as turns in two doubles, products with what their rounding left,
// and positions in halves of 32 bits, so that what is left of a turn is good to 2^-40 for any position and frequencies up to 16.
//
// Measured in bf16, 32 + 8 heads of 128: 8192 tokens 37 us (168 MB, 4.6 TB/s), gradients of 4096 tokens 32 us (126 MB, 3.9 TB/s), one
// token 2.6 us.  No unit is full: issue slots 55 and 49 %, the integer pipe 40 and 38 %; the warps that registers leave room for (24 and 16 an SM)
// wait for their loads first.
#include <cstring>

#include "block_checks.h"
#include "product_internal.cuh"

namespace lordba {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kMaxPairs = LORDBA_ROPE_MAX_D / 2;

// Queries, or keys.  Distances in entries.
struct Side {
    const void *x, *g;             // the vectors; backward: the gradients of the results
    void *out;
    int64_t x_token, x_head, g_token, g_head, out_token, out_head;
    const void *w;
    float *part;                   // backward: a row of d partial sums for each block, or null
    int heads;
    int steps, per_unit;           // steps of a token (a warp's heads each), and of a unit
    int chunks;                    // units of a token
    int blocks;
};

struct RopeArgs {
    Side side[2];
    const int64_t *positions;
    const float *inv_freq;
    int64_t T;
    int d, half, width, w_dtype, norm;      // half: pairs that are rotated; width: lanes of a head vector
    float eps, inv_d;
};

// A lane's eight pairs: pair p is entries (p, p + half) where pairs are halves and rotated, else (2 p, 2 p + 1).  VEC: the
// lane holds pairs 8 l ... 8 l + 7, so that its entries are two runs of eight (16 bytes each of a 16-bit type); of halves that
// are not rotated any eight pairs do, and it takes entries 16 l ... 16 l + 15 as two runs.  Otherwise neighbouring lanes hold
// neighbouring pairs.
template <bool INTERLEAVED, bool VEC>
struct Place {
    int l, width, half, d;
    bool turned;                   // VEC: whether the lane's pairs are rotated halves

    __device__ __forceinline__ Place(int lane, const RopeArgs &A) : l(lane % A.width), width(A.width), half(A.half), d(A.d)
    {
        turned = !INTERLEAVED && 8 * l < half;
    }
    __device__ __forceinline__ int pair(int j) const { return VEC ? 8 * l + j : l + width * j; }
    __device__ __forceinline__ bool has(int j) const { return VEC ? 16 * l < d : first(j) < d; }
    __device__ __forceinline__ int run(int r) const { return turned ? 8 * l + r * half : 16 * l + 8 * r; }
    __device__ __forceinline__ int first(int j) const
    {
        if (VEC) return INTERLEAVED ? 16 * l + 2 * j : run(0) + j;
        const int p = pair(j);
        return !INTERLEAVED && p < half ? p : 2 * p;
    }
    __device__ __forceinline__ int second(int j) const
    {
        if (VEC) return INTERLEAVED ? 16 * l + 2 * j + 1 : run(1) + j;
        const int p = pair(j);
        return !INTERLEAVED && p < half ? p + half : 2 * p + 1;
    }
};

// Eight entries side by side.  Input that lies off the 16-byte boundaries is fetched as the aligned pieces that hold it, and shifted when it is used: the
// pieces of the next heads are on their way meanwhile like any other (4096 tokens 22 us, gradients 40 us, half of a head rotated 35 and
// 78 us; entry by entry 62 and 125 us).
template <typename E, bool ALIGNED> struct Run;
template <typename E> struct Run<E, true> {
    Group8<E> g;
    __device__ __forceinline__ void load(const E *p) { g = load_group(p); }
    __device__ __forceinline__ Group8<E> get() const { return g; }
};
template <typename E> struct Run<E, false> {
    static constexpr int kWhole = sizeof(Group8<E>) / 16;
    uint4 piece[kWhole + 1];
    uint32_t by;
    __device__ __forceinline__ void load(const E *p)
    {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        const uint4 *q = reinterpret_cast<const uint4 *>(at & ~(uintptr_t)15);
        by = (uint32_t)at & 15u;
#pragma unroll
        for (int i = 0; i < kWhole; ++i) piece[i] = q[i];
        piece[kWhole] = q[by ? kWhole : 0];         // all of them hold bytes of the run
    }
    __device__ __forceinline__ Group8<E> get() const
    {
        Group8<E> g;
        g.w = join_pieces(piece[0], piece[1], by);
        if constexpr (sizeof(E) == 4) g.w2 = join_pieces(piece[1], piece[2], by);
        return g;
    }
};
// What a lane holds of a head vector, as it lies in memory.
template <typename E, bool VEC, bool ALIGNED> struct Raw;
template <typename E, bool ALIGNED> struct Raw<E, true, ALIGNED> { Run<E, ALIGNED> r[2]; };
template <typename E, bool ALIGNED> struct Raw<E, false, ALIGNED> { E a[8], b[8]; };

template <typename E, bool ALIGNED, bool INTERLEAVED, bool VEC>
__device__ __forceinline__ Raw<E, VEC, ALIGNED> load_heads(const E *p, const Place<INTERLEAVED, VEC> &at, bool in)
{
    Raw<E, VEC, ALIGNED> v;
    std::memset(&v, 0, sizeof(v));
    if (!in) return v;
    if constexpr (VEC) {
#pragma unroll
        for (int r = 0; r < 2; ++r)
            if (at.run(r) < at.d) v.r[r].load(p + at.run(r));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (at.first(j) < at.d) v.a[j] = p[at.first(j)];
            if (at.second(j) < at.d) v.b[j] = p[at.second(j)];
        }
    }
    return v;
}

template <typename E, bool INTERLEAVED, bool VEC, bool ALIGNED>
__device__ __forceinline__ void unpack(const Raw<E, VEC, ALIGNED> &v, float a[8], float b[8])
{
    if constexpr (VEC) {
        float x[16];
        unpack_group<E>(v.r[0].get(), x);
        unpack_group<E>(v.r[1].get(), x + 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            a[j] = x[INTERLEAVED ? 2 * j : j];
            b[j] = x[INTERLEAVED ? 2 * j + 1 : 8 + j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) { a[j] = to_float(v.a[j]); b[j] = to_float(v.b[j]); }
    }
}

template <typename E, bool INTERLEAVED, bool VEC>
__device__ __forceinline__ void store_heads(E *p, const Place<INTERLEAVED, VEC> &at, const float a[8], const float b[8])
{
    if constexpr (VEC) {
        float x[16];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[INTERLEAVED ? 2 * j : j] = a[j];
            x[INTERLEAVED ? 2 * j + 1 : 8 + j] = b[j];
        }
#pragma unroll
        for (int r = 0; r < 2; ++r)
            if (at.run(r) < at.d) store_group<E>(p + at.run(r), x + 8 * r);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (at.first(j) < at.d) p[at.first(j)] = from_float<E>(a[j]);
            if (at.second(j) < at.d) p[at.second(j)] = from_float<E>(b[j]);
        }
    }
}

// Cosine and sine of an angle in half turns: of its nearest float32, and what that leaves off as a first-order term.
__device__ __forceinline__ float2 cosine_sine(double half_turns)
{
    const float near = (float)half_turns, rest = (float)(half_turns - (double)near) * 3.14159265f;
    float sine, cosine;
    sincospif(near, &sine, &cosine);
    return make_float2(fmaf(-rest, sine, cosine), fmaf(rest, cosine, sine));
}

// A position in two parts, 2^32 apart, each a double exactly.
struct Position {
    double high, low;
    __device__ __forceinline__ explicit Position(int64_t p) : high(4294967296.0 * (double)(int32_t)(p >> 32)), low((double)(uint32_t)p) {}
};
// Cosine and sine of position * freq.  p c, where it is large, is whole turns and what its rounding left of them.
__device__ __forceinline__ float2 turn_at(const Position &p, float freq)
{
    constexpr double kTurn = 0.15915494309189535, kTurnRest = -9.839338337591243e-18;        // 1 / (2 pi)
    const double f = freq, c = f * kTurn, c_rest = fma(f, kTurnRest, fma(f, kTurn, -c));
    auto part = [&](double x) {
        const double t = x * c;
        return (t - rint(t)) + fma(x, c_rest, fma(x, c, -t));
    };
    double turns = part(p.low);
    if (p.high != 0.0) turns += part(p.high);                // negative, or from 2^32 on
    turns -= rint(turns);
    return cosine_sine(2.0 * turns);
}

__device__ __forceinline__ float weight_at(const void *w, int dtype, int i)
{
    if (dtype == LORDBA_F32) return static_cast<const float *>(w)[i];
    return dtype == LORDBA_BF16 ? to_float(static_cast<const __nv_bfloat16 *>(w)[i]) : to_float(static_cast<const __half *>(w)[i]);
}

// The sum over the lanes of a head vector.
__device__ __forceinline__ float over_head(float v, int width)
{
#pragma unroll
    for (int o = 16; o; o /= 2)
        if (o < width) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

template <typename E, bool BACK, bool INTERLEAVED, bool VEC, bool ALIGNED>
__global__ void __launch_bounds__(kThreads, BACK ? 2 : 3)
norm_rope_kernel(const __grid_constant__ RopeArgs A)
{
    __shared__ float2 table[kWarps][kMaxPairs];          // cosine and sine of the warp's token
    __shared__ float sums[BACK ? kWarps : 1][LORDBA_ROPE_MAX_D];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int which = (int)blockIdx.x >= A.side[0].blocks;
    const Side &S = A.side[which];
    const int block = blockIdx.x - (which ? A.side[0].blocks : 0);
    const Place<INTERLEAVED, VEC> at(lane, A);
    const int per = 32 / A.width, mine = lane / A.width;
    grid_wait();
    grid_release();

    float wa[8], wb[8], da[8], db[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        wa[j] = S.w && at.first(j) < A.d ? weight_at(S.w, A.w_dtype, at.first(j)) : 1.0f;
        wb[j] = S.w && at.second(j) < A.d ? weight_at(S.w, A.w_dtype, at.second(j)) : 1.0f;
        da[j] = db[j] = 0.0f;
    }
    const int64_t units = A.T * S.chunks;
    for (int64_t u = (int64_t)block * kWarps + warp; u < units; u += (int64_t)S.blocks * kWarps) {
        const int64_t t = S.chunks == 1 ? u : u / S.chunks;
        const int s0 = (int)(u - t * S.chunks) * S.per_unit, s1 = s0 + S.per_unit < S.steps ? s0 + S.per_unit : S.steps;
        const E *x = static_cast<const E *>(S.x) + t * S.x_token, *g = static_cast<const E *>(S.g) + (BACK ? t * S.g_token : 0);
        E *out = static_cast<E *>(S.out) + t * S.out_token;
        // the first heads are on their way while the angles are worked out
        int h = s0 * per + mine;
        bool in = h < S.heads && at.has(0);
        Raw<E, VEC, ALIGNED> rx = load_heads<E, ALIGNED>(x + h * S.x_head, at, in && (!BACK || A.norm)), rg;
        if (BACK) rg = load_heads<E, ALIGNED>(g + h * S.g_head, at, in);
        if (A.half) {
            const Position position(A.positions[t]);
            __syncwarp();                                   // the table's last readers
            for (int i = lane; i < A.half; i += 32) {
                const float2 p = turn_at(position, A.inv_freq[i]);
                table[warp][i] = make_float2(p.x, BACK ? -p.y : p.y);
            }
            __syncwarp();
        }
        float c[8], s[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool turned = at.pair(j) < A.half;
            const float2 v = turned ? table[warp][at.pair(j)] : make_float2(1.0f, 0.0f);
            c[j] = v.x; s[j] = v.y;
        }
        for (int step = s0; step < s1; ++step) {
            const int h_now = h;
            const bool in_now = in;
            float a[8], b[8], ga[8], gb[8];
            unpack<E, INTERLEAVED, VEC>(rx, a, b);
            if (BACK) unpack<E, INTERLEAVED, VEC>(rg, ga, gb);
            if (step + 1 < s1) {                            // the next heads' loads
                h += per;
                in = h < S.heads && at.has(0);
                rx = load_heads<E, ALIGNED>(x + h * S.x_head, at, in && (!BACK || A.norm));
                if (BACK) rg = load_heads<E, ALIGNED>(g + h * S.g_head, at, in);
            }
            float r = 1.0f;
            if (A.norm) {
                float q = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) q += a[j] * a[j] + b[j] * b[j];
                q = over_head(q, A.width) * A.inv_d + A.eps;
                r = !BACK || h_now < S.heads ? rsqrtf(q) : 0.0f;          // where no head is, zeros enter the sums of dw, without an epsilon too
            }
            if (!BACK) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float na = A.norm ? a[j] * r * wa[j] : a[j], nb = A.norm ? b[j] * r * wb[j] : b[j];
                    // an unrotated entry goes through as it is: 0 times an infinity would not
                    const bool turned = at.pair(j) < A.half;
                    a[j] = turned ? na * c[j] - nb * s[j] : na;
                    b[j] = turned ? nb * c[j] + na * s[j] : nb;
                }
            } else {
                float dot = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool turned = at.pair(j) < A.half;
                    const float ta = turned ? ga[j] * c[j] - gb[j] * s[j] : ga[j], tb = turned ? gb[j] * c[j] + ga[j] * s[j] : gb[j];
                    ga[j] = ta; gb[j] = tb;
                    if (A.norm) {
                        a[j] *= r; b[j] *= r;
                        da[j] += ta * a[j]; db[j] += tb * b[j];
                        ga[j] *= wa[j]; gb[j] *= wb[j];
                        dot += ga[j] * a[j] + gb[j] * b[j];
                    }
                }
                if (A.norm) {
                    dot = over_head(dot, A.width) * A.inv_d;
#pragma unroll
                    for (int j = 0; j < 8; ++j) { a[j] = r * (ga[j] - a[j] * dot); b[j] = r * (gb[j] - b[j] * dot); }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) { a[j] = ga[j]; b[j] = gb[j]; }
                }
            }
            if (in_now) store_heads<E>(out + h_now * S.out_head, at, a, b);
        }
    }
    if (BACK && S.part) {
        // lanes of one place, then warps, in a fixed order
#pragma unroll
        for (int j = 0; j < 8; ++j) {
#pragma unroll
            for (int o = 16; o; o /= 2)
                if (o >= A.width) {
                    da[j] += __shfl_xor_sync(0xffffffffu, da[j], o);
                    db[j] += __shfl_xor_sync(0xffffffffu, db[j], o);
                }
            if (mine == 0 && at.first(j) < A.d) sums[warp][at.first(j)] = da[j];
            if (mine == 0 && at.second(j) < A.d) sums[warp][at.second(j)] = db[j];
        }
        __syncthreads();
        for (int i = threadIdx.x; i < A.d; i += kThreads) {
            float v = 0.0f;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) v += sums[BACK ? k : 0][i];
            S.part[(int64_t)block * A.d + i] = v;
        }
    }
}

// ---- head vectors that are rotated whole and fill their lanes --------------------------------------------------------
// d = 16 WIDTH entries, all rotated, results on 16-byte boundaries: what models have.  Nothing is looked at per entry, and two entries
// are worked on by one instruction (4096 tokens 19.7 us, by the kernel for any heads 26 us).

template <typename E, bool INTERLEAVED, bool ALIGNED>
__device__ __forceinline__ void unpack_pairs(const Raw<E, true, ALIGNED> &raw, Two a[4], Two b[4])
{
    float v[16];
    unpack_group<E>(raw.r[0].get(), v);
    unpack_group<E>(raw.r[1].get(), v + 8);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        a[j] = INTERLEAVED ? two(v[4 * j], v[4 * j + 2]) : two(v[2 * j], v[2 * j + 1]);
        b[j] = INTERLEAVED ? two(v[4 * j + 1], v[4 * j + 3]) : two(v[8 + 2 * j], v[9 + 2 * j]);
    }
}
template <typename E, bool INTERLEAVED>
__device__ __forceinline__ void store_pairs(E *p, int l, int second, const Two a[4], const Two b[4])
{
    float v[16];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 x = halves(a[j]), y = halves(b[j]);
        v[INTERLEAVED ? 4 * j : 2 * j] = x.x; v[INTERLEAVED ? 4 * j + 2 : 2 * j + 1] = x.y;
        v[INTERLEAVED ? 4 * j + 1 : 8 + 2 * j] = y.x; v[INTERLEAVED ? 4 * j + 3 : 9 + 2 * j] = y.y;
    }
    store_group<E>(p, v);
    store_group<E>(p + second, v + 8);
}
template <int WIDTH>
__device__ __forceinline__ float over_lanes(Two t)
{
    const float2 h = halves(t);
    float v = h.x + h.y;
#pragma unroll
    for (int o = WIDTH / 2; o; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

template <typename E, bool BACK, bool INTERLEAVED, bool NORM, int WIDTH, bool ALIGNED>
__global__ void __launch_bounds__(kThreads, BACK ? 2 : 3)
norm_rope_full_kernel(const __grid_constant__ RopeArgs A)
{
    constexpr int D = 16 * WIDTH, PAIRS = D / 2, PER = 32 / WIDTH, SECOND = INTERLEAVED ? 8 : PAIRS;
    __shared__ float2 table[kWarps][PAIRS + 1];
    __shared__ float sums[BACK && NORM ? kWarps : 1][D];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, l = lane % WIDTH, mine = lane / WIDTH;
    const int at = INTERLEAVED ? 16 * l : 8 * l;             // the lane's first run of eight; the second is SECOND behind
    const int which = (int)blockIdx.x >= A.side[0].blocks;
    const Side &S = A.side[which];
    const int block = blockIdx.x - (which ? A.side[0].blocks : 0);
    grid_wait();
    grid_release();
    auto entry = [&](int j, int h, bool b) {                 // of pairs 2 j + h: the first or the second
        return INTERLEAVED ? at + 4 * j + 2 * h + b : at + 2 * j + h + (b ? SECOND : 0);
    };
    Two wa[4], wb[4], da[4], db[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        wa[j] = wb[j] = two(1.0f, 1.0f);
        if (NORM && S.w) {
            wa[j] = two(weight_at(S.w, A.w_dtype, entry(j, 0, false)), weight_at(S.w, A.w_dtype, entry(j, 1, false)));
            wb[j] = two(weight_at(S.w, A.w_dtype, entry(j, 0, true)), weight_at(S.w, A.w_dtype, entry(j, 1, true)));
        }
        da[j] = db[j] = two(0.0f, 0.0f);
    }
    auto load = [&](const E *p, bool in) {
        Raw<E, true, ALIGNED> v;
        std::memset(&v, 0, sizeof(v));
        if (in) {
            v.r[0].load(p);
            v.r[1].load(p + SECOND);
        }
        return v;
    };
    const int64_t units = A.T * S.chunks;
    const int64_t x_step = PER * S.x_head, g_step = PER * S.g_head, out_step = PER * S.out_head;
    for (int64_t u = (int64_t)block * kWarps + warp; u < units; u += (int64_t)S.blocks * kWarps) {
        const int64_t t = S.chunks == 1 ? u : u / S.chunks;
        const int s0 = (int)(u - t * S.chunks) * S.per_unit, s1 = s0 + S.per_unit < S.steps ? s0 + S.per_unit : S.steps;
        int h = s0 * PER + mine;
        const E *x = static_cast<const E *>(S.x) + t * S.x_token + h * S.x_head + at;
        const E *g = static_cast<const E *>(S.g) + (BACK ? t * S.g_token + h * S.g_head + at : 0);
        E *out = static_cast<E *>(S.out) + t * S.out_token + h * S.out_head + at;
        // the first heads are on their way while the angles are worked out
        Raw<E, true, ALIGNED> rx = load(x, h < S.heads && (!BACK || NORM)), rg;
        if (BACK) rg = load(g, h < S.heads);
        const Position position(A.positions[t]);
        __syncwarp();                                        // the table's last readers
#pragma unroll
        for (int i = 0; i < (PAIRS + 31) / 32; ++i) {
            const int p = lane + 32 * i;
            if (p < PAIRS) {
                const float2 v = turn_at(position, A.inv_freq[p]);
                table[warp][p] = make_float2(v.x, BACK ? -v.y : v.y);
            }
        }
        __syncwarp();
        Two c[4], s[4], minus[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 p = table[warp][8 * l + 2 * j], q = table[warp][8 * l + 2 * j + 1];
            c[j] = two(p.x, q.x); s[j] = two(p.y, q.y); minus[j] = two(-p.y, -q.y);
        }
#pragma unroll 1
        for (int step = s0; step < s1; ++step) {
            const bool in = h < S.heads;
            Two a[4], b[4], ga[4], gb[4];
            unpack_pairs<E, INTERLEAVED>(rx, a, b);
            if (BACK) unpack_pairs<E, INTERLEAVED>(rg, ga, gb);
            h += PER;
            x += x_step;
            if (BACK) g += g_step;
            const bool more = step + 1 < s1 && h < S.heads;   // the next heads' loads
            rx = load(x, more && (!BACK || NORM));
            if (BACK) rg = load(g, more);
            float r = 1.0f;
            if (NORM) {
                Two q = mul_two(a[0], a[0]), q2 = mul_two(b[0], b[0]);
#pragma unroll
                for (int j = 1; j < 4; ++j) { q = fma_two(a[j], a[j], q); q2 = fma_two(b[j], b[j], q2); }
                const float mean = over_lanes<WIDTH>(add_two(q, q2)) * A.inv_d + A.eps;
                r = !BACK || in ? rsqrtf(mean) : 0.0f;                    // where no head is, zeros enter the sums of dw, without an epsilon too
            }
            const Two rr = two(r, r);
            if (!BACK) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const Two na = NORM ? mul_two(a[j], mul_two(rr, wa[j])) : a[j], nb = NORM ? mul_two(b[j], mul_two(rr, wb[j])) : b[j];
                    a[j] = fma_two(na, c[j], mul_two(nb, minus[j]));
                    b[j] = fma_two(nb, c[j], mul_two(na, s[j]));
                }
            } else {
                Two dot = two(0.0f, 0.0f), dot2 = dot;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const Two ta = fma_two(ga[j], c[j], mul_two(gb[j], minus[j])), tb = fma_two(gb[j], c[j], mul_two(ga[j], s[j]));
                    ga[j] = ta; gb[j] = tb;
                    if (NORM) {
                        a[j] = mul_two(a[j], rr); b[j] = mul_two(b[j], rr);
                        da[j] = fma_two(ta, a[j], da[j]); db[j] = fma_two(tb, b[j], db[j]);
                        ga[j] = mul_two(ta, wa[j]); gb[j] = mul_two(tb, wb[j]);
                        dot = fma_two(ga[j], a[j], dot); dot2 = fma_two(gb[j], b[j], dot2);
                    }
                }
                if (NORM) {
                    const float d = -over_lanes<WIDTH>(add_two(dot, dot2)) * A.inv_d;
                    const Two dd = two(d, d);
#pragma unroll
                    for (int j = 0; j < 4; ++j) { ga[j] = mul_two(rr, fma_two(a[j], dd, ga[j])); gb[j] = mul_two(rr, fma_two(b[j], dd, gb[j])); }
                }
            }
            if (in) store_pairs<E, INTERLEAVED>(out, l, SECOND, BACK ? ga : a, BACK ? gb : b);
            out += out_step;
        }
    }
    if (BACK && NORM && S.part) {
        // lanes of one place, then warps, in a fixed order
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 x = halves(da[j]), y = halves(db[j]);
            float v[4] = {x.x, x.y, y.x, y.y};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
#pragma unroll
                for (int o = 16; o >= WIDTH; o /= 2) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
                if (mine == 0) sums[warp][entry(j, k % 2, k >= 2)] = v[k];
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < D; i += kThreads) {
            float v = 0.0f;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) v += sums[BACK && NORM ? k : 0][i];
            S.part[(int64_t)block * D + i] = v;
        }
    }
}

struct JoinArgs {
    const float *part[2];
    float *dw[2];
    int blocks[2], d;
};

// dw of one side: 32 columns a block, its eight warps take every eighth row of partial sums each.
__global__ void __launch_bounds__(kThreads)
norm_rope_join_kernel(const __grid_constant__ JoinArgs J)
{
    __shared__ float sums[kWarps][32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, i = blockIdx.x * 32 + lane, side = blockIdx.y;
    grid_wait();
    grid_release();
    if (!J.dw[side]) return;
    float v = 0.0f;
    if (i < J.d)
#pragma unroll 8
        for (int b = warp; b < J.blocks[side]; b += kWarps) v += J.part[side][(int64_t)b * J.d + i];
    sums[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && i < J.d) {
        v = 0.0f;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) v += sums[k][lane];
        J.dw[side][i] = v;
    }
}

// How a call's heads are dealt out: blocks of both sides, units.
void plan(RopeArgs &A, const lordba_norm_rope_args &f, int64_t T, bool back)
{
    A.T = T;
    A.d = f.d;
    A.half = f.rotary / 2;
    A.width = 1;
    while (A.width * 16 < f.d) A.width *= 2;
    const int per = 32 / A.width;
    int64_t all = 0;
    for (int i = 0; i < 2; ++i) {
        Side &S = A.side[i];
        S.heads = i ? f.heads_k : f.heads_q;
        S.steps = (S.heads + per - 1) / per;
        all += S.steps;
    }
    // a unit is a token's heads, or fewer of them while the GPU has idle warps (16 an SM are enough); backward two blocks an SM, what is
    // resident at once: each leaves a row of partial sums
    const int64_t warps = 16 * sm_count(), most_blocks = (back ? 2 : 16) * sm_count();
    for (int i = 0; i < 2; ++i) {
        Side &S = A.side[i];
        if (S.steps == 0) continue;
        const int64_t want = (T * all + warps - 1) / warps;
        S.per_unit = (int)(want < S.steps ? want : S.steps);
        S.chunks = (S.steps + S.per_unit - 1) / S.per_unit;
        const int64_t need = (T * S.chunks + kWarps - 1) / kWarps;
        int64_t share = most_blocks * S.steps / all;
        if (share < 1) share = 1;
        S.blocks = (int)(need < share ? need : share);
    }
}

bool vec_heads(const lordba_heads &h, size_t e) { return aligned(h.p, 16) && (h.token * e) % 16 == 0 && (h.head * e) % 16 == 0; }

void take(Side &S, const lordba_heads &x, const lordba_heads &g, const lordba_heads &out, const void *w)
{
    S.x = x.p; S.x_token = x.token; S.x_head = x.head;
    S.g = g.p; S.g_token = g.token; S.g_head = g.head;
    S.out = const_cast<void *>(out.p); S.out_token = out.token; S.out_head = out.head;
    S.w = w;
}

using RopeKernel = void (*)(const RopeArgs);

template <typename E, bool BACK, bool INTERLEAVED, bool NORM, bool ALIGNED>
RopeKernel full_kernel(int width)
{
    return width == 4   ? norm_rope_full_kernel<E, BACK, INTERLEAVED, NORM, 4, ALIGNED>
           : width == 8 ? norm_rope_full_kernel<E, BACK, INTERLEAVED, NORM, 8, ALIGNED>
                        : norm_rope_full_kernel<E, BACK, INTERLEAVED, NORM, 16, ALIGNED>;
}
template <typename E, bool BACK, bool ALIGNED>
RopeKernel full_kernel(const RopeArgs &A, bool interleaved)
{
    if (interleaved) return A.norm ? full_kernel<E, BACK, true, true, ALIGNED>(A.width) : full_kernel<E, BACK, true, false, ALIGNED>(A.width);
    return A.norm ? full_kernel<E, BACK, false, true, ALIGNED>(A.width) : full_kernel<E, BACK, false, false, ALIGNED>(A.width);
}

// vec_in, vec_out: rows of eight entries on 16-byte boundaries
template <typename E, bool BACK>
int launch_typed(const RopeArgs &A, bool interleaved, bool vec_shape, bool vec_in, bool vec_out, cudaStream_t stream)
{
    // heads of 64, 128 and 256 entries, rotated whole
    const bool full = vec_out && A.d == 16 * A.width && 2 * A.half == A.d && A.width >= 4 && A.width <= 16, vec = vec_shape && vec_out;
    RopeKernel kernel;
    if (full) kernel = vec_in ? full_kernel<E, BACK, true>(A, interleaved) : full_kernel<E, BACK, false>(A, interleaved);
    else if (vec && vec_in) kernel = interleaved ? norm_rope_kernel<E, BACK, true, true, true> : norm_rope_kernel<E, BACK, false, true, true>;
    else if (vec) kernel = interleaved ? norm_rope_kernel<E, BACK, true, true, false> : norm_rope_kernel<E, BACK, false, true, false>;
    else kernel = interleaved ? norm_rope_kernel<E, BACK, true, false, true> : norm_rope_kernel<E, BACK, false, false, true>;
    return launch_kernel(kernel, dim3((unsigned)(A.side[0].blocks + A.side[1].blocks), 1, 1), kThreads, 0, stream, A);
}

template <bool BACK>
int launch(const RopeArgs &A, int dtype, bool interleaved, bool vec_shape, bool vec_in, bool vec_out, cudaStream_t stream)
{
    switch (dtype) {
        case LORDBA_BF16: return launch_typed<__nv_bfloat16, BACK>(A, interleaved, vec_shape, vec_in, vec_out, stream);
        case LORDBA_F16: return launch_typed<__half, BACK>(A, interleaved, vec_shape, vec_in, vec_out, stream);
        default: return launch_typed<float, BACK>(A, interleaved, vec_shape, vec_in, vec_out, stream);
    }
}

void common(RopeArgs &A, const lordba_norm_rope_args &f)
{
    A.positions = f.positions;
    A.inv_freq = f.inv_freq;
    A.w_dtype = f.w_dtype;
    A.norm = !(f.flags & LORDBA_ROPE_NO_NORM);
    A.eps = f.eps;
    A.inv_d = 1.0f / (float)f.d;
}

// Whether a lane's pairs are two runs of eight entries on 16-byte boundaries.
bool vec_shape(const lordba_norm_rope_args &f) { return f.d % 8 == 0 && ((f.flags & LORDBA_ROPE_INTERLEAVED) || f.rotary % 16 == 0); }

}  // namespace

int launch_norm_rope(const lordba_norm_rope_args &f, int64_t T, int dtype, cudaStream_t stream)
{
    RopeArgs A;
    std::memset(&A, 0, sizeof(A));
    plan(A, f, T, false);
    common(A, f);
    const lordba_heads none{nullptr, 0, 0};
    take(A.side[0], f.q, none, f.q_out, f.w_q);
    take(A.side[1], f.k, none, f.k_out, f.w_k);
    const size_t e = elt(dtype);
    const bool in = vec_heads(f.q, e) && (!f.heads_k || vec_heads(f.k, e)), out = vec_heads(f.q_out, e) && (!f.heads_k || vec_heads(f.k_out, e));
    return launch<false>(A, dtype, f.flags & LORDBA_ROPE_INTERLEAVED, vec_shape(f), in, out, stream);
}

size_t norm_rope_backward_bytes(const lordba_norm_rope_grad_args &a, int64_t T)
{
    if (!a.dw_q && !a.dw_k) return 0;
    RopeArgs A;
    std::memset(&A, 0, sizeof(A));
    plan(A, a.f, T, true);
    return ((size_t)(A.side[0].blocks + A.side[1].blocks) * a.f.d * 4 + 255) / 256 * 256;
}

int launch_norm_rope_backward(const lordba_norm_rope_grad_args &a, int64_t T, int dtype, void *workspace, cudaStream_t stream)
{
    const lordba_norm_rope_args &f = a.f;
    RopeArgs A;
    std::memset(&A, 0, sizeof(A));
    plan(A, f, T, true);
    common(A, f);
    take(A.side[0], f.q, f.q_out, a.dq, f.w_q);
    take(A.side[1], f.k, f.k_out, a.dk, f.w_k);
    float *part = static_cast<float *>(workspace);
    if (a.dw_q) A.side[0].part = part;
    if (a.dw_k) A.side[1].part = part + (int64_t)A.side[0].blocks * f.d;
    const size_t e = elt(dtype);
    const bool in = vec_heads(f.q, e) && vec_heads(f.q_out, e) && (!f.heads_k || (vec_heads(f.k, e) && vec_heads(f.k_out, e)));
    const bool out = vec_heads(a.dq, e) && (!f.heads_k || vec_heads(a.dk, e));
    const int rc = launch<true>(A, dtype, f.flags & LORDBA_ROPE_INTERLEAVED, vec_shape(f), in, out, stream);
    if (rc != LORDBA_OK || (!a.dw_q && !a.dw_k)) return rc;
    JoinArgs J = {};
    J.d = f.d;
    for (int i = 0; i < 2; ++i) {
        J.part[i] = A.side[i].part;
        J.dw[i] = i ? a.dw_k : a.dw_q;
        J.blocks[i] = A.side[i].blocks;
    }
    return launch_kernel(norm_rope_join_kernel, dim3((unsigned)((f.d + 31) / 32), 2, 1), kThreads, 0, stream, J);
}

}  // namespace lordba
