// Distillation from a teacher's top logits: the loss of a row, its log-sum, and the gradient to the student's logits.
//
// Bound: HBM.  A row's logits are read once, and for the gradient written once, because the row stays in registers in
// between: 64 KB of it in a CTA of 512 threads, and a row that is longer, or one of few, is shared by a cluster of up to eight
// CTAs, which exchange their maxima and sums through distributed shared memory.  All of a thread's loads are on the way
// before it looks at the first.  (What a row has beyond eight CTAs' registers is read again, from L2.)
//
// The exponentials are powers of two of  z log2(e)/temperature - m : one multiply-add and one instruction each.
#include <cstring>

#include "block_checks.h"
#include "block_common.cuh"
#include "sm100.cuh"

namespace lordba {
namespace {

constexpr int kMaxThreads = 512;
constexpr int kMaxSplit = 8;
constexpr int kMaxTop = LORDBA_DISTILL_MAX_TOP, kPerLane = kMaxTop / 32;
constexpr float kLn2 = 0.6931471805599453f;

struct DistillArgs {
    const void *logits, *ids, *teacher;
    const float *weight;
    float *loss, *lse;
    void *dlogits;
    int64_t ld_logits, ld_ids, ld_teacher, ld_dlogits, vocab;
    int top, ids64, teacher_dtype, split;
    float temperature, inverse, scale;        // scale: log2(e) / temperature
    int vec_in, vec_out;
};

__device__ __forceinline__ float exp2_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// sum of 2^(scale (z - max)) and the max it is relative to
struct Stat {
    float max, sum;
};
__device__ __forceinline__ Stat join(Stat a, Stat b, float scale)
{
    // of an empty side (-inf, 0), or one of minus infinities only, nothing is taken; a NaN sum stays one
    const float m = fmaxf(a.max, b.max), at = m == -INFINITY ? 0.0f : m;
    return Stat{m, a.sum * exp2_of((a.max - at) * scale) + b.sum * exp2_of((b.max - at) * scale)};
}

template <typename E> constexpr int kHeld = sizeof(E) == 4 ? 4 : 8;        // groups of eight a thread keeps

// STAT: max and sum are looked for (and loss and lse written); else lse is given.  GRAD: dlogits is written.
template <typename E, bool STAT, bool GRAD>
__global__ void __launch_bounds__(kMaxThreads, 2)
distill_kernel(const __grid_constant__ DistillArgs A)
{
    __shared__ float top_p[kMaxTop], top_log[kMaxTop], top_z[kMaxTop];      // p, log p, the student's logit
    __shared__ int top_id[kMaxTop];
    __shared__ Stat part[kMaxThreads / 32], peers[kMaxSplit];
    __shared__ float teacher_live;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
    const int64_t t = blockIdx.x / A.split;
    const int rank = blockIdx.x - (int)t * A.split;
    const int groups = (int)((A.vocab + 7) / 8);
    const int first = (int)((int64_t)groups * rank / A.split), last = (int)((int64_t)groups * (rank + 1) / A.split);
    const int V = (int)A.vocab;
    const E *z = static_cast<const E *>(A.logits) + t * A.ld_logits;
    grid_wait();
    grid_release();
    if (STAT && A.split > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");    // the peers run
    const float weight = A.weight ? A.weight[t] : 1.0f;
    constexpr int H = kHeld<E>;
    Group8<E> held[H];
    const bool wanted = STAT || weight != 0.0f;
    if (wanted) {
#pragma unroll
        for (int i = 0; i < H; ++i) {
            const int g = first + threadIdx.x + i * blockDim.x;
            if (g < last) held[i] = load8(z, g, V, A.vec_in);
        }
    }
    // the teacher: warp 0, entry lane + 32 i
    if (warp == 0) {
        float v[kPerLane], zt[kPerLane];
        int id[kPerLane];
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) {
            const int j = lane + 32 * i;
            v[i] = -INFINITY; id[i] = -1; zt[i] = 0.0f;
            if (j < A.top) {
                const int64_t k = A.ids64 ? static_cast<const int64_t *>(A.ids)[t * A.ld_ids + j]
                                          : (int64_t)static_cast<const int32_t *>(A.ids)[t * A.ld_ids + j];
                if (k >= 0 && k < A.vocab) {
                    id[i] = (int)k;
                    const int64_t at = t * A.ld_teacher + j;
                    v[i] = A.teacher_dtype == LORDBA_F32    ? static_cast<const float *>(A.teacher)[at]
                           : A.teacher_dtype == LORDBA_BF16 ? to_float(static_cast<const __nv_bfloat16 *>(A.teacher)[at])
                                                            : to_float(static_cast<const __half *>(A.teacher)[at]);
                    // dlogits may be the logits: CTAs that share a row without a barrier read here only what they write themselves
                    const bool own = k >= 8 * (int64_t)first && k < 8 * (int64_t)last;
                    if (STAT || own) zt[i] = to_float(z[k]);
                }
            }
            most = fmaxf(most, v[i]);
        }
        for (int o = 16; o; o /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        float total = 0.0f;                // 0 where no entry has a chance; a NaN comes through here
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) {
            if (v[i] != -INFINITY) v[i] = __fdiv_rn(v[i] - most, A.temperature);
            total += expf(v[i]);
        }
        for (int o = 16; o; o /= 2) total += __shfl_xor_sync(0xffffffffu, total, o);
        const float log_total = logf(total), inverse = 1.0f / total;
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) {
            const int j = lane + 32 * i;
            if (j < A.top) {
                top_p[j] = v[i] == -INFINITY ? 0.0f : expf(v[i]) * inverse;
                top_log[j] = v[i] - log_total;
                top_z[j] = zt[i];
                top_id[j] = id[i];
            }
        }
        if (lane == 0) teacher_live = total;
    }
    Stat all = {0.0f, 1.0f};
    if (STAT) {
        Stat s = {-INFINITY, 0.0f};
        auto top_of = [&](const Group8<E> &h, int g) {
            float v[8];
            unpack_group<E>(h, v);
            const int left = V - 8 * g;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < left) s.max = fmaxf(s.max, v[j]);
        };
        auto add = [&](const Group8<E> &h, int g, float minus) {
            float v[8];
            unpack_group<E>(h, v);
            const int left = V - 8 * g;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < left) s.sum += exp2_of(fmaf(v[j], A.scale, minus));
        };
#pragma unroll
        for (int i = 0; i < H; ++i) {
            const int g = first + threadIdx.x + i * blockDim.x;
            if (g < last) top_of(held[i], g);
        }
        for (int g = first + threadIdx.x + H * blockDim.x; g < last; g += blockDim.x) top_of(load8(z, g, V, A.vec_in), g);
        const float minus = s.max == -INFINITY ? 0.0f : -s.max * A.scale;
#pragma unroll
        for (int i = 0; i < H; ++i) {
            const int g = first + threadIdx.x + i * blockDim.x;
            if (g < last) add(held[i], g, minus);
        }
        for (int g = first + threadIdx.x + H * blockDim.x; g < last; g += blockDim.x) add(load8(z, g, V, A.vec_in), g, minus);
        for (int o = 16; o; o /= 2)
            s = join(s, Stat{__shfl_xor_sync(0xffffffffu, s.max, o), __shfl_xor_sync(0xffffffffu, s.sum, o)}, A.scale);
        if (lane == 0) part[warp] = s;
        __syncthreads();
        if (A.split > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (warp == 0) {
            s = lane < warps ? part[lane] : Stat{-INFINITY, 0.0f};
            for (int o = 16; o; o /= 2)
                s = join(s, Stat{__shfl_xor_sync(0xffffffffu, s.max, o), __shfl_xor_sync(0xffffffffu, s.sum, o)}, A.scale);
            if (A.split == 1) {
                if (lane == 0) peers[0] = s;
            } else if (lane < A.split) {
                const uint32_t to = sm100::peer_addr(sm100::smem_addr(&peers[rank]), lane);
                sm100::store_peer(to, __float_as_uint(s.max));
                sm100::store_peer(to + 4, __float_as_uint(s.sum));
            }
            __syncwarp();
        }
        if (A.split > 1) sm100::cluster_sync();
        else __syncthreads();
        all = peers[0];
        for (int r = 1; r < A.split; ++r) all = join(all, peers[r], A.scale);
    } else {
        __syncthreads();
    }
    const bool live = weight != 0.0f && teacher_live != 0.0f;
    // logits less `shift` powers are the student's probabilities
    const float shift = STAT ? all.max * A.scale + log2f(all.sum) : A.lse[t] * (1.0f / kLn2);
    if (STAT && rank == 0 && warp == 0) {
        // log p - log q from what is left of both maxima: neither lse nor a logit of its size enters
        const float log_sum = logf(all.sum);
        float loss = 0.0f;
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) {
            const int j = lane + 32 * i;
            if (j < A.top && top_p[j] != 0.0f) loss += top_p[j] * (top_log[j] - ((top_z[j] - all.max) * A.inverse - log_sum));
        }
        for (int o = 16; o; o /= 2) loss += __shfl_xor_sync(0xffffffffu, loss, o);
        if (lane == 0) {
            A.lse[t] = all.max * A.inverse + log_sum;
            A.loss[t] = live ? weight * A.temperature * A.temperature * loss : 0.0f;
        }
    }
    if (!GRAD) return;
    E *dz = static_cast<E *>(A.dlogits) + t * A.ld_dlogits;
    const float factor = weight * A.temperature;
    auto put = [&](const Group8<E> &h, int g) {
        float v[8];
        unpack_group<E>(h, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = live ? factor * exp2_of(fmaf(v[j], A.scale, -shift)) : 0.0f;
        store8(dz, g, V, A.vec_out, v);
    };
#pragma unroll
    for (int i = 0; i < H; ++i) {
        const int g = first + threadIdx.x + i * blockDim.x;
        if (g < last) put(held[i], g);
    }
    for (int g = first + threadIdx.x + H * blockDim.x; g < last; g += blockDim.x) put(wanted ? load8(z, g, V, A.vec_in) : held[0], g);
    if (!live) return;
    __syncthreads();                       // the top entries' gradients are written over what was put there
    for (int j = threadIdx.x; j < A.top; j += blockDim.x) {
        const int id = top_id[j];
        if (id < 8 * first || id >= 8 * last) continue;
        float p = 0.0f;                    // an index that stands there twice: both write the same value
        for (int k = 0; k < A.top; ++k) p += top_id[k] == id ? top_p[k] : 0.0f;
        dz[id] = from_float<E>(factor * (exp2_of(fmaf(top_z[j], A.scale, -shift)) - p));
    }
}

template <typename E, bool STAT, bool GRAD>
int launch_distill_typed(DistillArgs A, int64_t T, cudaStream_t stream)
{
    const int64_t groups = (A.vocab + 7) / 8;
    constexpr int H = kHeld<E>;
    // As many CTAs a row as hold it, more while there are SMs without one and a CTA keeps a kilobyte or so.
    int split = 1;
    while (split < kMaxSplit && (groups > (int64_t)split * kMaxThreads * H || (T * split < 148 && groups >= 256 * split))) split *= 2;
    const int64_t mine = (groups + split - 1) / split;
    int threads = 128;
    while (threads < kMaxThreads && mine > (int64_t)threads * (H / 2)) threads *= 2;
    A.split = split;
    if (T * split > 0x7fffffff) return LORDBA_EUNSUPPORTED;
    LaunchRec rec;
    std::memset(&rec, 0, sizeof(rec));
    rec.func = reinterpret_cast<const void *>(&distill_kernel<E, STAT, GRAD>);
    rec.grid[0] = (unsigned)(T * split);
    rec.grid[1] = rec.grid[2] = 1;
    rec.block = (uint32_t)threads;
    rec.cluster = STAT ? (uint32_t)split : 1;
    rec.pdl = 1;
    rec.n_args = 1;
    rec.arg_bytes[0] = sizeof(DistillArgs);
    return launch_record(rec, &A, nullptr, stream);
}

template <typename E>
int launch_distill_mode(const DistillArgs &A, int64_t T, bool stat, cudaStream_t stream)
{
    if (!stat) return launch_distill_typed<E, false, true>(A, T, stream);
    return A.dlogits ? launch_distill_typed<E, true, true>(A, T, stream) : launch_distill_typed<E, true, false>(A, T, stream);
}

}  // namespace

int launch_distill(const lordba_distill &d, int64_t T, int dtype, bool backward, cudaStream_t stream)
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
    A.temperature = d.temperature;
    A.inverse = 1.0f / d.temperature;
    A.scale = (float)(1.4426950408889634 / (double)d.temperature);
    const size_t e = elt(dtype);
    A.vec_in = aligned(d.logits, 16) && (d.ld_logits * e) % 16 == 0;
    A.vec_out = aligned(d.dlogits, 16) && (d.ld_dlogits * e) % 16 == 0;
    switch (dtype) {
        case LORDBA_BF16: return launch_distill_mode<__nv_bfloat16>(A, T, !backward, stream);
        case LORDBA_F16: return launch_distill_mode<__half>(A, T, !backward, stream);
        default: return launch_distill_mode<float>(A, T, !backward, stream);
    }
}

}  // namespace lordba
