// Products with an epilogue: the 8-bit base projection, the gated block and its gradients.
//
// One kernel for every form, type, size, pitch and alignment: 64 x 64 outputs a block, the operands
// staged in shared memory 16 contraction steps at a time as 32-bit values, sums in 32-bit integers (int8)
// or floats.
#include "block_common.cuh"

namespace lordba {
namespace {

constexpr int kTile = 64, kStep = 16;

struct Side {
    const void *p;
    int64_t ld;
    int mn_major;
};

struct SimpleArgs {
    Side a[2], b[2];
    int64_t M, N, K;
    int form, kind;
    void *out[2];
    int64_t ldo;
    int dtype;
    const float *s_row, *s_col[2];
    const void *add[2];
    void *pre[2];
    int64_t ld_add, ld_pre;
    int act;
};

__device__ __forceinline__ float load_any(const void *p, int64_t i, int dtype)
{
    if (dtype == LORDBA_F32) return static_cast<const float *>(p)[i];
    if (dtype == LORDBA_BF16) return to_float(static_cast<const __nv_bfloat16 *>(p)[i]);
    return to_float(static_cast<const __half *>(p)[i]);
}

__device__ __forceinline__ void store_any(void *p, int64_t i, int dtype, float v)
{
    if (dtype == LORDBA_F32) static_cast<float *>(p)[i] = v;
    else if (dtype == LORDBA_BF16) static_cast<__nv_bfloat16 *>(p)[i] = from_float<__nv_bfloat16>(v);
    else static_cast<__half *>(p)[i] = from_float<__half>(v);
}

template <typename Acc>
__device__ __forceinline__ Acc element(const Side &s, int kind, int64_t mn, int64_t k)
{
    const int64_t i = s.mn_major ? k * s.ld + mn : mn * s.ld + k;
    if (kind == kProductInt8) return (Acc) static_cast<const int8_t *>(s.p)[i];
    return (Acc)load_any(s.p, i, kind == kProductBf16 ? LORDBA_BF16 : LORDBA_F16);
}

template <typename Acc>
__global__ void __launch_bounds__(256)
product_kernel(const SimpleArgs P)
{
    __shared__ Acc As[kStep][kTile + 1], Bs[2][kStep][kTile + 1];
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int64_t n0 = (int64_t)blockIdx.x * kTile;
    const int problem = P.form == Product::kPair ? blockIdx.z : 0;
    const int parts = P.form == Product::kSum ? 2 : 1, cols = P.form == Product::kGated ? 2 : 1;
    grid_wait();
    grid_release();
    for (int64_t m0 = (int64_t)blockIdx.y * kTile; m0 < P.M; m0 += (int64_t)gridDim.y * kTile) {
        Acc acc[2][4][4] = {};
        for (int part = 0; part < parts; ++part) {
            const Side &a = P.a[P.form == Product::kPair ? problem : part];
            for (int64_t k0 = 0; k0 < P.K; k0 += kStep) {
                __syncthreads();
                for (int e = threadIdx.x; e < kTile * kStep; e += 256) {
                    const int am = a.mn_major ? e % kTile : e / kStep, ak = a.mn_major ? e / kTile : e % kStep;
                    As[ak][am] = m0 + am < P.M && k0 + ak < P.K ? element<Acc>(a, P.kind, m0 + am, k0 + ak) : (Acc)0;
                    for (int c = 0; c < cols; ++c) {
                        const Side &b = P.b[cols == 2 ? c : part];
                        const int bn = b.mn_major ? e % kTile : e / kStep, bk = b.mn_major ? e / kTile : e % kStep;
                        Bs[c][bk][bn] = n0 + bn < P.N && k0 + bk < P.K ? element<Acc>(b, P.kind, n0 + bn, k0 + bk) : (Acc)0;
                    }
                }
                __syncthreads();
#pragma unroll
                for (int k = 0; k < kStep; ++k)
                    for (int c = 0; c < cols; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int j = 0; j < 4; ++j) acc[c][i][j] += As[k][ty + 16 * i] * Bs[c][k][tx + 16 * j];
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
                if (m >= P.M || n >= P.N) continue;
                float v[2] = {(float)acc[0][i][j], (float)acc[1][i][j]};
                for (int c = 0; c < cols; ++c) {
                    if (P.kind == kProductInt8) v[c] = v[c] * P.s_row[m] * P.s_col[c][n];
                    if (P.add[c]) v[c] += load_any(P.add[c], m * P.ld_add + n, P.dtype);
                    if (P.pre[c]) store_any(P.pre[c], m * P.ld_pre + n, P.dtype, v[c]);
                }
                if (cols == 2)
                    v[0] = (P.act == LORDBA_ACT_SILU ? act_gate<LORDBA_ACT_SILU>(v[0]) : act_gate<LORDBA_ACT_GELU_TANH>(v[0])) * v[1];
                store_any(P.out[problem], m * P.ldo + n, P.dtype, v[0]);
            }
    }
}

}  // namespace

size_t product_workspace_bytes(const Product &p)
{
    (void)p;
    return 0;
}

int launch_product(const Product &p, void *workspace, cudaStream_t stream)
{
    (void)workspace;
    SimpleArgs a = {};
    for (int i = 0; i < 2; ++i) {
        a.a[i] = Side{p.a[i].p, p.a[i].ld, p.a[i].mn_major};
        a.b[i] = Side{p.b[i].p, p.b[i].ld, p.b[i].mn_major};
        a.out[i] = p.out[i];
        a.s_col[i] = p.s_col[i];
        a.add[i] = p.add[i];
        a.pre[i] = p.pre[i];
    }
    a.M = p.M; a.N = p.N; a.K = p.K;
    a.form = p.form; a.kind = p.kind;
    a.ldo = p.ldo; a.dtype = p.dtype; a.s_row = p.s_row;
    a.ld_add = p.ld_add; a.ld_pre = p.ld_pre; a.act = p.act;
    const int64_t gy = (p.M + kTile - 1) / kTile;
    const dim3 grid((unsigned)((p.N + kTile - 1) / kTile), (unsigned)(gy < 65535 ? gy : 65535), p.form == Product::kPair ? 2 : 1);
    return p.kind == kProductInt8 ? launch_kernel(product_kernel<int>, grid, 256, 0, stream, a)
                                  : launch_kernel(product_kernel<float>, grid, 256, 0, stream, a);
}

}  // namespace lordba
