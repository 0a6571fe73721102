// Products with an epilogue: the 8-bit base projection, the gated block and its gradients.  Operands that the
// copy engine cannot take are copied into the workspace first; the number of rows chooses the kernel.
#include <mutex>

#include "product_internal.cuh"

namespace lordba {

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiledFn encode_fn()
{
    static EncodeTiledFn fn = []() -> EncodeTiledFn {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            return nullptr;
        return reinterpret_cast<EncodeTiledFn>(p);
    }();
    return fn;
}

bool encode_map(CUtensorMap *map, const void *p, int64_t rows, int64_t cols, int64_t ld, int e, int box_rows)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld * e};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / e), (cuuint32_t)box_rows}, step[2] = {1, 1};
    // 16-bit elements keep their bits whatever they are called here
    return fn(map, e == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void *>(p), dims,
              strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool encode_store_map(CUtensorMap *map, void *p, int64_t rows, int64_t cols, int64_t ld, int e)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld * e};
    const cuuint32_t box[2] = {(cuuint32_t)(64 / e), 32}, step[2] = {1, 1};
    return fn(map, e == 2 ? CU_TENSOR_MAP_DATA_TYPE_UINT16 : CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, p, dims, strides, box, step,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int sm_count()
{
    static std::mutex mu;
    static int count[64] = {0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
    std::lock_guard<std::mutex> lock(mu);
    if (count[dev] == 0 && (cudaDeviceGetAttribute(&count[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || count[dev] < 1))
        count[dev] = 148;
    return count[dev];
}

namespace {

int elt_of(const Product &p) { return p.kind == kProductInt8 ? 1 : 2; }

// Rows and columns of an operand as it lies in memory.
int64_t rows_of(const Operand &o, int64_t mn, int64_t k) { return o.mn_major ? k : mn; }
int64_t cols_of(const Operand &o, int64_t mn, int64_t k) { return o.mn_major ? mn : k; }

size_t packed_pitch(const Operand &o, int64_t mn, int64_t k, int e) { return ((size_t)cols_of(o, mn, k) * e + 15) / 16 * 16; }

size_t packed_bytes(const Operand &o, int64_t mn, int64_t k, int e)
{
    return taken_as_is(o, e) ? 0 : (packed_pitch(o, mn, k, e) * (size_t)rows_of(o, mn, k) + 255) / 256 * 256;
}

// The product with its unaligned operands as copies would leave them (for planning: the addresses are not
// looked at).
Product copied_form(const Product &p)
{
    Product q = p;
    for (int i = 0; i < 2; ++i) {
        if (!taken_as_is(q.a[i], elt_of(p))) q.a[i] = Operand{reinterpret_cast<const void *>(uintptr_t(256)), (int64_t)packed_pitch(p.a[i], p.M, p.K, elt_of(p)) / elt_of(p), p.a[i].mn_major};
        if (!taken_as_is(q.b[i], elt_of(p))) q.b[i] = Operand{reinterpret_cast<const void *>(uintptr_t(256)), (int64_t)packed_pitch(p.b[i], p.N, p.K, elt_of(p)) / elt_of(p), p.b[i].mn_major};
    }
    return q;
}

// Few rows, or few results of long sums: the streaming kernel.  Else tiles.  Unaligned operands are copied for the
// tiles, and for the streaming kernel where that is quicker than its own shifting (many rows, which shift the
// weights once for each 128 of them); copies cost a launch and three passes over their bytes.
// Measured, 8-bit 4096 x 4096: 64 rows 9.0 us streaming, 15.5 us in tiles; 256 rows 13.8 and 15.8 us; 2048 rows 44 and
// 29 us.  Gated, 16-bit 4096 x 11008: 64 rows 36 and 54 us, 128 rows 45 and 54 us, 256 rows 95 and 54 us.
struct Way {
    bool stream, copy;
};

// Whether tiles would take the product without the rest of its entries' rounding.
bool drops_rest(const Product &p) { return p.lo[0].p && p.form == Product::kSum; }

Way way_of(const Product &p)
{
    double copied = 0;
    for (int i = 0; i < 2; ++i) copied += (double)packed_bytes(p.a[i], p.M, p.K, elt_of(p)) + (double)packed_bytes(p.b[i], p.N, p.K, elt_of(p));
    const double copies = copied > 0 ? 2.5 + copied * 3 / 6.0e6 : 0.0;
    // the second terms of a sum: streaming, and tiles, without them, only where that cannot be had
    Way best = {false, copied > 0};
    double us = drops_rest(p) ? 1e30 : tile_estimate(p) + copies;
    if (copied > 0) {
        const double t = stream_estimate(copied_form(p));
        if (t >= 0 && t + copies <= us) { best = Way{true, true}; us = t + copies; }
    }
    const double t = stream_estimate(p);
    if (t >= 0 && t <= us) best = Way{true, false};
    return best;
}

bool rows_vec(const void *p, int64_t ld, size_t e) { return aligned(p, 16) && ((size_t)ld * e) % 16 == 0; }

}  // namespace

size_t product_workspace_bytes(const Product &p)
{
    const Way way = way_of(p);
    size_t n = 0;
    for (int i = 0; way.copy && i < 2; ++i) n += packed_bytes(p.a[i], p.M, p.K, elt_of(p)) + packed_bytes(p.b[i], p.N, p.K, elt_of(p));
    return n + (way.stream ? stream_workspace_bytes(way.copy ? copied_form(p) : p) : 0);
}

int launch_product(const Product &given, void *workspace, cudaStream_t stream)
{
    Product p = given;
    const int e = elt_of(p);
    uint8_t *next = static_cast<uint8_t *>(workspace);
    RepackList list = {};
    const Way way = way_of(p);
    if (!way.stream && drops_rest(p)) p.lo[0] = p.lo[1] = Operand{};
    for (int i = 0; i < 4; ++i) {
        Operand &o = i < 2 ? p.a[i] : p.b[i - 2];
        const int64_t mn = i < 2 ? p.M : p.N;
        if (!way.copy || taken_as_is(o, e)) continue;
        const int64_t pitch = (int64_t)packed_pitch(o, mn, p.K, e);
        list.item[list.n++] = RepackList::Item{o.p, next, o.ld * e, pitch, rows_of(o, mn, p.K), cols_of(o, mn, p.K) * e};
        const size_t bytes = packed_bytes(o, mn, p.K, e);
        o.p = next;
        o.ld = pitch / e;
        next += bytes;
    }
    const int rc = launch_repack(list, stream);
    if (rc != LORDBA_OK) return rc;
    Finish f = {};
    for (int i = 0; i < 2; ++i) {
        f.out[i] = p.out[i]; f.s_col[i] = p.s_col[i]; f.add[i] = p.add[i]; f.pre[i] = p.pre[i];
    }
    f.ldo = p.ldo; f.s_row = p.s_row; f.ld_add = p.ld_add; f.ld_pre = p.ld_pre;
    f.M = p.M; f.N = p.N; f.dtype = p.dtype; f.act = p.act;
    const size_t eo = p.dtype == LORDBA_F32 ? 4 : 2;
    f.vec_out = rows_vec(p.out[0], p.ldo, eo) && aligned(p.out[1], 16);
    f.vec_add = rows_vec(p.add[0], p.ld_add, eo) && aligned(p.add[1], 16);
    f.vec_pre = rows_vec(p.pre[0], p.ld_pre, eo) && aligned(p.pre[1], 16);
    f.vec_scale = aligned(p.s_col[0], 16) && aligned(p.s_col[1], 16);
    if (way.stream) return launch_product_stream(p, f, next, stream);
    return launch_product_tile(p, f, stream);
}

}  // namespace lordba
