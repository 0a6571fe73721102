// Internal declarations shared by the translation units of liblordba.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "lordba.h"

namespace lordba {

constexpr int kMaxRank = 64;

// Device status codes written by bounded waits (0 = none).
enum DeviceCode : int {
    kDevOk = 0,
    kDevTmaWaitTimeout = 1,
    kDevMmaWaitTimeout = 2,
    kDevClusterWaitTimeout = 3,
    kDevEpilogueWaitTimeout = 4,
};

// Cycles after which a bounded device-side wait gives up (about a second).  The test-hooks build
// (-DLORDBA_TEST_HOOKS, never the product library) cuts it to about a millisecond so that a test
// can watch a wait run out.
#ifdef LORDBA_TEST_HOOKS
constexpr long long kWaitLimitCycles = 2000000LL;
#else
constexpr long long kWaitLimitCycles = 1500000000LL;
#endif

// Test-hooks build only: index of the one pipeline item whose copy request the producer of the
// tensor-core kernels leaves out (-1 = none), so that the consumers' wait for it runs out with
// nothing in flight.  Always -1 in the product library.
int test_skip_item();

// Test-hooks build only: whether the streaming product kernel's residency queries are to be taken as failed.  Always
// false in the product library.
bool test_fail_queries();

// Every kernel launch of the library goes through this counter.
void count_launch(int n = 1);

// Address of the device status word (resolved once per device).
int *device_status_word();

// ---- prepared launches ---------------------------------------------------------------------
// Every forward launcher describes its launches as records (kernel, grid, attributes, the
// kernel's argument blocks by value) and hands them to a sink.  The sink of a plain call
// launches each record at once; the sink of lordba_plan_init stores them in the caller's plan
// storage, and lordba_adapter_forward_planned replays them: the two paths launch the same
// kernels with the same arguments by construction.
struct LaunchRec {
    const void *func;
    uint32_t grid[3];
    uint32_t block;
    uint32_t smem;
    uint32_t cluster;      // CTAs per cluster (0 or 1: no cluster attribute)
    uint32_t pdl;          // 1: programmatic stream serialization allowed
    uint32_t n_args;       // 1 or 2 argument blocks
    uint32_t arg_bytes[2];
    uint32_t total_bytes;  // this record + its argument blocks in plan storage (multiple of 64)
    uint32_t cluster_z;    // 1: the cluster lies along grid z instead of grid x
};

struct LaunchSink {
    cudaStream_t stream = nullptr;
    bool immediate = true;   // launch now; otherwise append to buf (buf == nullptr: only count bytes)
    uint8_t *buf = nullptr;
    size_t cap = 0, used = 0;
    int count = 0;
    // arg1 may be null when rec.n_args == 1.  Returns a lordba_status.
    int emit(LaunchRec rec, const void *arg0, const void *arg1);
};

// Launch a stored record (args point into plan storage).
int launch_record(const LaunchRec &rec, const void *arg0, const void *arg1, cudaStream_t stream);

// A call holds at most this many projections (index arrays live on the stack).
constexpr int kMaxCallProjs = LORDBA_MAX_PROJS;

// Which projections of a call a launcher takes: those the selector maps to its own family.
struct FamilySelector {
    int dtype;
    int variant;       // the pinned family, or LORDBA_VARIANT_AUTO
    bool use_tc;       // AUTO decided for the tcgen05 kernel (or it is pinned)
    // LORDBA_VARIANT_FMA / _TC / _MMA for a projection with `rows` > 0 token rows; 0 for an empty one
    int family(const lordba_proj &p, int64_t rows) const;
};

// --- pack.cu ---------------------------------------------------------------
int launch_pack(const int8_t *signs, int64_t rows, int64_t cols, int role, uint32_t *packed,
                cudaStream_t stream);
int launch_widen_scales(const uint16_t *src, float *dst, int64_t n, cudaStream_t stream);
int launch_unpack(const uint32_t *packed, int64_t rows, int64_t cols, int role, int8_t *signs,
                  cudaStream_t stream);

// --- fit.cu ----------------------------------------------------------------
size_t fit_workspace_bytes(int64_t d_in, int64_t d_out, int r);
int launch_fit_scales(const float *target, int64_t ld, const uint32_t *pa, const uint32_t *pb, float *s_in, float *s_r,
                      float *s_out, int64_t d_in, int64_t d_out, int r, int sweeps, int axes, void *workspace,
                      cudaStream_t stream);

// --- forward_*.cu ------------------------------------------------------------
// Each launcher walks the n projections of a call (validated by the caller; tokens[i] = token
// rows of projection i, or T for all when tokens is null), takes those whose family is its own,
// and emits its launches into the sink.  *launches counts the launches of the call so far, over
// all families (the first launch of a call waits for the stream's previous kernel).
// batch_checked: the projections are known to be independent of one another, so the launches of
// this call may overlap each other; LORDBA_PROJ_OVERLAP on every projection lets the first
// launch overlap the previous call as well.
int launch_forward_fma(const lordba_proj *projs, const int64_t *tokens, int64_t T, int n, const FamilySelector &sel,
                       LaunchSink &sink);
bool tc_supported(const lordba_proj &p, int64_t T, int dtype);
int launch_forward_tc(const lordba_proj *projs, const int64_t *tokens, int64_t T, int n, const FamilySelector &sel,
                      LaunchSink &sink, bool batch_checked, int *launches);
bool mma_supported(const lordba_proj &p, int64_t T, int dtype);
int launch_forward_mma(const lordba_proj *projs, const int64_t *tokens, int64_t T, int n, const FamilySelector &sel,
                       LaunchSink &sink, bool batch_checked, int *launches);

// --- elementwise.cu ----------------------------------------------------------
int launch_quantize_rows(const void *x, int64_t ldx, int8_t *q, int64_t ldq, float *scale, int64_t T, int64_t d,
                         int dtype, cudaStream_t stream);
int launch_dropout(const void *x, int64_t ldx, const void *residual, int64_t ldr, void *out, int64_t ldo, int64_t T,
                   int64_t d, int cut, uint64_t seed, uint64_t offset, int dtype, cudaStream_t stream);
// lo_gate, lo_up (pitch ld_lo, 16-byte rows; null: not wanted): what rounding took from dgate and dup
int launch_gated_grad(const lordba_gated_grad &g, int64_t T, int dtype, void *lo_gate, void *lo_up, int64_t ld_lo,
                      cudaStream_t stream);
// Copies that give operands a pitch of 16-byte multiples: rows x cols bytes each, any alignment of src.
struct RepackList {
    struct Item {
        const void *src;
        void *dst;
        int64_t ld_src, ld_dst, rows, cols;      // bytes
    } item[4];
    int n;
};
int launch_repack(const RepackList &list, cudaStream_t stream);

// --- int4.cu -----------------------------------------------------------------
int launch_int4_pack(const uint8_t *values, int64_t ldv, uint8_t *q, int64_t ldq, int64_t d_out, int64_t d_in, cudaStream_t stream);
int launch_int4_quantize(const void *w, int64_t ldw, int wdtype, uint8_t *q, int64_t ldq, void *scale, int64_t ld_scale, uint8_t *zero,
                         int64_t ld_zero, int64_t d_out, int64_t d_in, int group, int dtype, cudaStream_t stream);
int launch_int4_dequantize(const lordba_int4_proj &p, int dtype, cudaStream_t stream);      // to p.out

// --- int4_few.cu -------------------------------------------------------------
constexpr int64_t kInt4Stream = 256;    // tokens up to which the weights are widened on their way
constexpr int64_t kInt4Few = 32;        // tokens it takes at most
int launch_int4_few(const lordba_int4_proj &p, int64_t T, int dtype, cudaStream_t stream);

// --- int4_stream.cu ----------------------------------------------------------
bool int4_stream_takes(const lordba_int4_proj &p, int64_t T, bool backward);         // whether its counters have room for the sizes
int launch_int4_stream(const lordba_int4_proj &p, int64_t T, int dtype, bool backward, cudaStream_t stream);      // p.in: as above

// --- rope.cu -----------------------------------------------------------------
int launch_norm_rope(const lordba_norm_rope_args &f, int64_t T, int dtype, cudaStream_t stream);
size_t norm_rope_backward_bytes(const lordba_norm_rope_grad_args &a, int64_t T);
int launch_norm_rope_backward(const lordba_norm_rope_grad_args &a, int64_t T, int dtype, void *workspace, cudaStream_t stream);

// --- distill.cu --------------------------------------------------------------
size_t distill_bytes(const lordba_distill &d, int64_t T);
int launch_distill(const lordba_distill &d, int64_t T, int dtype, bool backward, void *workspace, cudaStream_t stream);

// --- product.cu --------------------------------------------------------------
// D[m,n] = sum_k A[m,k] B[n,k], then an epilogue.  An operand is a row-major matrix; its rows run along m
// (n) with the contraction contiguous, or, mn_major, along the contraction with m (n) contiguous.
struct Operand {
    const void *p;
    int64_t ld;          // pitch in elements
    bool mn_major;
};

enum ProductKind { kProductBf16, kProductF16, kProductInt8 };

struct Product {
    ProductKind kind;
    int64_t M, N, K;
    Operand a[2], b[2];
    Operand lo[2];       // added to a[0], a[1] (kSum with at most kLoTokens rows, kPair), or null: A in twice the bits.
                         // A kSum of more columns than the streaming kernel can take goes without.
    // kSingle: D = A0 B0.  kSum: D = A0 B0 + A1 B1.  kGated: gate = A0 B0, up = A0 B1.
    // kPair: two products A0 B0 and A1 B0 with an output each.
    enum Form { kSingle, kSum, kGated, kPair } form;
    // epilogue
    void *out[2];                 // [1]: kPair only
    int64_t ldo;
    int dtype;                    // of out, add and pre
    const float *s_row, *s_col[2];    // int8 only: scales per row and per column (of gate and up)
    const void *add[2];           // kGated only: addends of gate and up, or null
    void *pre[2];                 // kGated only: where gate and up go, or null
    int64_t ld_add, ld_pre;
    int act;
};

// A product over a gradient's entries inherits their rounding.  Where it is bound by other bytes (the weights that
// stream past a few tokens, the gradients of the weights) the entries go in with their rounding's rest, which
// costs nothing; with more tokens they do not: the sums average over the errors (1.4 times that of rounding the
// result, 1e-3 of it in bfloat16), and the products would take twice as long.
constexpr int64_t kLoTokens = 64;

size_t product_workspace_bytes(const Product &p);
int launch_product(const Product &p, void *workspace, cudaStream_t stream);

// --- argument checks -----------------------------------------------------------
inline bool aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

inline bool overlaps(const void *a, size_t na, const void *b, size_t nb)
{
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return a0 < b0 + nb && b0 < a0 + na;
}

inline bool known_dtype(int dtype) { return dtype == LORDBA_F32 || dtype == LORDBA_BF16 || dtype == LORDBA_F16; }

inline int64_t rows_of(const int64_t *tokens, int64_t T, int i) { return tokens ? tokens[i] : T; }

}  // namespace lordba
