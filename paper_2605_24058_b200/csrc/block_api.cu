// C ABI of the operators next to the adapters: the 8-bit base projection, the gated feed-forward block and
// dropout.  Argument checks on the host, then launches; include/lordba.h states every contract.
#include <cmath>
#include <cstring>

#include "block_checks.h"

namespace lordba {
namespace {

Product int8_product(const lordba_int8_proj &p, int64_t T, int dtype)
{
    Product q = {};
    q.kind = kProductInt8;
    q.form = Product::kSingle;
    q.M = T; q.N = p.d_out; q.K = p.d_in;
    q.a[0] = Operand{p.x, p.ldx, false};
    q.b[0] = Operand{p.w, p.ldw, false};
    q.out[0] = p.y; q.ldo = p.ldy; q.dtype = dtype;
    q.s_row = p.s_x; q.s_col[0] = p.s_w;
    return q;
}

Product gated_product(const lordba_gated &g, int64_t T, int dtype)
{
    const bool int8 = (g.flags & LORDBA_GATED_INT8) != 0;
    Product q = {};
    q.kind = int8 ? kProductInt8 : dtype == LORDBA_BF16 ? kProductBf16 : kProductF16;
    q.form = Product::kGated;
    q.M = T; q.N = g.d_hidden; q.K = g.d_in;
    q.a[0] = Operand{g.x, g.ldx, false};
    q.b[0] = Operand{g.w_gate, g.ldw, false};
    q.b[1] = Operand{g.w_up, g.ldw, false};
    q.out[0] = g.h; q.ldo = g.ldh; q.dtype = dtype;
    q.s_row = g.s_x; q.s_col[0] = g.s_gate; q.s_col[1] = g.s_up;
    q.add[0] = g.gate_add; q.add[1] = g.up_add; q.ld_add = g.ld_add;
    q.pre[0] = g.gate; q.pre[1] = g.up; q.ld_pre = g.ld_pre;
    q.act = g.act;
    return q;
}

// dx = dgate w_gate + dup w_up: the contraction runs over d_hidden, along the weights' rows
Product dx_product(const lordba_gated_grad &g, int64_t T, int dtype)
{
    Product q = {};
    q.kind = dtype == LORDBA_BF16 ? kProductBf16 : kProductF16;
    q.form = Product::kSum;
    q.M = T; q.N = g.d_in; q.K = g.d_hidden;
    q.a[0] = Operand{g.dgate, g.ld_dpre, false};
    q.a[1] = Operand{g.dup, g.ld_dpre, false};
    q.b[0] = Operand{g.w_gate, g.ldw, true};
    q.b[1] = Operand{g.w_up, g.ldw, true};
    q.out[0] = g.dx; q.ldo = g.ld_dx; q.dtype = dtype;
    return q;
}

// dw_gate = dgate^T x, dw_up = dup^T x: the contraction runs over the tokens, along every operand's rows
Product dw_product(const lordba_gated_grad &g, int64_t T, int dtype)
{
    Product q = {};
    q.kind = dtype == LORDBA_BF16 ? kProductBf16 : kProductF16;
    q.form = Product::kPair;
    q.M = g.d_hidden; q.N = g.d_in; q.K = T;
    q.a[0] = Operand{g.dgate, g.ld_dpre, true};
    q.a[1] = Operand{g.dup, g.ld_dpre, true};
    q.b[0] = Operand{g.x, g.ldx, true};
    q.out[0] = g.dw_gate; q.out[1] = g.dw_up; q.ldo = g.ld_dw; q.dtype = dtype;
    return q;
}

int check_int8(const lordba_int8_proj &p, int64_t T, int dtype)
{
    if (!known_dtype(dtype)) return LORDBA_EUNSUPPORTED;
    if (bad_size(T, p.d_in) || bad_size(T, p.d_out) || p.ldx < p.d_in || p.ldw < p.d_in || p.ldy < p.d_out)
        return LORDBA_EINVAL;
    if (p.d_in > LORDBA_INT8_MAX_DIN) return LORDBA_EUNSUPPORTED;      // the 32-bit sum could wrap
    if (T == 0) return LORDBA_OK;
    const Matrix x{p.x, T, p.d_in, p.ldx, 1}, w{p.w, p.d_out, p.d_in, p.ldw, 1}, y{p.y, T, p.d_out, p.ldy, elt(dtype)};
    const Matrix sx{p.s_x, 1, T, T, 4}, sw{p.s_w, 1, p.d_out, p.d_out, 4};
    for (const Matrix *m : {&x, &w, &y, &sx, &sw}) {
        const int rc = check_matrix(*m);
        if (rc != LORDBA_OK) return rc;
    }
    return meet(y, x) || meet(y, w) || meet(y, sx) || meet(y, sw) ? LORDBA_EINVAL : LORDBA_OK;
}

int check_gated(const lordba_gated &g, int64_t T, int dtype)
{
    if (dtype != LORDBA_BF16 && dtype != LORDBA_F16) return LORDBA_EUNSUPPORTED;
    if (g.act != LORDBA_ACT_SILU && g.act != LORDBA_ACT_GELU_TANH) return LORDBA_EUNSUPPORTED;
    if (g.flags & ~LORDBA_GATED_INT8) return LORDBA_EINVAL;
    const bool int8 = (g.flags & LORDBA_GATED_INT8) != 0;
    if (bad_size(T, g.d_in) || bad_size(T, g.d_hidden) || g.ldx < g.d_in || g.ldw < g.d_in || g.ldh < g.d_hidden)
        return LORDBA_EINVAL;
    if (!g.gate_add != !g.up_add || !g.gate != !g.up) return LORDBA_EINVAL;
    if ((g.gate_add && g.ld_add < g.d_hidden) || (g.gate && g.ld_pre < g.d_hidden)) return LORDBA_EINVAL;
    if (int8 && g.d_in > LORDBA_INT8_MAX_DIN) return LORDBA_EUNSUPPORTED;
    if (T == 0) return LORDBA_OK;
    const size_t e = int8 ? 1 : 2;
    const Matrix none{};
    const Matrix x{g.x, T, g.d_in, g.ldx, e}, wg{g.w_gate, g.d_hidden, g.d_in, g.ldw, e}, wu{g.w_up, g.d_hidden, g.d_in, g.ldw, e};
    const Matrix ga{g.gate_add, T, g.d_hidden, g.ld_add, 2}, ua{g.up_add, T, g.d_hidden, g.ld_add, 2};
    const Matrix gp{g.gate, T, g.d_hidden, g.ld_pre, 2}, up{g.up, T, g.d_hidden, g.ld_pre, 2}, h{g.h, T, g.d_hidden, g.ldh, 2};
    const Matrix sx = int8 ? Matrix{g.s_x, 1, T, T, 4} : none, sg = int8 ? Matrix{g.s_gate, 1, g.d_hidden, g.d_hidden, 4} : none,
                 su = int8 ? Matrix{g.s_up, 1, g.d_hidden, g.d_hidden, 4} : none;
    if (!int8 && (g.s_x || g.s_gate || g.s_up)) return LORDBA_EINVAL;
    for (const Matrix *m : {&x, &wg, &wu, &h, &ga, &ua, &gp, &up, &sx, &sg, &su}) {
        const bool optional = m == &ga || m == &ua || m == &gp || m == &up || (!int8 && (m == &sx || m == &sg || m == &su));
        if (optional && !m->p) continue;
        const int rc = check_matrix(*m);
        if (rc != LORDBA_OK) return rc;
    }
    // the outputs meet neither one another nor an input, except that gate / up may be gate_add / up_add
    const Matrix *outs[3] = {&h, &gp, &up};
    for (int i = 0; i < 3; ++i) {
        for (int j = i + 1; j < 3; ++j)
            if (meet(*outs[i], *outs[j])) return LORDBA_EINVAL;
        for (const Matrix *m : {&x, &wg, &wu, &sx, &sg, &su})
            if (meet(*outs[i], *m)) return LORDBA_EINVAL;
        if (meet(*outs[i], ga) && !(i == 1 && same(gp, ga))) return LORDBA_EINVAL;
        if (meet(*outs[i], ua) && !(i == 2 && same(up, ua))) return LORDBA_EINVAL;
    }
    return LORDBA_OK;
}

int check_grad(const lordba_gated_grad &g, int64_t T, int dtype)
{
    if (dtype != LORDBA_BF16 && dtype != LORDBA_F16) return LORDBA_EUNSUPPORTED;
    if (g.act != LORDBA_ACT_SILU && g.act != LORDBA_ACT_GELU_TANH) return LORDBA_EUNSUPPORTED;
    if (g.flags) return LORDBA_EINVAL;
    if (bad_size(T, g.d_in) || bad_size(T, g.d_hidden)) return LORDBA_EINVAL;
    if (!g.dw_gate != !g.dw_up) return LORDBA_EINVAL;
    if (g.ld_dh < g.d_hidden || g.ld_pre < g.d_hidden || g.ld_dpre < g.d_hidden || (g.dx && (g.ldw < g.d_in || g.ld_dx < g.d_in)) ||
        (g.dw_gate && (g.ldx < g.d_in || g.ld_dw < g.d_in)))
        return LORDBA_EINVAL;
    const Matrix none{};
    const Matrix dwg = g.dw_gate ? Matrix{g.dw_gate, g.d_hidden, g.d_in, g.ld_dw, 2} : none;
    const Matrix dwu = g.dw_up ? Matrix{g.dw_up, g.d_hidden, g.d_in, g.ld_dw, 2} : none;
    if (T == 0) {
        if (dwg.p && (!aligned(dwg.p, 2) || !aligned(dwu.p, 2))) return LORDBA_EALIGN;
        return meet(dwg, dwu) ? LORDBA_EINVAL : LORDBA_OK;
    }
    const Matrix dh{g.dh, T, g.d_hidden, g.ld_dh, 2}, gp{g.gate, T, g.d_hidden, g.ld_pre, 2}, up{g.up, T, g.d_hidden, g.ld_pre, 2};
    const Matrix dg{g.dgate, T, g.d_hidden, g.ld_dpre, 2}, du{g.dup, T, g.d_hidden, g.ld_dpre, 2};
    const Matrix dx = g.dx ? Matrix{g.dx, T, g.d_in, g.ld_dx, 2} : none;
    const Matrix wg = g.dx ? Matrix{g.w_gate, g.d_hidden, g.d_in, g.ldw, 2} : none;
    const Matrix wu = g.dx ? Matrix{g.w_up, g.d_hidden, g.d_in, g.ldw, 2} : none;
    const Matrix x = g.dw_gate ? Matrix{g.x, T, g.d_in, g.ldx, 2} : none;
    for (const Matrix *m : {&dh, &gp, &up, &dg, &du, &dx, &wg, &wu, &x, &dwg, &dwu}) {
        const bool optional = (!g.dx && (m == &dx || m == &wg || m == &wu)) || (!g.dw_gate && (m == &x || m == &dwg || m == &dwu));
        if (optional) continue;
        const int rc = check_matrix(*m);
        if (rc != LORDBA_OK) return rc;
    }
    const Matrix *outs[5] = {&dg, &du, &dx, &dwg, &dwu};
    for (int i = 0; i < 5; ++i) {
        for (int j = i + 1; j < 5; ++j)
            if (meet(*outs[i], *outs[j])) return LORDBA_EINVAL;
        for (const Matrix *m : {&dh, &gp, &up, &wg, &wu, &x})
            if (meet(*outs[i], *m)) return LORDBA_EINVAL;
    }
    return LORDBA_OK;
}

// The workspace of a backward pass: what rounding took from dgate and dup, where that is kept (few tokens), then
// the operands that a product copies; the two products run one after the other and share that part.
struct GradWorkspace {
    size_t lo_bytes, bytes;      // of one of dgate and dup; in all
    int64_t ld_lo;
};

GradWorkspace grad_workspace(const lordba_gated_grad &g, int64_t T, int dtype)
{
    GradWorkspace w = {};
    if ((g.dx || g.dw_gate) && T <= kLoTokens) {
        w.ld_lo = (g.d_hidden + 7) / 8 * 8;
        w.lo_bytes = ((size_t)T * (size_t)w.ld_lo * 2 + 255) / 256 * 256;
    }
    Product dx = dx_product(g, T, dtype), dw = dw_product(g, T, dtype);
    // the rest lies aligned and is never copied: its place says only that it is there
    for (Product *q : {&dx, &dw})
        if (w.lo_bytes) q->lo[0] = q->lo[1] = Operand{reinterpret_cast<const void *>(uintptr_t(256)), w.ld_lo, false};
    const size_t a = g.dx ? product_workspace_bytes(dx) : 0, b = g.dw_gate ? product_workspace_bytes(dw) : 0;
    w.bytes = 2 * w.lo_bytes + (a > b ? a : b);
    return w;
}

}  // namespace
}  // namespace lordba

using namespace lordba;

extern "C" {

int lordba_int8_quantize_rows(const void *x, int64_t ldx, int8_t *q, int64_t ldq, float *scale, int64_t T, int64_t d,
                              int dtype, void *stream)
{
    if (!known_dtype(dtype)) return LORDBA_EUNSUPPORTED;
    if (bad_size(T, d) || ldx < d || ldq < d) return LORDBA_EINVAL;
    if (T == 0) return LORDBA_OK;
    const Matrix mx{x, T, d, ldx, elt(dtype)}, mq{q, T, d, ldq, 1}, ms{scale, 1, T, T, 4};
    for (const Matrix *m : {&mx, &mq, &ms}) {
        const int rc = check_matrix(*m);
        if (rc != LORDBA_OK) return rc;
    }
    if (meet(mq, mx) || meet(ms, mx) || meet(ms, mq)) return LORDBA_EINVAL;
    return launch_quantize_rows(x, ldx, q, ldq, scale, T, d, dtype, static_cast<cudaStream_t>(stream));
}

size_t lordba_int8_linear_workspace_bytes(const lordba_int8_proj *p, int64_t T)
{
    if (!p || bad_size(T, p->d_in) || bad_size(T, p->d_out) || T == 0) return 0;
    return product_workspace_bytes(int8_product(*p, T, LORDBA_F32));
}

int lordba_int8_linear(const lordba_int8_proj *p, int64_t T, int dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!p) return LORDBA_EINVAL;
    int rc = check_int8(*p, T, dtype);
    if (rc != LORDBA_OK || T == 0) return rc;
    const Product q = int8_product(*p, T, dtype);
    rc = check_workspace(product_workspace_bytes(q), workspace, workspace_bytes);
    return rc != LORDBA_OK ? rc : launch_product(q, workspace, static_cast<cudaStream_t>(stream));
}

size_t lordba_gated_workspace_bytes(const lordba_gated *g, int64_t T)
{
    if (!g || bad_size(T, g->d_in) || bad_size(T, g->d_hidden) || T == 0) return 0;
    return product_workspace_bytes(gated_product(*g, T, LORDBA_BF16));
}

int lordba_gated_forward(const lordba_gated *g, int64_t T, int dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!g) return LORDBA_EINVAL;
    int rc = check_gated(*g, T, dtype);
    if (rc != LORDBA_OK || T == 0) return rc;
    const Product q = gated_product(*g, T, dtype);
    rc = check_workspace(product_workspace_bytes(q), workspace, workspace_bytes);
    return rc != LORDBA_OK ? rc : launch_product(q, workspace, static_cast<cudaStream_t>(stream));
}

size_t lordba_gated_backward_workspace_bytes(const lordba_gated_grad *g, int64_t T)
{
    if (!g || bad_size(T, g->d_in) || bad_size(T, g->d_hidden) || T == 0) return 0;
    return grad_workspace(*g, T, LORDBA_BF16).bytes;
}

int lordba_gated_backward(const lordba_gated_grad *g, int64_t T, int dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!g) return LORDBA_EINVAL;
    int rc = check_grad(*g, T, dtype);
    if (rc != LORDBA_OK) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (T == 0) {
        // sums over no token
        for (void *w : {g->dw_gate, g->dw_up})
            if (w && cudaMemset2DAsync(w, (size_t)g->ld_dw * 2, 0, (size_t)g->d_in * 2, (size_t)g->d_hidden, s) != cudaSuccess) {
                cudaGetLastError();
                return LORDBA_ECUDA;
            }
        return LORDBA_OK;
    }
    const GradWorkspace w = grad_workspace(*g, T, dtype);
    rc = check_workspace(w.bytes, workspace, workspace_bytes);
    if (rc != LORDBA_OK) return rc;
    uint8_t *lo_gate = w.lo_bytes ? static_cast<uint8_t *>(workspace) : nullptr, *lo_up = lo_gate ? lo_gate + w.lo_bytes : nullptr;
    uint8_t *copies = static_cast<uint8_t *>(workspace) + 2 * w.lo_bytes;
    rc = launch_gated_grad(*g, T, dtype, lo_gate, lo_up, w.ld_lo, s);
    for (int i = 0; i < 2 && rc == LORDBA_OK; ++i) {
        if (!(i == 0 ? g->dx : g->dw_gate)) continue;
        Product q = i == 0 ? dx_product(*g, T, dtype) : dw_product(*g, T, dtype);
        if (lo_gate) {
            q.lo[0] = Operand{lo_gate, w.ld_lo, q.a[0].mn_major};
            q.lo[1] = Operand{lo_up, w.ld_lo, q.a[0].mn_major};
        }
        rc = launch_product(q, copies, s);
    }
    return rc;
}

int lordba_dropout(const void *x, int64_t ldx, const void *residual, int64_t ldr, void *out, int64_t ldo, int64_t T, int64_t d,
                   float p, uint64_t seed, uint64_t offset, int dtype, void *stream)
{
    if (!known_dtype(dtype)) return LORDBA_EUNSUPPORTED;
    if (!(p >= 0.0f && p <= 1.0f)) return LORDBA_EINVAL;
    if (T < 0 || T >= (int64_t(1) << 32) || d < 1 || d >= (int64_t(1) << 34) || ldx < d || ldo < d || (residual && ldr < d))
        return LORDBA_EINVAL;
    if (T == 0) return LORDBA_OK;
    const size_t e = elt(dtype);
    const Matrix mx{x, T, d, ldx, e}, mr{residual, T, d, ldr, e}, mo{out, T, d, ldo, e};
    for (const Matrix *m : {&mx, &mo, &mr}) {
        if (m == &mr && !residual) continue;
        const int rc = check_matrix(*m);
        if (rc != LORDBA_OK) return rc;
    }
    if ((meet(mo, mx) && !same(mo, mx)) || (meet(mo, mr) && !same(mo, mr))) return LORDBA_EINVAL;
    const int cut = (int)std::nearbyint((double)p * 65536.0);
    return launch_dropout(x, ldx, residual, ldr, out, ldo, T, d, cut, seed, offset, dtype, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
