// C ABI of the operators around a 4-bit base: products with 4-bit weights, norms of queries and keys with the rotation,
// distillation.  Argument checks on the host, then launches; include/lordba.h states every contract.
#include <cmath>
#include <cstring>
#include <numeric>

#include "block_checks.h"

namespace lordba {
namespace {

// ---- 4-bit weights -----------------------------------------------------------------------------------------------
int64_t carrier_bytes(int64_t d_in) { return (d_in + 127) / 128 * 64; }
bool bad_group(int group) { return group < 32 || (group & (group - 1)); }
int64_t groups_of(int64_t d_in, int group) { return (d_in + group - 1) / group; }

struct Carrier {
    Matrix q, scale, zero;
};

Carrier carrier_of(const lordba_int4_proj &p)
{
    const int64_t g = groups_of(p.d_in, p.group);
    return Carrier{Matrix{p.q, p.d_out, carrier_bytes(p.d_in), p.ldq, 1}, Matrix{p.scale, p.d_out, g, p.ld_scale, 2},
                   Matrix{p.zero, p.d_out, g, p.ld_zero, 1}};
}

int check_carrier(const lordba_int4_proj &p)
{
    if (bad_size(p.d_out, p.d_in) || p.d_out < 1 || bad_group(p.group) || p.flags) return LORDBA_EINVAL;
    const int64_t g = groups_of(p.d_in, p.group);
    if (p.ldq < carrier_bytes(p.d_in) || p.ld_scale < g || (p.zero && p.ld_zero < g)) return LORDBA_EINVAL;
    return LORDBA_OK;
}

int check_carrier_pointers(const Carrier &c)
{
    int rc = check_matrix(c.q);
    if (rc == LORDBA_OK) rc = check_matrix(c.scale);
    if (rc == LORDBA_OK && too_far(c.zero)) rc = LORDBA_EINVAL;
    if (rc != LORDBA_OK) return rc;
    return aligned(c.q.p, 16) && c.q.ld % 16 == 0 ? LORDBA_OK : LORDBA_EALIGN;
}

int check_int4(const lordba_int4_proj &p, int64_t T, int dtype, bool backward)
{
    if (dtype != LORDBA_BF16 && dtype != LORDBA_F16) return LORDBA_EUNSUPPORTED;
    int rc = check_carrier(p);
    if (rc != LORDBA_OK) return rc;
    const int64_t n_in = backward ? p.d_out : p.d_in, n_out = backward ? p.d_in : p.d_out;
    if (T < 0 || T > kMaxRows || p.ld_in < n_in || p.ld_out < n_out) return LORDBA_EINVAL;
    if (T == 0) return LORDBA_OK;
    const Carrier c = carrier_of(p);
    const Matrix in{p.in, T, n_in, p.ld_in, 2}, out{p.out, T, n_out, p.ld_out, 2};
    rc = check_carrier_pointers(c);
    if (rc == LORDBA_OK) rc = check_matrix(in);
    if (rc == LORDBA_OK) rc = check_matrix(out);
    if (rc != LORDBA_OK) return rc;
    return meet(out, in) || meet(out, c.q) || meet(out, c.scale) || meet(out, c.zero) ? LORDBA_EINVAL : LORDBA_OK;
}

// The product that follows where the weights were laid out in 16 bits first (w, pitch ldw).
Product int4_product(const lordba_int4_proj &p, int64_t T, int dtype, bool backward, const void *w, int64_t ldw)
{
    Product q = {};
    q.kind = dtype == LORDBA_BF16 ? kProductBf16 : kProductF16;
    q.form = Product::kSingle;
    q.M = T;
    q.N = backward ? p.d_in : p.d_out;
    q.K = backward ? p.d_out : p.d_in;
    q.a[0] = Operand{p.in, p.ld_in, false};
    q.b[0] = Operand{w, ldw, backward};
    q.out[0] = p.out; q.ldo = p.ld_out; q.dtype = dtype;
    return q;
}

// How a product is done: a few tokens, some tens of them, or many, for which the weights are laid out in 16 bits first.  Up to 256 tokens,
// whatever the weights' size, widening them on the way (once for each 128 tokens) is as quick or quicker than laying them out, groups of 128, bf16:
//   tokens                     48             129             256
//   512 x 512             5.3 and 6.5     6.7 and 8.6     6.7 and 8.7 us      gradient 5.3 and 7.1,  6.7 and 8.6,  6.7 and 8.6
//   4096 x 4096            12 and 18       22 and 22       22 and 24           13 and 19,   20 and 24,   20 and 26
//   4096 -> 11008          21 and 39       46 and 48       49 and 49           22 and 42,   38 and 53,   38 and 56
//   4096 -> 32000          47 and 114     103 and 125     105 and 133          44 and 116,  88 and 139,  88 and 144
// (4096 -> 1024, 256 tokens, is the one shape measured that loses: 14.4 and 13.5).
enum class Int4Way { kFew, kStream, kWide };

Int4Way int4_way(const lordba_int4_proj &p, int64_t T, bool backward)
{
    if (!backward && T <= kInt4Few) return Int4Way::kFew;
    return T <= kInt4Stream && int4_stream_takes(p, T, backward) ? Int4Way::kStream : Int4Way::kWide;
}

struct Int4Workspace {
    Int4Way way;
    size_t first, bytes;         // of the weights in 16 bits, or of the activations on 16-byte boundaries where they are not; in all
    int64_t ld;
};

Int4Workspace int4_workspace(const lordba_int4_proj &p, int64_t T, int dtype, bool backward)
{
    Int4Workspace w = {};
    w.way = int4_way(p, T, backward);
    if (w.way != Int4Way::kWide) {
        w.ld = ((backward ? p.d_out : p.d_in) + 7) / 8 * 8;
        if (!aligned(p.in, 16) || (T > 1 && p.ld_in % 8)) w.first = ((size_t)T * (size_t)w.ld * 2 + 255) / 256 * 256;
        w.bytes = w.first;
        return w;
    }
    w.ld = (p.d_in + 7) / 8 * 8;
    w.first = ((size_t)p.d_out * (size_t)w.ld * 2 + 255) / 256 * 256;
    // the weights' place says only that they lie aligned
    w.bytes = w.first + product_workspace_bytes(int4_product(p, T, dtype, backward, reinterpret_cast<const void *>(uintptr_t(256)), w.ld));
    return w;
}

size_t int4_bytes(const lordba_int4_proj *p, int64_t T, bool backward)
{
    if (!p || check_carrier(*p) != LORDBA_OK || T <= 0 || T > kMaxRows) return 0;
    return int4_workspace(*p, T, LORDBA_BF16, backward).bytes;
}

int int4_call(const lordba_int4_proj *p, int64_t T, int dtype, void *workspace, size_t workspace_bytes, void *stream, bool backward)
{
    if (!p) return LORDBA_EINVAL;
    int rc = check_int4(*p, T, dtype, backward);
    if (rc != LORDBA_OK || T == 0) return rc;
    const Int4Workspace w = int4_workspace(*p, T, dtype, backward);
    rc = check_workspace(w.bytes, workspace, workspace_bytes);
    if (rc != LORDBA_OK) return rc;
    const cudaStream_t on = static_cast<cudaStream_t>(stream);
    lordba_int4_proj call = *p;
    if (w.way == Int4Way::kWide) {
        call.out = workspace;
        call.ld_out = w.ld;
        rc = launch_int4_dequantize(call, dtype, on);
        if (rc != LORDBA_OK) return rc;
        return launch_product(int4_product(*p, T, dtype, backward, workspace, w.ld), static_cast<uint8_t *>(workspace) + w.first, on);
    }
    if (T == 1) call.ld_in = w.ld;              // a single row has no pitch of its own
    if (w.first) {
        call.in = workspace;
        call.ld_in = w.ld;
        RepackList list = {};
        list.item[list.n++] = RepackList::Item{p->in, workspace, p->ld_in * 2, w.ld * 2, T, (backward ? p->d_out : p->d_in) * 2};
        rc = launch_repack(list, on);
        if (rc != LORDBA_OK) return rc;
    }
    return w.way == Int4Way::kFew ? launch_int4_few(call, T, dtype, on) : launch_int4_stream(call, T, dtype, backward, on);
}

// ---- heads --------------------------------------------------------------------------------------------------------
// Head vectors as a matrix: a row a token (or, head by head, a row a head), from the first entry to the last.  One that is
// neither, such as heads that share their entries, is a single row.  clear: no two vectors share an entry.  Sizes have been looked at (far_heads).
struct Heads {
    Matrix m;
    bool clear;
};

Heads heads_of(const lordba_heads &h, int64_t T, int64_t heads, int64_t d, size_t e)
{
    const int64_t token = T > 1 ? h.token : 0, head = heads > 1 ? h.head : 0;
    const int64_t by_token = (heads - 1) * head + d, by_head = (T - 1) * token + d;
    if ((heads == 1 || head >= d) && (T == 1 || token >= by_token)) return Heads{Matrix{h.p, T, by_token, T > 1 ? token : by_token, e}, true};
    if ((T == 1 || token >= d) && (heads == 1 || head >= by_head)) return Heads{Matrix{h.p, heads, by_head, heads > 1 ? head : by_head, e}, true};
    const int64_t all = (T - 1) * token + (heads - 1) * head + d;
    return Heads{Matrix{h.p, 1, all, all, e}, false};
}

// Whether head vectors reach further than any memory does.
bool far_heads(const lordba_heads &h, int64_t T, int64_t heads, size_t e)
{
    const int64_t most = kMostBytes / 4 / (int64_t)e;
    return (T > 1 && h.token > most / (T - 1)) || (heads > 1 && h.head > most / (heads - 1));
}

// Whether two sets of head vectors share an entry's bytes.  Beyond what `meet` sees: where all distances are multiples of one, such as in
// a joint projection's output that holds a head's query, key and value side by side, vectors that do not meet within it do not meet.
bool meet_heads(const lordba_heads &a, int64_t heads_a, const lordba_heads &b, int64_t heads_b, int64_t T, int64_t d, size_t e)
{
    if (!meet(heads_of(a, T, heads_a, d, e).m, heads_of(b, T, heads_b, d, e).m)) return false;
    int64_t step = 0;
    if (T > 1) step = std::gcd(a.token, b.token);
    if (heads_a > 1) step = std::gcd(step, a.head);
    if (heads_b > 1) step = std::gcd(step, b.head);
    if (step == 0) return true;
    const size_t pitch = (size_t)step * e, bytes = (size_t)d * e;
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
    const size_t shift = pb >= pa ? (pb - pa) % pitch : (pitch - (pa - pb) % pitch) % pitch;
    return !(bytes <= shift && shift + bytes <= pitch);
}

bool same_heads(const lordba_heads &a, const lordba_heads &b, int64_t T, int64_t heads)
{
    return a.p == b.p && (T <= 1 || a.token == b.token) && (heads <= 1 || a.head == b.head);
}

int check_norm_rope(const lordba_norm_rope_args &a, int64_t T, int dtype)
{
    if (!known_dtype(dtype)) return LORDBA_EUNSUPPORTED;
    if (a.flags & ~(LORDBA_ROPE_NO_NORM | LORDBA_ROPE_INTERLEAVED)) return LORDBA_EINVAL;
    if (a.d < 1 || a.heads_q < 1 || a.heads_k < 0 || a.rotary < 0 || a.rotary > a.d || a.rotary % 2) return LORDBA_EINVAL;
    if (a.d > LORDBA_ROPE_MAX_D || a.heads_q > (1 << 20) || a.heads_k > (1 << 20)) return LORDBA_EUNSUPPORTED;
    if ((a.w_q || a.w_k) && !known_dtype(a.w_dtype)) return LORDBA_EUNSUPPORTED;
    if ((a.flags & LORDBA_ROPE_NO_NORM) && (a.w_q || a.w_k)) return LORDBA_EINVAL;
    if (!(a.eps >= 0.0f) || std::isinf(a.eps)) return LORDBA_EINVAL;
    if (T < 0 || T > kMaxRows) return LORDBA_EINVAL;
    return LORDBA_OK;
}

// Vectors read and written by a call, and plain vectors read.
struct RopeCall {
    struct Item {
        const lordba_heads *h;
        int64_t heads;
        int side;                 // 0: queries, 1: keys
    };
    Item in[4], out[2];
    int n_in, n_out;
};

int check_heads(const RopeCall &c, const lordba_norm_rope_args &a, int64_t T, int dtype, float *const *dw)
{
    const size_t e = elt(dtype), ew = elt(a.w_dtype);
    for (int i = 0; i < c.n_in + c.n_out; ++i) {
        const RopeCall::Item &item = i < c.n_in ? c.in[i] : c.out[i - c.n_in];
        const lordba_heads &h = *item.h;
        if (!h.p || h.token < 0 || h.head < 0 || far_heads(h, T, item.heads, e)) return LORDBA_EINVAL;
        if (!aligned(h.p, e)) return LORDBA_EALIGN;
    }
    if (!a.positions || (a.rotary && !a.inv_freq)) return LORDBA_EINVAL;
    if (!aligned(a.positions, 8) || !aligned(a.inv_freq, 4)) return LORDBA_EALIGN;
    if ((a.w_q && !aligned(a.w_q, ew)) || (a.w_k && !aligned(a.w_k, ew))) return LORDBA_EALIGN;
    const Matrix flat[4] = {Matrix{a.positions, 1, T, T, 8}, Matrix{a.rotary ? a.inv_freq : nullptr, 1, a.rotary / 2, a.rotary / 2, 4},
                            Matrix{a.w_q, 1, a.d, a.d, ew}, Matrix{a.w_k, 1, a.d, a.d, ew}};
    Matrix outs[4];
    int n = 0;
    for (int i = 0; i < c.n_out; ++i) {
        const Heads h = heads_of(*c.out[i].h, T, c.out[i].heads, a.d, e);
        if (!h.clear) return LORDBA_EINVAL;
        outs[n++] = h.m;
        for (int j = 0; j < c.n_in; ++j) {
            // an input of the same side may be the output's very place
            if (c.in[j].side == c.out[i].side && same_heads(*c.out[i].h, *c.in[j].h, T, c.out[i].heads)) continue;
            if (meet_heads(*c.out[i].h, c.out[i].heads, *c.in[j].h, c.in[j].heads, T, a.d, e)) return LORDBA_EINVAL;
        }
    }
    if (n == 2 && meet_heads(*c.out[0].h, c.out[0].heads, *c.out[1].h, c.out[1].heads, T, a.d, e)) return LORDBA_EINVAL;
    const int vectors = n;
    for (int i = 0; dw && i < 2; ++i)
        if (dw[i]) {
            if (!aligned(dw[i], 4)) return LORDBA_EALIGN;
            const Matrix m{dw[i], 1, a.d, a.d, 4};
            for (int j = 0; j < c.n_in; ++j)
                if (meet(m, heads_of(*c.in[j].h, T, c.in[j].heads, a.d, e).m)) return LORDBA_EINVAL;
            outs[n++] = m;
        }
    for (int i = 0; i < n; ++i) {
        for (int j = i + 1 < vectors ? vectors : i + 1; j < n; ++j)
            if (meet(outs[i], outs[j])) return LORDBA_EINVAL;
        for (const Matrix &m : flat)
            if (meet(outs[i], m)) return LORDBA_EINVAL;
    }
    return LORDBA_OK;
}

// The arguments, without what would belong to keys where there are none: nothing of it is looked at.
lordba_norm_rope_args without_absent_keys(lordba_norm_rope_args a)
{
    if (a.heads_k == 0) {
        a.k = a.k_out = lordba_heads{};
        a.w_k = nullptr;
    }
    return a;
}

int check_rope_grad(const lordba_norm_rope_grad_args &a, int64_t T, int dtype)
{
    const int rc = check_norm_rope(a.f, T, dtype);
    if (rc != LORDBA_OK) return rc;
    if (a.dw_k && !a.f.heads_k) return LORDBA_EINVAL;
    if ((a.f.flags & LORDBA_ROPE_NO_NORM) && (a.dw_q || a.dw_k)) return LORDBA_EINVAL;
    return LORDBA_OK;
}

// ---- distillation ---------------------------------------------------------------------------------------------------
int check_distill(const lordba_distill &d, int64_t T, int dtype, bool backward)
{
    if (!known_dtype(dtype) || !known_dtype(d.teacher_dtype)) return LORDBA_EUNSUPPORTED;
    if (d.flags & ~LORDBA_DISTILL_IDS_64) return LORDBA_EINVAL;
    if (bad_size(T, d.vocab) || d.top < 1 || d.ld_logits < d.vocab || d.ld_ids < d.top || d.ld_teacher < d.top) return LORDBA_EINVAL;
    if (d.top > LORDBA_DISTILL_MAX_TOP) return LORDBA_EUNSUPPORTED;
    // its inverse, in powers of two, is a number too
    if (!(d.temperature > 0.0f) || std::isinf(d.temperature) || std::isinf((float)(1.4426950408889634 / (double)d.temperature))) return LORDBA_EINVAL;
    if (backward && !d.dlogits) return LORDBA_EINVAL;
    if (d.dlogits && d.ld_dlogits < d.vocab) return LORDBA_EINVAL;
    if (T == 0) return LORDBA_OK;
    const size_t e = elt(dtype);
    const Matrix z{d.logits, T, d.vocab, d.ld_logits, e}, ids{d.ids, T, d.top, d.ld_ids, size_t(d.flags & LORDBA_DISTILL_IDS_64 ? 8 : 4)},
        teacher{d.teacher, T, d.top, d.ld_teacher, elt(d.teacher_dtype)}, lse{d.lse, 1, T, T, 4};
    const Matrix weight{d.weight, 1, T, T, 4}, loss{backward ? nullptr : d.loss, 1, T, T, 4}, dz{d.dlogits, T, d.vocab, d.ld_dlogits, e};
    for (const Matrix *m : {&z, &ids, &teacher, &lse, &weight, &loss, &dz}) {
        if (!m->p && (m == &weight || (m == &loss && backward) || m == &dz)) continue;
        const int rc = check_matrix(*m);
        if (rc != LORDBA_OK) return rc;
    }
    const Matrix none{};
    const Matrix outs[3] = {dz, loss, backward ? none : lse};
    const Matrix ins[5] = {z, ids, teacher, weight, backward ? lse : none};
    for (int i = 0; i < 3; ++i) {
        for (int j = i + 1; j < 3; ++j)
            if (meet(outs[i], outs[j])) return LORDBA_EINVAL;
        for (int j = 0; j < 5; ++j)
            if (meet(outs[i], ins[j]) && !(i == 0 && j == 0 && same(dz, z))) return LORDBA_EINVAL;
    }
    return LORDBA_OK;
}

int distill_call(const lordba_distill *d, int64_t T, int dtype, void *workspace, size_t workspace_bytes, void *stream, bool backward)
{
    if (!d) return LORDBA_EINVAL;
    int rc = check_distill(*d, T, dtype, backward);
    if (rc != LORDBA_OK || T == 0) return rc;
    rc = check_workspace(distill_bytes(*d, T), workspace, workspace_bytes);
    return rc != LORDBA_OK ? rc : launch_distill(*d, T, dtype, backward, workspace, static_cast<cudaStream_t>(stream));
}

}  // namespace
}  // namespace lordba

using namespace lordba;

extern "C" {

int64_t lordba_int4_row_bytes(int64_t d_in) { return d_in < 1 || d_in > kMaxRows ? -1 : carrier_bytes(d_in); }

int lordba_int4_pack(const uint8_t *values, int64_t ldv, uint8_t *q, int64_t ldq, int64_t d_out, int64_t d_in, void *stream)
{
    if (bad_size(d_out, d_in) || ldv < d_in || ldq < carrier_bytes(d_in)) return LORDBA_EINVAL;
    if (d_out == 0) return LORDBA_OK;
    const Matrix v{values, d_out, d_in, ldv, 1}, c{q, d_out, carrier_bytes(d_in), ldq, 1};
    if (!v.p || !c.p || too_far(v) || too_far(c)) return LORDBA_EINVAL;
    if (!aligned(q, 16) || ldq % 16) return LORDBA_EALIGN;
    if (meet(v, c)) return LORDBA_EINVAL;
    return launch_int4_pack(values, ldv, q, ldq, d_out, d_in, static_cast<cudaStream_t>(stream));
}

int lordba_int4_quantize(const void *w, int64_t ldw, int wdtype, uint8_t *q, int64_t ldq, void *scale, int64_t ld_scale, uint8_t *zero,
                         int64_t ld_zero, int64_t d_out, int64_t d_in, int group, int dtype, void *stream)
{
    if (!known_dtype(wdtype) || (dtype != LORDBA_BF16 && dtype != LORDBA_F16)) return LORDBA_EUNSUPPORTED;
    lordba_int4_proj p = {};
    p.q = q; p.scale = scale; p.zero = zero;
    p.d_in = d_in; p.d_out = d_out < 1 ? 1 : d_out; p.ldq = ldq; p.ld_scale = ld_scale; p.ld_zero = ld_zero; p.group = group;
    int rc = check_carrier(p);
    if (rc != LORDBA_OK) return rc;
    if (d_out < 0 || ldw < d_in) return LORDBA_EINVAL;
    if (d_out == 0) return LORDBA_OK;
    const Carrier c = carrier_of(p);
    const Matrix m{w, d_out, d_in, ldw, elt(wdtype)};
    rc = check_carrier_pointers(c);
    if (rc == LORDBA_OK) rc = check_matrix(m);
    if (rc != LORDBA_OK) return rc;
    if (meet(m, c.q) || meet(m, c.scale) || meet(m, c.zero) || meet(c.q, c.scale) || meet(c.q, c.zero) || meet(c.scale, c.zero)) return LORDBA_EINVAL;
    return launch_int4_quantize(w, ldw, wdtype, q, ldq, scale, ld_scale, zero, ld_zero, d_out, d_in, group, dtype, static_cast<cudaStream_t>(stream));
}

int lordba_int4_dequantize(const lordba_int4_proj *p, int dtype, void *stream)
{
    if (!p) return LORDBA_EINVAL;
    if (dtype != LORDBA_BF16 && dtype != LORDBA_F16) return LORDBA_EUNSUPPORTED;
    int rc = check_carrier(*p);
    if (rc != LORDBA_OK) return rc;
    if (p->ld_out < p->d_in) return LORDBA_EINVAL;
    const Carrier c = carrier_of(*p);
    const Matrix out{p->out, p->d_out, p->d_in, p->ld_out, 2};
    rc = check_carrier_pointers(c);
    if (rc == LORDBA_OK) rc = check_matrix(out);
    if (rc != LORDBA_OK) return rc;
    if (meet(out, c.q) || meet(out, c.scale) || meet(out, c.zero)) return LORDBA_EINVAL;
    return launch_int4_dequantize(*p, dtype, static_cast<cudaStream_t>(stream));
}

size_t lordba_int4_linear_workspace_bytes(const lordba_int4_proj *p, int64_t T) { return int4_bytes(p, T, false); }

int lordba_int4_linear(const lordba_int4_proj *p, int64_t T, int dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    return int4_call(p, T, dtype, workspace, workspace_bytes, stream, false);
}

size_t lordba_int4_linear_backward_workspace_bytes(const lordba_int4_proj *p, int64_t T) { return int4_bytes(p, T, true); }

int lordba_int4_linear_backward(const lordba_int4_proj *p, int64_t T, int dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    return int4_call(p, T, dtype, workspace, workspace_bytes, stream, true);
}

int lordba_norm_rope(const lordba_norm_rope_args *given, int64_t T, int dtype, void *stream)
{
    if (!given) return LORDBA_EINVAL;
    const lordba_norm_rope_args own = without_absent_keys(*given), *a = &own;
    int rc = check_norm_rope(*a, T, dtype);
    if (rc != LORDBA_OK || T == 0) return rc;
    const int sides = a->heads_k ? 2 : 1;
    const RopeCall c{{{&a->q, a->heads_q, 0}, {&a->k, a->heads_k, 1}, {}, {}}, {{&a->q_out, a->heads_q, 0}, {&a->k_out, a->heads_k, 1}}, sides, sides};
    rc = check_heads(c, *a, T, dtype, nullptr);
    return rc != LORDBA_OK ? rc : launch_norm_rope(*a, T, dtype, static_cast<cudaStream_t>(stream));
}

size_t lordba_norm_rope_backward_workspace_bytes(const lordba_norm_rope_grad_args *given, int64_t T)
{
    if (!given) return 0;
    lordba_norm_rope_grad_args a = *given;
    a.f = without_absent_keys(a.f);
    return check_rope_grad(a, T, LORDBA_F32) != LORDBA_OK || T == 0 ? 0 : norm_rope_backward_bytes(a, T);
}

int lordba_norm_rope_backward(const lordba_norm_rope_grad_args *given, int64_t T, int dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!given) return LORDBA_EINVAL;
    lordba_norm_rope_grad_args own = *given;
    own.f = without_absent_keys(own.f);
    const lordba_norm_rope_grad_args *a = &own;
    int rc = check_rope_grad(*a, T, dtype);
    if (rc != LORDBA_OK) return rc;
    const lordba_norm_rope_args &f = a->f;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (T == 0) {
        // sums over no token
        for (float *dw : {a->dw_q, a->dw_k}) {
            if (!dw) continue;
            if (!aligned(dw, 4)) return LORDBA_EALIGN;
            if (cudaMemsetAsync(dw, 0, (size_t)f.d * 4, s) != cudaSuccess) {
                cudaGetLastError();
                return LORDBA_ECUDA;
            }
        }
        return LORDBA_OK;
    }
    const int sides = f.heads_k ? 2 : 1;
    const RopeCall c{{{&f.q, f.heads_q, 0}, {&f.q_out, f.heads_q, 0}, {&f.k, f.heads_k, 1}, {&f.k_out, f.heads_k, 1}},
                     {{&a->dq, f.heads_q, 0}, {&a->dk, f.heads_k, 1}}, 2 * sides, sides};
    float *const dw[2] = {a->dw_q, a->dw_k};
    rc = check_heads(c, f, T, dtype, dw);
    if (rc != LORDBA_OK) return rc;
    rc = check_workspace(norm_rope_backward_bytes(*a, T), workspace, workspace_bytes);
    return rc != LORDBA_OK ? rc : launch_norm_rope_backward(*a, T, dtype, workspace, s);
}

size_t lordba_distill_workspace_bytes(const lordba_distill *d, int64_t T)
{
    if (!d || bad_size(T, d->vocab) || d->top < 1 || d->top > LORDBA_DISTILL_MAX_TOP) return 0;
    return distill_bytes(*d, T);
}

int lordba_distill_loss(const lordba_distill *d, int64_t T, int dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    return distill_call(d, T, dtype, workspace, workspace_bytes, stream, false);
}

int lordba_distill_backward(const lordba_distill *d, int64_t T, int dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    return distill_call(d, T, dtype, workspace, workspace_bytes, stream, true);
}

}  // extern "C"
