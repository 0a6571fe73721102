// Argument checks shared by the entry points next to the adapters (block_api.cu, base4_api.cu).
#pragma once

#include "lordba_internal.h"

namespace lordba {

constexpr int64_t kMaxRows = (int64_t(1) << 31) - 512;     // rows and columns are 32-bit coordinates of the copy engine

inline size_t elt(int dtype) { return dtype == LORDBA_F32 ? 4 : 2; }

// A matrix of a call: rows x cols elements of e bytes, row pitch ld elements.
struct Matrix {
    const void *p;
    int64_t rows, cols, ld;
    size_t e;
    size_t span() const { return rows > 0 ? ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * e : 0; }
};

// Whether two matrices share an element's bytes.  Matrices of one pitch may be interleaved (the two halves
// of a joint buffer): they are apart when their columns are.
inline bool meet(const Matrix &a, const Matrix &b)
{
    if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0) return false;
    if (!overlaps(a.p, a.span(), b.p, b.span())) return false;
    const size_t pitch = (size_t)a.ld * a.e;
    if (pitch != (size_t)b.ld * b.e) return true;
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
    const size_t shift = pb >= pa ? (pb - pa) % pitch : (pitch - (pa - pb) % pitch) % pitch;   // of b's columns against a's
    return !((size_t)a.cols * a.e <= shift && shift + (size_t)b.cols * b.e <= pitch);
}

inline bool same(const Matrix &a, const Matrix &b) { return a.p == b.p && a.ld == b.ld && a.e == b.e && a.cols == b.cols; }

// No range of addresses is longer, and sizes within it can be multiplied out in 64 bits.
constexpr int64_t kMostBytes = int64_t(1) << 56;
inline bool too_far(const Matrix &m)
{
    if (!m.p) return false;
    const int64_t most = kMostBytes / (int64_t)m.e;
    return m.ld > most || m.cols > most || (m.rows > 1 && m.ld > (most - m.cols) / (m.rows - 1));
}

// Of each matrix that a call is given, before `meet` looks at it.
inline int check_matrix(const Matrix &m)
{
    if (!m.p || too_far(m)) return LORDBA_EINVAL;
    if (!aligned(m.p, m.e)) return LORDBA_EALIGN;
    return LORDBA_OK;
}

inline int check_workspace(size_t need, const void *ws, size_t bytes)
{
    if (need == 0) return LORDBA_OK;
    if (!ws || bytes < need) return LORDBA_EINVAL;
    return aligned(ws, 256) ? LORDBA_OK : LORDBA_EALIGN;
}

// Sizes and pitches of a product: what can be said without looking at a pointer.
inline bool bad_size(int64_t rows, int64_t cols) { return rows < 0 || cols < 1 || rows > kMaxRows || cols > kMaxRows; }

}  // namespace lordba
