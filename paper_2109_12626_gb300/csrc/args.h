// args.h -- checks of the matrix arguments of a call, and refusals.  Not part of
// the public ABI.
#pragma once

#include <cstdint>
#include <cstdio>

#include "dpdr_internal.h"

namespace dpdr {
namespace proj {

// A refusal as "who: what", without allocating.
inline int refuse(const char* who, const char* what, const char* more = "")
{
    char msg[200];
    std::snprintf(msg, sizeof msg, "%s: %s%s%s", who, what, *more ? " " : "", more);
    return fail_c(DPDR_ERR_INVALID, msg);
}

// A matrix argument in bytes: which range of memory it touches, and which
// part of each row of its pitch.
struct Span {
    uintptr_t lo = 0, hi = 0, pitch = 0, width = 0;
};

inline Span span_of(const dpdr_matrix& m, int64_t rows, int64_t cols, int esize)
{
    Span s;
    if (rows == 0 || cols == 0) return s;
    s.lo = reinterpret_cast<uintptr_t>(m.data);
    const uintptr_t last = uintptr_t(rows - 1) * uintptr_t(m.row_stride) + uintptr_t(cols - 1) * uintptr_t(m.col_stride);
    s.hi = s.lo + (last + 1) * esize;
    s.pitch = uintptr_t(m.row_stride) * esize;
    s.width = m.col_stride == 1 ? uintptr_t(cols) * esize : s.pitch;
    return s;
}

// Whether two arguments may share a byte.  Column slices of one wider array
// (equal pitch, disjoint parts of it) do not.
inline bool overlap(const Span& a, const Span& b)
{
    if (a.lo == a.hi || b.lo == b.hi || a.hi <= b.lo || b.hi <= a.lo) return false;
    if (a.pitch == b.pitch && a.pitch > 0 && a.width <= a.pitch && b.width <= b.pitch) {
        const uintptr_t d = b.lo >= a.lo ? (b.lo - a.lo) % a.pitch : (a.pitch - (a.lo - b.lo) % a.pitch) % a.pitch;
        if (d >= a.width && d + b.width <= a.pitch) return false;
    }
    return true;
}

// The arguments of one call, checked as they are added.
struct Args {
    const char* who;
    Span in[8], out[4];
    int nin = 0, nout = 0;
    int rc = DPDR_OK;

    void refuse(const char* name, const char* what)
    {
        if (rc == DPDR_OK) rc = proj::refuse(who, name, what);
    }
    void input(const char* name, const dpdr_matrix* m, int64_t rows, int64_t cols, int esize)
    {
        if (!m) return refuse(name, "is NULL");
        check(name, *m, rows, cols, esize);
        if (m->row_stride < 0 || m->col_stride < 0) return refuse(name, "has a negative stride");
        in[nin++] = span_of(*m, rows, cols, esize);
    }
    void output(const char* name, const dpdr_matrix* m, int64_t rows, int64_t cols, int esize)
    {
        if (!m) return refuse(name, "is NULL");
        check(name, *m, rows, cols, esize);
        if (cols > 1 && m->col_stride != 1) return refuse(name, "needs col_stride 1");
        if (rows > 1 && m->row_stride < cols) return refuse(name, "has rows that overlap");
        dpdr_matrix unit = *m;
        unit.col_stride = 1;
        out[nout++] = span_of(unit, rows, cols, esize);
    }
    void check(const char* name, const dpdr_matrix& m, int64_t rows, int64_t cols, int esize)
    {
        if (rows == 0 || cols == 0) return;
        if (!m.data) return refuse(name, "has no address");
        if (reinterpret_cast<uintptr_t>(m.data) % uintptr_t(esize)) refuse(name, "is not aligned to its element");
        // byte offsets stay within 2^62
        const __int128 far = (__int128)(rows - 1) * m.row_stride + (__int128)(cols - 1) * m.col_stride;
        if (far > (__int128(1) << 59)) refuse(name, "reaches too far");
    }
    // matrices of one shape, `stride` elements apart, each with contiguous rows
    void stack(const char* name, const dpdr_matrices* m, int64_t count, int64_t rows, int64_t cols, int esize)
    {
        if (!m) return refuse(name, "is NULL");
        const dpdr_matrix one{m->data, m->row_stride, m->col_stride}, all{m->data, m->stride, 1};
        check(name, one, rows, cols, esize);
        if (m->stride < 0 || m->row_stride < 0) return refuse(name, "has a negative stride");
        if (cols > 1 && m->col_stride != 1) return refuse(name, "needs col_stride 1");
        if (rc != DPDR_OK) return;
        const int64_t each = (rows - 1) * m->row_stride + cols;   // elements from the first to the last
        check(name, all, count, each, esize);
        if (rc != DPDR_OK) return;
        in[nin] = span_of(all, count, each, esize);
        in[nin].pitch = in[nin].width = 0;
        nin++;
    }
    void vector(const char* name, const void* p, int64_t n, int esize, bool result)
    {
        const dpdr_matrix m{const_cast<void*>(p), n, 1};
        if (result) output(name, &m, 1, n, esize);
        else input(name, &m, 1, n, esize);
    }
    // no result may touch another argument (but the residual, which is checked
    // on its own)
    int done()
    {
        for (int i = 0; i < nout && rc == DPDR_OK; i++) {
            for (int k = 0; k < nin; k++)
                if (overlap(out[i], in[k])) return rc = proj::refuse(who, "a result overlaps an input");
            for (int k = 0; k < i; k++)
                if (overlap(out[i], out[k])) return rc = proj::refuse(who, "two results overlap");
        }
        return rc;
    }
};

}  // namespace proj
}  // namespace dpdr
