// Argument checks shared by the operators around the recurrences (selective block, gated
// recurrence, embedding, logits): sizes, rows a distance apart, workspaces, and all buffers
// of a call at once.
#pragma once

#include "lh_check.hpp"

namespace lh {
namespace check {

inline size_t esize(lh_dtype t) { return t == LH_BF16 ? 2 : 4; }

inline lh_status check_at_least(const char* name, int64_t v, int64_t least)
{
    if (v < least)
        return fail(LH_ERR_INVALID_ARG, "%s = %lld must be >= %lld", name, (long long)v,
                    (long long)least);
    return LH_OK;
}

// n = a b c ... must stay small enough for byte offsets.
template <typename... I>
lh_status check_product(const char* what, I... v)
{
    int64_t n = 16;
    for (int64_t i : {int64_t(v)...})
        if (!mul_ok(n, i > 0 ? i : 1, &n))
            return fail(LH_ERR_INVALID_ARG, "sizes overflow (%s)", what);
    return LH_OK;
}

// One launch holds fewer than 2^32 threads.
inline lh_status check_threads(int64_t threads)
{
    if (threads >= (INT64_C(1) << 32))
        return fail(LH_ERR_INVALID_ARG, "sizes need %lld threads, a launch holds fewer than 2^32",
                    (long long)threads);
    return LH_OK;
}

// `rows` rows of `width` elements, `ld` apart.
inline Buf row_buf(const char* name, const void* p, int64_t rows, int64_t width, int64_t ld, size_t es)
{
    return buf(name, p, p && rows > 0 ? es * (size_t(rows - 1) * ld + width) : 0);
}

inline lh_status check_ld(const char* name, int64_t ld, int64_t width, int64_t rows)
{
    if (ld < width)
        return fail(LH_ERR_INVALID_ARG, "%s = %lld must be >= the row's %lld elements", name,
                    (long long)ld, (long long)width);
    return check_product(name, rows, ld);
}

inline lh_status check_workspace(const Buf& b, size_t have)
{
    const size_t need = b.hi - b.lo;
    if (need == 0) return LH_OK;
    if (!b.lo) return fail(LH_ERR_WORKSPACE, "workspace is NULL but %zu bytes are needed", need);
    if (have < need)
        return fail(LH_ERR_WORKSPACE, "workspace has %zu bytes, %zu are needed", have, need);
    return check_align(b, 256);
}

// Every buffer of a call: alignments, no output over another buffer, all accessible.
// An output that may be the same buffer as an input names it in `same`.
struct Arg {
    Buf b;
    size_t align;
    const void* same[2] = {nullptr, nullptr};
};

template <size_t I, size_t O>
lh_status check_buffers(const Arg (&ins)[I], const Arg (&outs)[O])
{
    lh_status s;
    for (const Arg& a : ins)
        if ((s = check_align(a.b, a.align))) return s;
    for (const Arg& a : outs)
        if ((s = check_align(a.b, a.align))) return s;
    for (const Arg& o : outs) {
        for (const Arg& i : ins) {
            const uintptr_t lo = i.b.lo;
            const bool same = lo == o.b.lo && i.b.hi == o.b.hi &&
                              (lo == reinterpret_cast<uintptr_t>(o.same[0]) ||
                               lo == reinterpret_cast<uintptr_t>(o.same[1]));
            if (!same && overlaps(o.b, i.b))
                return fail(LH_ERR_OVERLAP, "%s overlaps %s", o.b.name, i.b.name);
        }
        for (const Arg& p : outs)
            if (&p != &o && overlaps(o.b, p.b))
                return fail(LH_ERR_OVERLAP, "%s overlaps %s", o.b.name, p.b.name);
    }
    int dev = 0;
    if ((s = check_device(&dev)) != LH_OK) return s;
    // the allocations found accessible in this call: a framework's tensors share them
    Buf seen[I + O] = {};
    size_t n = 0;
    auto accessible = [&](const Buf& b) {
        for (size_t i = 0; i < n; ++i)
            if (b.lo >= seen[i].lo && b.hi <= seen[i].hi) return LH_OK;
        Buf found{"", 0, 0};
        const lh_status r = check_accessible(b, dev, &found);
        if (found.hi > found.lo) seen[n++] = found;
        return r;
    };
    for (const Arg& a : ins)
        if ((s = accessible(a.b)) != LH_OK) return s;
    for (const Arg& a : outs)
        if ((s = accessible(a.b)) != LH_OK) return s;
    return LH_OK;
}

}  // namespace check
}  // namespace lh
