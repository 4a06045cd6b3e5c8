// What the page and attention entry points share: checks of arguments that need no device.
#pragma once
#include "../../include/preft.h"
#include "common.hpp"

namespace preft {

// Pages hold 8..1024 tokens, a power of two: the rows that one load of a wavefront fetches then lie in one page.
inline int page_shift_of(int32_t page_size)
{
    for (int s = 3; s <= 10; ++s)
        if (page_size == 1 << s) return s;
    return -1;
}

inline int64_t elem_bytes(int dtype) { return dtype == PREFT_BF16 ? 2 : 4; }

inline int check_heads(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int dtype)
{
    if (dtype != PREFT_F32 && dtype != PREFT_BF16) return PREFT_EINVAL;
    if (n_heads < 1 || n_kv_heads < 1 || n_heads > PREFT_MAX_HEADS || n_heads % n_kv_heads != 0) return PREFT_EINVAL;
    if (head_dim != 64 && head_dim != 128) return PREFT_EUNSUPPORTED;
    return PREFT_OK;
}

// rows of `width` elements, ld apart.  2^20 elements apart at most: offsets inside a tile of rows stay far below 2^31.
inline int check_rows(const void *p, int64_t ld, int64_t width, int dtype)
{
    const int64_t per16 = 16 / elem_bytes(dtype);
    if (!p || ld < width || ld > (1 << 20)) return PREFT_EINVAL;
    if ((reinterpret_cast<uintptr_t>(p) & 15) != 0 || ld % per16 != 0) return PREFT_EALIGN;
    return PREFT_OK;
}

struct Span {
    const void *p;
    int64_t bytes;
    bool meets(const Span &o) const
    {
        const char *a = (const char *)p, *b = (const char *)o.p;
        return a < b + o.bytes && b < a + bytes;
    }
};

// Two matrices of `rows` rows overlap, unless they are disjoint column ranges of one buffer.
inline bool rows_meet(const void *p, int64_t ldp, int64_t wp, const void *q, int64_t ldq, int64_t wq, int64_t rows, int dtype)
{
    const int64_t e = elem_bytes(dtype);
    if (rows <= 0) return false;
    const Span a{p, ((rows - 1) * ldp + wp) * e}, b{q, ((rows - 1) * ldq + wq) * e};
    if (!a.meets(b)) return false;
    if (ldp != ldq) return true;
    const char *x = (const char *)p, *y = (const char *)q;
    const int64_t pitch = ldp * e, d = x < y ? y - x : x - y;
    const int64_t first = x < y ? wp * e : wq * e, second = x < y ? wq * e : wp * e;
    return !(d >= first && d + second <= pitch);
}

inline bool aligned_workspace(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Workgroups of kernels whose wavefronts take a row each.  A launch may have fewer than 2^32 threads in a dimension, and of one that asks for more the remainder runs, without an error: the threads
// stand along y, so that along x only workgroups count, and these are fewer than 2^31 for any number of rows.
inline dim3 row_threads() { return dim3(1, 256); }

inline int launched() { return hipGetLastError() == hipSuccess ? PREFT_OK : PREFT_EHIP; }

}  // namespace preft
