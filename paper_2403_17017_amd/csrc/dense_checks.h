// Checks of arguments that the C entry points over dense rows share.
#pragma once
#include "dense_launch.h"

namespace seer {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool is_float(int type) { return type == SEER_F32 || type == SEER_BF16 || type == SEER_F16; }
inline size_t size_of(int type) { return type == SEER_F32 ? 4 : type == SEER_I8 ? 1 : 2; }

// Bytes from `begin` to `end`; nothing if there are no elements.
struct Extent {
    uintptr_t begin, end;
};
inline Extent extent(const void *p, size_t bytes)
{
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    return {b, b + bytes};
}
inline Extent extent(const seer_dense *m)
{
    if (m->rows == 0 || m->cols == 0) return {0, 0};
    return extent(m->data, (size_t)((m->rows - 1) * m->ld + m->cols) * size_of(m->type));
}
inline bool overlap(Extent a, Extent b) { return a.begin < b.end && b.begin < a.end; }

inline bool bad_pointer(const void *p, size_t multiple) { return !p || reinterpret_cast<uintptr_t>(p) % multiple != 0; }

// A dense matrix of the expected size; type -1: one of the floating types.
inline int check_dense(const seer_dense *m, int64_t rows, int64_t cols, int type)
{
    if (!m || m->rows != rows || m->cols != cols || m->ld < cols) return SEER_EINVAL;
    if (rows < 0 || cols < 0 || rows > INT32_MAX || cols > INT32_MAX) return SEER_EINVAL;
    if (type < 0 ? !is_float(m->type) : m->type != type) return SEER_EINVAL;
    // (the byte extent has to fit an address)
    if (rows > 0 && m->ld > (INT64_MAX / 8) / rows) return SEER_EINVAL;
    if (rows > 0 && cols > 0 && bad_pointer(m->data, size_of(m->type))) return SEER_EINVAL;
    return SEER_OK;
}

inline int check_routing(const seer_routing *r, bool entries)
{
    if (!r || r->tokens < 0 || r->choices < 1 || r->experts < 1) return SEER_EINVAL;
    if (r->experts > SEER_MAX_EXPERTS) return SEER_ELIMIT;
    if ((int64_t)r->tokens * r->choices > INT32_MAX) return SEER_EINVAL;
    if (entries && r->tokens > 0 && bad_pointer(r->choice_slot, 4)) return SEER_EINVAL;
    return SEER_OK;
}

inline RouteRows rows_of(const seer_routing *r, int64_t cols)
{
    return RouteRows{r->choice_slot, (uint32_t)r->tokens, (uint32_t)r->choices, (uint32_t)cols};
}

inline int done()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SEER_OK : hip_fail(e);
}

inline hipStream_t on(void *stream) { return static_cast<hipStream_t>(stream); }

} // namespace seer
