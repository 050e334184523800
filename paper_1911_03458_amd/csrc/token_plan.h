// Plan code that the token operators share (token_plan.cpp, token_mixer_plan.cpp).  Host code only.
#pragma once

#include <cmath>
#include <cstring>
#include <limits>
#include <new>

#include "tokens.h"

namespace merit {

constexpr int64_t MAX_CHANNELS = 1 << 24, MAX_ROWS = std::numeric_limits<int32_t>::max() - 1023;   // (rows are counted in 32 bits, past the last by up to four of a workgroup's)
constexpr int64_t MAX_THREADS = 1ll << 32;              // a launch holds fewer
constexpr int64_t MAX_BLOCKS = MAX_THREADS / 256;       // workgroups of 256 threads (where a kernel has more: at its rule)

// elements of a tensor at most: scratch memory in bytes and every offset stay far from 2^63
inline bool too_large(int64_t a, int64_t b, int64_t c) { return a != 0 && b != 0 && a > (1ll << 46) / b / c; }

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int elem_bytes(int type) { return type == MERIT_F32 ? 4 : 2; }
inline bool type_ok(int type) { return type == MERIT_F16 || type == MERIT_BF16 || type == MERIT_F32; }

// ---- operands --------------------------------------------------------------------------
// Reads views one by one; the first thing wrong with one of them stays.
struct Views {
    int type;
    merit_status st = MERIT_OK;

    bool take(const merit_view &v, bool required, int bytes)
    {
        if (!v.data) {
            if (required && st == MERIT_OK) st = MERIT_ERR_NULL;
            return false;
        }
        if (reinterpret_cast<uintptr_t>(v.data) % (uintptr_t)bytes != 0 && st == MERIT_OK) st = MERIT_ERR_ALIGNMENT;
        return true;
    }
    void want(const merit_view &v, int dtype)
    {
        if (v.dtype != dtype && st == MERIT_OK) st = MERIT_ERR_INVALID_ARG;
    }
    Rows rows(const merit_view &v, bool required = true)
    {
        if (!take(v, required, elem_bytes(type))) return Rows{nullptr, 0, 0};
        want(v, type);
        return Rows{v.data, v.stride[0], v.stride[1]};
    }
    float *f32(const merit_view &v, bool required = false)
    {
        if (!take(v, required, 4)) return nullptr;
        want(v, MERIT_F32);
        return static_cast<float *>(v.data);
    }
    Param param(const merit_view &v, bool required = false)
    {
        if (!take(v, required, v.dtype == MERIT_F32 ? 4 : 2)) return Param{nullptr, 0};
        if (v.dtype != MERIT_F32) want(v, type);
        return Param{v.data, v.dtype == MERIT_F32};
    }
    const int32_t *lens(const merit_view &v)
    {
        return take(v, false, 4) ? static_cast<const int32_t *>(v.data) : nullptr;
    }
};

// whether every row of `r` starts on a boundary of `vec` elements (n0, n1: its extents; the stride of an extent of 1 says nothing)
inline bool wide(const Rows &r, int64_t n0, int64_t n1, int vec, int type)
{
    return !r.data || (reinterpret_cast<uintptr_t>(r.data) % (uintptr_t)(vec * elem_bytes(type)) == 0 && (n0 <= 1 || r.s0 % vec == 0) &&
                       (n1 <= 1 || r.s1 % vec == 0));
}

inline merit_status scratch(int64_t need, void *workspace, int64_t bytes)
{
    if (need == 0) return MERIT_OK;
    if (!workspace) return MERIT_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return MERIT_ERR_ALIGNMENT;
    return bytes >= need ? MERIT_OK : MERIT_ERR_INVALID_ARG;
}

inline merit_status done(hipError_t e) { return e == hipSuccess ? MERIT_OK : MERIT_ERR_HIP; }

inline merit_token_plan *new_plan(int kind, int type)
{
    merit_token_plan *p = new (std::nothrow) merit_token_plan;
    if (!p) return nullptr;
    std::memset(static_cast<void *>(p), 0, sizeof(*p));
    p->kind = kind;
    p->type = type;
    return p;
}

enum { NORM = 0, CONV = 1, SCAN = 2, DELTA = 3, BLOCK = 4 };

}  // namespace merit
