// Argument checks that every file of entry points shares (host only).
#pragma once

#include <initializer_list>

#include "common.h"

namespace dsv {

inline bool supported_d(int d) { return d == 64 || d == 128; }
inline bool supported_dtype(int t) { return t == DSV_F32 || t == DSV_BF16; }
inline size_t esize(int dtype) { return dtype == DSV_BF16 ? 2 : 4; }
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// true when every pointer is non-null and 16-byte aligned
inline bool ok_ptrs(std::initializer_list<const void *> ps)
{
    for (const void *p : ps)
        if (!p || !aligned16(p)) return false;
    return true;
}

inline dsv_status check_workspace(const void *ws, size_t have, size_t need)
{
    if (need == 0) return DSV_OK;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || have < need) return DSV_EWORKSPACE;
    return DSV_OK;
}

// Strides of an input: whole 16 bytes.  Of an output: also no two of its rows on the same memory.
inline bool ok_strides(const dsv_rows &s, size_t es)
{
    const int64_t unit = 16 / (int64_t)es, most = (int64_t)1 << 40;
    return s.row >= 0 && s.head >= 0 && s.row < most && s.head < most && s.row % unit == 0 && s.head % unit == 0;
}
typedef __int128 wide_t;  // counts below 2^31 times strides below 2^40: more than 64 bits
inline bool rows_apart(const dsv_rows &s, int64_t rows, int64_t heads, int64_t n)
{
    if (rows <= 1 && heads <= 1) return true;
    if (rows <= 1) return s.head >= n;
    if (heads <= 1) return s.row >= n;
    return (s.head >= n && s.row >= (wide_t)(heads - 1) * s.head + n) || (s.row >= n && s.head >= (wide_t)(rows - 1) * s.row + n);
}

// every pointer on an element
inline bool on_elements(std::initializer_list<const void *> ps, size_t es)
{
    for (const void *q : ps)
        if (reinterpret_cast<uintptr_t>(q) % es) return false;
    return true;
}
}  // namespace dsv
