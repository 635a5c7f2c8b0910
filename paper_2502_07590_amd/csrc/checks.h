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

}  // namespace dsv
