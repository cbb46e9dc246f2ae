// Argument checks shared by the files of the C ABI (capi.cpp, capi_ops.cpp).
#pragma once

#include <hip/hip_runtime.h>

#include <initializer_list>

#include "launch.hpp"
#include "recblr.h"

namespace recblr {

constexpr size_t kWsAlign = 256;

inline size_t align_up(size_t v) { return (v + kWsAlign - 1) / kWsAlign * kWsAlign; }

struct Buf {
    const void* p;
    size_t bytes;
};

inline bool overlaps(Buf a, Buf b) {
    if (!a.p || !b.p || a.bytes == 0 || b.bytes == 0) return false;
    uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
    return a0 < b0 + b.bytes && b0 < a0 + a.bytes;
}

inline bool aligned(const void* p, size_t a) { return p == nullptr || ((uintptr_t)p % a) == 0; }

// Outputs must not overlap inputs or each other.
inline bool disjoint(std::initializer_list<Buf> outs, std::initializer_list<Buf> ins) {
    for (auto o = outs.begin(); o != outs.end(); ++o) {
        for (const Buf& i : ins)
            if (overlaps(*o, i)) return false;
        for (auto o2 = o + 1; o2 != outs.end(); ++o2)
            if (overlaps(*o, *o2)) return false;
    }
    return true;
}

inline int check_ws(void* ws, size_t ws_bytes, size_t need) {
    if (need == 0) return RECBLR_OK;
    if (ws == nullptr || ws_bytes < need || !aligned(ws, kWsAlign)) return RECBLR_ERR_WORKSPACE;
    return RECBLR_OK;
}

inline int status_of(hipError_t e) { return e == hipSuccess ? RECBLR_OK : RECBLR_ERR_HIP; }

inline IoType io_of(int io) { return io == RECBLR_BF16 ? IoType::kBf16 : IoType::kF32; }

inline size_t esz(int io) { return io == RECBLR_BF16 ? 2 : 4; }

}  // namespace recblr
