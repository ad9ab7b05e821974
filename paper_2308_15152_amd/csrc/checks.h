// Argument checks shared by the C entry points (host only).
#pragma once

#include <stdint.h>

#include <initializer_list>

#include <hip/hip_runtime_api.h>

namespace sgemm_emu {

// Keeps e as the calling thread's last HIP error; returns SGEMM_EMU_ERR_HIP.
int hip_fail(hipError_t e);

struct Extent {
    uintptr_t lo, hi;  // [lo, hi) in bytes; empty if lo == hi
    bool ok;           // false: the span runs past the end of the address space
};

// Bytes spanned by `items` row-major matrices of rows x cols with leading
// dimension ld and item stride s (elements of `elem` bytes), starting at p.
// All arguments are non-negative; the span is computed in 128 bits, so no
// stride or leading dimension can wrap it.
inline Extent extent(const void* p, int64_t items, int64_t rows, int64_t cols, int64_t ld, int64_t s,
              int64_t elem = sizeof(float)) {
    Extent e{(uintptr_t)p, (uintptr_t)p, true};
    if (items <= 0 || rows <= 0 || cols <= 0) return e;
    const __int128 last = (__int128)(items - 1) * s + (__int128)(rows - 1) * ld + cols;
    const __int128 bytes = last * elem;
    if (bytes > (__int128)(UINTPTR_MAX - e.lo)) {
        e.ok = false;
        return e;
    }
    e.hi = e.lo + (uintptr_t)bytes;
    return e;
}

inline bool all_ok(std::initializer_list<Extent> es) {
    for (const Extent& e : es)
        if (!e.ok) return false;
    return true;
}

inline bool overlap(Extent a, Extent b) {
    if (a.lo == a.hi || b.lo == b.hi) return false;
    return a.lo < b.hi && b.lo < a.hi;
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

}  // namespace sgemm_emu
