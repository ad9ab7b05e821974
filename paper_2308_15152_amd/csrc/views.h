// What the checks of the token mixing entries ask of tensor views (host only).
#pragma once

#include <stdint.h>

#include <algorithm>
#include <utility>

#include "checks.h"
#include "mixing_emu.h"

namespace sgemm_emu {

// A tensor argument: its view, sizes and element bytes.
struct Tensor {
    const sgemm_emu_view_t& v;
    int64_t batch, tokens, heads, size, elem;
    bool empty() const { return batch == 0 || tokens == 0 || heads == 0 || size == 0; }
};

inline bool negative(const sgemm_emu_view_t& v) { return v.batch < 0 || v.token < 0 || v.head < 0; }

// Bytes the tensor spans (strides not negative).
inline Extent span(const Tensor& t) {
    Extent e{(uintptr_t)t.v.p, (uintptr_t)t.v.p, true};
    if (t.empty()) return e;
    const __int128 last = (__int128)(t.batch - 1) * t.v.batch + (__int128)(t.tokens - 1) * t.v.token +
                          (__int128)(t.heads - 1) * t.v.head + t.size;
    const __int128 bytes = last * t.elem;
    if (bytes > (__int128)(UINTPTR_MAX - e.lo)) {
        e.ok = false;
        return e;
    }
    e.hi = e.lo + (uintptr_t)bytes;
    return e;
}

// Whether the elements of an output are apart: with the dimensions of more
// than one entry ordered by stride, each stride steps over all that the
// smaller ones reach.
inline bool apart(const Tensor& t) {
    if (t.empty()) return true;
    int64_t n[3] = {t.batch, t.tokens, t.heads}, s[3] = {t.v.batch, t.v.token, t.v.head};
    for (int i = 0; i < 2; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (s[j] < s[i]) {
                std::swap(s[i], s[j]);
                std::swap(n[i], n[j]);
            }
    __int128 reach = t.size;
    for (int i = 0; i < 3; ++i) {
        if (n[i] <= 1) continue;
        if (s[i] < reach) return false;
        reach += (__int128)(n[i] - 1) * s[i];
    }
    return true;
}

// Whether two outputs, each with its own elements apart, share any.  They may lie in
// one buffer between each other (slices of one projection's gradient): where the
// longest of their strides is the same, the blocks that it steps over are compared in
// pairs, from the outside in, and what is left as whole stretches.
inline bool meet(const Tensor& a, const Tensor& b) {
    if (a.empty() || b.empty()) return false;
    struct Steps {
        __int128 step[3];
        int64_t count[3];
        __int128 reach;  // bytes
    };
    const auto steps = [](const Tensor& t) {
        Steps s{{t.v.batch * (__int128)t.elem, t.v.token * (__int128)t.elem,
                 t.v.head * (__int128)t.elem},
                {t.batch, t.tokens, t.heads},
                t.size * (__int128)t.elem};
        for (int i = 0; i < 3; ++i) {
            if (s.count[i] == 1) s.step[i] = 0;
            s.reach += (s.count[i] - 1) * s.step[i];
        }
        return s;
    };
    // by: bytes from a's first element to b's
    const auto shared = [](auto&& self, Steps x, Steps y, __int128 by) -> bool {
        if (by >= x.reach || by <= -y.reach) return false;
        __int128 step = 0;
        for (int i = 0; i < 3; ++i) step = std::max(step, std::max(x.step[i], y.step[i]));
        if (step == 0) return true;
        const auto inside = [&](Steps& s) {  // the block that it steps over; how many
            for (int i = 0; i < 3; ++i)
                if (s.step[i] == step) {
                    const int64_t n = s.count[i];
                    s.reach -= (n - 1) * step;
                    s.step[i] = 0;
                    return n;
                }
            return int64_t{1};
        };
        const int64_t n = inside(x), m = inside(y);
        if (x.reach > step || y.reach > step) return true;  // no such blocks
        // block j of b less block i of a: those that can meet, at most two
        __int128 d = -by / step - 2;
        for (const __int128 end = d + 4; d <= end; ++d)
            if (d > -n && d < m && self(self, x, y, by + d * step)) return true;
        return false;
    };
    return shared(shared, steps(a), steps(b),
                  (__int128)(uintptr_t)b.v.p - (__int128)(uintptr_t)a.v.p);
}

inline bool same(const sgemm_emu_view_t& a, const sgemm_emu_view_t& b) {
    return a.p == b.p && a.batch == b.batch && a.token == b.token && a.head == b.head;
}

}  // namespace sgemm_emu
