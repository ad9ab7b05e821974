// What the checks of the token mixing and attention entries ask of tensor views (host only).
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

inline bool known_dtype(int d) { return d >= SGEMM_EMU_F32 && d <= SGEMM_EMU_F16; }
inline int64_t dtype_bytes(int d) { return d == SGEMM_EMU_F32 ? 4 : 2; }

// A contiguous array of `bytes` bytes.
inline Extent array(const void* p, __int128 bytes) {
    Extent e{(uintptr_t)p, (uintptr_t)p, true};
    if (p == nullptr || bytes <= 0) return e;
    if (bytes > (__int128)(UINTPTR_MAX - e.lo)) {
        e.ok = false;
        return e;
    }
    e.hi = e.lo + (uintptr_t)bytes;
    return e;
}

// Strides not negative, every output apart, no output over an input or another one.
inline int check_tensors(std::initializer_list<Tensor> ins, std::initializer_list<Tensor> outs,
                         std::initializer_list<Extent> arrays_in,
                         std::initializer_list<Extent> arrays_out) {
    for (const auto* list : {&ins, &outs})
        for (const Tensor& t : *list) {
            if (negative(t.v)) return SGEMM_EMU_ERR_STRIDE;
            if (t.v.p != nullptr && !span(t).ok) return SGEMM_EMU_ERR_STRIDE;
        }
    if (!all_ok(arrays_in) || !all_ok(arrays_out)) return SGEMM_EMU_ERR_DIM;
    for (const Tensor& o : outs)
        if (o.v.p != nullptr && !apart(o)) return SGEMM_EMU_ERR_STRIDE;
    const auto clear = [&](const Extent& o) {
        for (const Tensor& t : ins)
            if (t.v.p != nullptr && overlap(o, span(t))) return false;
        for (const Extent& e : arrays_in)
            if (overlap(o, e)) return false;
        return true;
    };
    for (const Tensor& o : outs) {
        if (o.v.p == nullptr) continue;
        if (!clear(span(o))) return SGEMM_EMU_ERR_ALIAS;
        for (const Extent& e : arrays_out)
            if (overlap(span(o), e)) return SGEMM_EMU_ERR_ALIAS;
        for (const Tensor* other = outs.begin(); other != &o; ++other)
            if (other->v.p != nullptr && meet(*other, o)) return SGEMM_EMU_ERR_ALIAS;
    }
    const Extent* prev = arrays_out.begin();
    for (const Extent* e = prev; e != arrays_out.end(); ++e) {
        for (const Extent* f = prev; f != e; ++f)
            if (overlap(*e, *f)) return SGEMM_EMU_ERR_ALIAS;
        if (!clear(*e)) return SGEMM_EMU_ERR_ALIAS;
    }
    return SGEMM_EMU_OK;
}

}  // namespace sgemm_emu
