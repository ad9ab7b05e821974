// C entry points of the token mixing operators: argument checks and launches.
// As in capi.hip, every check runs on the host before any HIP call.
#include <stdint.h>

#include <cmath>

#include "checks.h"
#include "delta.h"
#include "mixing.h"
#include "views.h"

namespace {

using namespace sgemm_emu;

bool known_dtype(int d) { return d >= SGEMM_EMU_F32 && d <= SGEMM_EMU_F16; }
int64_t dtype_bytes(int d) { return d == SGEMM_EMU_F32 ? 4 : 2; }

// A contiguous array of `bytes` bytes.
Extent array(const void* p, __int128 bytes) {
    Extent e{(uintptr_t)p, (uintptr_t)p, true};
    if (p == nullptr || bytes <= 0) return e;
    if (bytes > (__int128)(UINTPTR_MAX - e.lo)) {
        e.ok = false;
        return e;
    }
    e.hi = e.lo + (uintptr_t)bytes;
    return e;
}

// Sizes that the delta entries share.
template <class A>
int check_sizes(const A& a) {
    if (!known_dtype(a.dtype)) return SGEMM_EMU_ERR_UNSUPPORTED;
    if (a.batch < 0 || a.tokens < 0 || a.k_heads < 0 || a.v_heads < 0 || a.k_size < 0 ||
        a.v_size < 0)
        return SGEMM_EMU_ERR_DIM;
    if (a.k_size < 1 || a.k_size > kDeltaMaxK || a.k_heads < 1 || a.v_heads < 1 ||
        a.v_heads % a.k_heads != 0 || a.v_size > kDeltaMaxV)
        return SGEMM_EMU_ERR_UNSUPPORTED;
    return SGEMM_EMU_OK;
}

// The chunk kernels address a chunk's 64 rows of a head with 32-bit offsets.
bool within_reach(std::initializer_list<sgemm_emu_view_t> views) {
    for (const sgemm_emu_view_t& v : views)
        if (v.token > kDeltaMostStride) return false;
    return true;
}

// Strides not negative, every output apart, no output over an input or another one.
int check_tensors(std::initializer_list<Tensor> ins, std::initializer_list<Tensor> outs,
                  std::initializer_list<Extent> arrays_in, std::initializer_list<Extent> arrays_out) {
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

// Checks that do not look behind pointers, for the workspace queries and the
// calls alike.  columns: that a block of the call's walks takes, 0 without a walk.
template <class A>
int check_shape(const A& a, int columns) {
    if (int rc = check_sizes(a)) return rc;
    if (a.cu_seqlens == nullptr && (int64_t)a.batch * a.tokens > INT32_MAX)
        return SGEMM_EMU_ERR_UNSUPPORTED;
    if (delta_chunks(a.batch, a.tokens, a.cu_seqlens != nullptr) > kDeltaMostTasks / a.v_heads)
        return SGEMM_EMU_ERR_UNSUPPORTED;
    const int64_t group = columns > 0 ? 2 * columns : 64;
    if ((int64_t)a.batch * ((a.v_size + group - 1) / group) > kDeltaMostTasks / a.v_heads)
        return SGEMM_EMU_ERR_UNSUPPORTED;
    return SGEMM_EMU_OK;
}

int check_shape(const delta_emu_forward_t& a) {
    return check_shape(a, delta_few_tokens(a) ? 0 : delta_columns(a.dtype, a.k_size).outputs);
}
int check_shape(const delta_emu_backward_t& a) {
    // (a block of the walk back that takes 16 columns has half of the threads)
    return check_shape(a, delta_columns(a.dtype, a.k_size).states);
}

int done(hipError_t e) { return e == hipSuccess ? SGEMM_EMU_OK : hip_fail(e); }

}  // namespace

extern "C" {

int rotary_emu(const rotary_emu_t* args, hipStream_t stream) {
    if (args == nullptr) return SGEMM_EMU_ERR_NULL;
    const rotary_emu_t& a = *args;
    if (!known_dtype(a.dtype)) return SGEMM_EMU_ERR_UNSUPPORTED;
    if (a.batch < 0 || a.tokens < 0 || a.size < 0 || a.heads[0] < 0 || a.heads[1] < 0 ||
        a.table_rows < 0 || a.offset < 0)
        return SGEMM_EMU_ERR_DIM;
    if (a.rot < 0 || a.rot > a.size || a.rot % 2 != 0) return SGEMM_EMU_ERR_UNSUPPORTED;
    if (a.positions != nullptr && a.position_bytes != 4 && a.position_bytes != 8)
        return SGEMM_EMU_ERR_UNSUPPORTED;
    if ((int64_t)a.batch * a.tokens > INT32_MAX ||
        ((int64_t)a.heads[0] + a.heads[1]) * a.size > INT32_MAX)
        return SGEMM_EMU_ERR_UNSUPPORTED;
    if (a.batch == 0 || a.tokens == 0 || a.size == 0) return SGEMM_EMU_OK;
    const int64_t elem = dtype_bytes(a.dtype);
    const int heads1 = a.x[1].p == nullptr ? 0 : a.heads[1];
    const int heads[2] = {a.heads[0], heads1};
    for (int i = 0; i < 2; ++i)
        if (heads[i] > 0 && (a.x[i].p == nullptr || a.y[i].p == nullptr)) return SGEMM_EMU_ERR_NULL;
    if (heads[0] + heads[1] == 0) return SGEMM_EMU_OK;
    if (a.rot > 0 && (a.cos_table == nullptr || a.sin_table == nullptr)) return SGEMM_EMU_ERR_NULL;
    if (a.positions != nullptr && (a.position_batch < 0 || a.position_token < 0))
        return SGEMM_EMU_ERR_STRIDE;
    const __int128 table = (__int128)a.table_rows * (a.rot / 2) * 4;
    const sgemm_emu_view_t at{const_cast<void*>(a.positions), a.position_batch, a.position_token, 0};
    const Tensor places{at, a.batch, a.tokens, 1, 1, a.positions ? a.position_bytes : 1};
    const Extent tables[2] = {array(a.cos_table, table), array(a.sin_table, table)};
    // an output may only meet its own input, in place, and not the other output
    for (int i = 0; i < 2; ++i) {
        if (heads[i] == 0) continue;
        const Tensor y{a.y[i], a.batch, a.tokens, heads[i], a.size, elem};
        const Tensor x{a.x[i], a.batch, a.tokens, heads[i], a.size, elem};
        const Tensor other{a.x[1 - i], a.batch, a.tokens, heads[1 - i], a.size, elem};
        const Tensor others{a.y[1 - i], a.batch, a.tokens, heads[1 - i], a.size, elem};
        const bool in_place = same(a.x[i], a.y[i]);
        int rc;
        if (in_place)  // x is y; the other tensor may be interleaved with it, in place as well
            rc = check_tensors({places}, {y}, {tables[0], tables[1]}, {});
        else
            rc = check_tensors({x, places}, {y}, {tables[0], tables[1]}, {});
        if (rc != SGEMM_EMU_OK) return rc;
        if (heads[1 - i] > 0 && !(in_place && same(a.x[1 - i], a.y[1 - i]))) {
            if (negative(other.v) || negative(others.v) || !span(other).ok)
                return SGEMM_EMU_ERR_STRIDE;
            if (overlap(span(y), span(other))) return SGEMM_EMU_ERR_ALIAS;
        }
        if (i == 1 && heads[0] > 0 && meet(others, y)) return SGEMM_EMU_ERR_ALIAS;
    }
    return done(launch_rotary(a, stream));
}

int rotary_emu_table(int rows, int rot, double base, double factor, double original, double low,
                     double high, double amplitude, float* cos_table, float* sin_table,
                     hipStream_t stream) {
    if (rows < 0 || rot < 0 || rot % 2 != 0) return SGEMM_EMU_ERR_DIM;
    for (double x : {base, factor, original, low, high, amplitude})
        if (!std::isfinite(x)) return SGEMM_EMU_ERR_UNSUPPORTED;
    if (base <= 0 || factor <= 0 || low > high) return SGEMM_EMU_ERR_UNSUPPORTED;
    if (rows == 0 || rot == 0) return SGEMM_EMU_OK;
    if (cos_table == nullptr || sin_table == nullptr) return SGEMM_EMU_ERR_NULL;
    const __int128 bytes = (__int128)rows * (rot / 2) * 4;
    const Extent c = array(cos_table, bytes), s = array(sin_table, bytes);
    if (!all_ok({c, s})) return SGEMM_EMU_ERR_DIM;
    if (overlap(c, s)) return SGEMM_EMU_ERR_ALIAS;
    return done(launch_rotary_table(rows, rot, base, factor, original, low, high, amplitude,
                                    cos_table, sin_table, stream));
}

int delta_emu_step(const delta_emu_step_t* args, hipStream_t stream) {
    if (args == nullptr) return SGEMM_EMU_ERR_NULL;
    const delta_emu_step_t& a = *args;
    if (int rc = check_sizes(a)) return rc;
    if (a.n_slots < 0 || (a.slots == nullptr && a.batch > a.n_slots)) return SGEMM_EMU_ERR_DIM;
    const __int128 each = (__int128)a.v_heads * a.k_size * a.v_size;
    if (a.state_stride < 0 || (a.n_slots > 1 && a.state_stride < each)) return SGEMM_EMU_ERR_STRIDE;
    if (a.batch == 0 || a.tokens == 0 || a.v_size == 0) return SGEMM_EMU_OK;
    if (!a.q.p || !a.k.p || !a.v.p || !a.o.p) return SGEMM_EMU_ERR_NULL;
    if (a.state == nullptr && a.n_slots > 0) return SGEMM_EMU_ERR_NULL;
    const int64_t e = dtype_bytes(a.dtype);
    const Tensor q{a.q, a.batch, a.tokens, a.k_heads, a.k_size, e};
    const Tensor k{a.k, a.batch, a.tokens, a.k_heads, a.k_size, e};
    const Tensor v{a.v, a.batch, a.tokens, a.v_heads, a.v_size, e};
    const Tensor g{a.g, a.batch, a.tokens, a.v_heads, 1, 4};
    const Tensor beta{a.beta, a.batch, a.tokens, a.v_heads, 1, 4};
    const Tensor o{a.o, a.batch, a.tokens, a.v_heads, a.v_size, e};
    const __int128 pool =
        a.n_slots == 0 ? 0 : ((__int128)(a.n_slots - 1) * a.state_stride + each) * 4;
    const Extent state = array(a.state, pool);
    const Extent slots = array(a.slots, (__int128)a.batch * 4);
    if (int rc = check_tensors({q, k, v, g, beta}, {o}, {slots}, {state})) return rc;
    DeltaStep s{};
    s.dtype = a.dtype, s.batch = a.batch, s.tokens = a.tokens;
    s.k_heads = a.k_heads, s.v_heads = a.v_heads, s.k_size = a.k_size, s.v_size = a.v_size;
    s.scale = a.scale;
    s.q = a.q, s.k = a.k, s.v = a.v, s.g = a.g, s.beta = a.beta, s.o = a.o;
    s.from = a.state, s.to = a.state, s.state_stride = a.state_stride;
    s.slots = a.slots, s.n_slots = a.n_slots;
    return done(launch_delta_step(s, stream));
}

int64_t delta_emu_forward_workspace(const delta_emu_forward_t* a) {
    if (a == nullptr) return SGEMM_EMU_ERR_NULL;
    if (int rc = check_shape(*a)) return rc;
    return delta_forward_workspace(*a);
}

int delta_emu_forward(const delta_emu_forward_t* args, hipStream_t stream) {
    if (args == nullptr) return SGEMM_EMU_ERR_NULL;
    const delta_emu_forward_t& a = *args;
    if (int rc = check_shape(a)) return rc;
    if (!within_reach({a.q, a.k, a.v, a.o})) return SGEMM_EMU_ERR_UNSUPPORTED;
    if (a.batch == 0 || a.v_size == 0) return SGEMM_EMU_OK;
    const bool packed = a.cu_seqlens != nullptr;
    const int64_t batch = packed ? 1 : a.batch, e = dtype_bytes(a.dtype);
    if (a.tokens > 0 && (!a.q.p || !a.k.p || !a.v.p || !a.o.p)) return SGEMM_EMU_ERR_NULL;
    const Tensor q{a.q, batch, a.tokens, a.k_heads, a.k_size, e};
    const Tensor k{a.k, batch, a.tokens, a.k_heads, a.k_size, e};
    const Tensor v{a.v, batch, a.tokens, a.v_heads, a.v_size, e};
    const Tensor g{a.g, batch, a.tokens, a.v_heads, 1, 4};
    const Tensor beta{a.beta, batch, a.tokens, a.v_heads, 1, 4};
    const Tensor o{a.o, batch, a.tokens, a.v_heads, a.v_size, e};
    const __int128 states = (__int128)a.batch * a.v_heads * a.k_size * a.v_size * 4;
    const int64_t need = delta_forward_workspace(a);
    if (need > 0 && a.workspace == nullptr) return SGEMM_EMU_ERR_NULL;
    if (need > 0 && (a.workspace_bytes < need || (uintptr_t)a.workspace % 256 != 0))
        return SGEMM_EMU_ERR_DIM;
    const Extent first = array(a.initial == a.final_state ? nullptr : a.initial, states);
    if (int rc = check_tensors({q, k, v, g, beta}, {o},
                               {first, array(a.cu_seqlens, ((__int128)a.batch + 1) * 4)},
                               {array(a.final_state, states), array(a.workspace, need)}))
        return rc;
    return done(launch_delta_forward(a, stream));
}

int64_t delta_emu_backward_workspace(const delta_emu_backward_t* a) {
    if (a == nullptr) return SGEMM_EMU_ERR_NULL;
    if (int rc = check_shape(*a)) return rc;
    return delta_backward_workspace(*a);
}

int delta_emu_backward(const delta_emu_backward_t* args, hipStream_t stream) {
    if (args == nullptr) return SGEMM_EMU_ERR_NULL;
    const delta_emu_backward_t& a = *args;
    if (int rc = check_shape(a)) return rc;
    if (!within_reach({a.q, a.k, a.v, a.d_o, a.dq, a.dk, a.dv}))
        return SGEMM_EMU_ERR_UNSUPPORTED;
    if (a.batch == 0) return SGEMM_EMU_OK;
    const bool packed = a.cu_seqlens != nullptr;
    const int64_t batch = packed ? 1 : a.batch, e = dtype_bytes(a.dtype);
    if (a.tokens > 0 && (!a.q.p || !a.k.p || !a.dq.p || !a.dk.p)) return SGEMM_EMU_ERR_NULL;
    if (a.tokens > 0 && a.v_size > 0 && (!a.v.p || !a.d_o.p || !a.dv.p)) return SGEMM_EMU_ERR_NULL;
    const Tensor q{a.q, batch, a.tokens, a.k_heads, a.k_size, e};
    const Tensor k{a.k, batch, a.tokens, a.k_heads, a.k_size, e};
    const Tensor v{a.v, batch, a.tokens, a.v_heads, a.v_size, e};
    const Tensor g{a.g, batch, a.tokens, a.v_heads, 1, 4};
    const Tensor beta{a.beta, batch, a.tokens, a.v_heads, 1, 4};
    const Tensor d_o{a.d_o, batch, a.tokens, a.v_heads, a.v_size, e};
    const Tensor dq{a.dq, batch, a.tokens, a.k_heads, a.k_size, e};
    const Tensor dk{a.dk, batch, a.tokens, a.k_heads, a.k_size, e};
    const Tensor dv{a.dv, batch, a.tokens, a.v_heads, a.v_size, e};
    const Tensor dg{a.dg, batch, a.tokens, a.v_heads, 1, 4};
    const Tensor dbeta{a.dbeta, batch, a.tokens, a.v_heads, 1, 4};
    const __int128 states = (__int128)a.batch * a.v_heads * a.k_size * a.v_size * 4;
    const int64_t need = delta_backward_workspace(a);
    if (need > 0 && a.workspace == nullptr) return SGEMM_EMU_ERR_NULL;
    if (need > 0 && (a.workspace_bytes < need || (uintptr_t)a.workspace % 256 != 0))
        return SGEMM_EMU_ERR_DIM;
    const Extent last = array(a.dfinal == a.dinitial ? nullptr : a.dfinal, states);
    if (int rc = check_tensors({q, k, v, g, beta, d_o}, {dq, dk, dv, dg, dbeta},
                               {array(a.initial, states), last,
                                array(a.cu_seqlens, ((__int128)a.batch + 1) * 4)},
                               {array(a.dinitial, states), array(a.workspace, need)}))
        return rc;
    return done(launch_delta_backward(a, stream));
}

}  // extern "C"
