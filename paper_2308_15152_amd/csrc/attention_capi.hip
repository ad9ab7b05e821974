// C entry points of the attention operators: argument checks and launches.  As
// in capi.hip, every check runs on the host before any HIP call.
#include <stdint.h>

#include <cmath>

#include "attention.h"
#include "checks.h"
#include "views.h"

namespace {

using namespace sgemm_emu;

int done(hipError_t e) { return e == hipSuccess ? SGEMM_EMU_OK : hip_fail(e); }

bool within_reach(std::initializer_list<sgemm_emu_view_t> views) {
    for (const sgemm_emu_view_t& v : views)
        if (v.token > kAttentionMostStride) return false;
    return true;
}

int check_heads(int q_heads, int k_heads, int size, float scale) {
    if (q_heads < 0 || k_heads < 0 || size < 0) return SGEMM_EMU_ERR_DIM;
    if (q_heads < 1 || k_heads < 1 || q_heads % k_heads != 0 || size < 1 ||
        size > kAttentionMostSize || !std::isfinite(scale) || scale == 0.0f)
        return SGEMM_EMU_ERR_UNSUPPORTED;
    return SGEMM_EMU_OK;
}

// Checks that do not look at pointers but for being NULL, for the query and the calls.
template <class A>
int check_sequences(const A& a) {
    if (!known_dtype(a.dtype)) return SGEMM_EMU_ERR_UNSUPPORTED;
    if (a.batch < 0 || a.tokens < 0 || a.keys < 0) return SGEMM_EMU_ERR_DIM;
    if (int rc = check_heads(a.q_heads, a.k_heads, a.size, a.scale)) return rc;
    if (a.cu_seqlens == nullptr && a.cu_keys != nullptr) return SGEMM_EMU_ERR_NULL;
    if (a.cu_seqlens != nullptr && a.cu_keys == nullptr && a.keys != a.tokens)
        return SGEMM_EMU_ERR_DIM;
    // rows of the FP16 planes of FP32 tensors (2 x 64 or 128 elements for each head) are as near
    // to each other as those of tensors have to be
    if (a.dtype == SGEMM_EMU_F32 && a.q_heads > kAttentionMostStride / 256)
        return SGEMM_EMU_ERR_UNSUPPORTED;
    // rows and blocks of at least 32 rows or keys are counted in 32 bits
    const int64_t sequences = a.cu_seqlens != nullptr ? 1 : a.batch;
    if ((int64_t)a.tokens * a.q_heads > INT32_MAX - 4096 || a.keys > INT32_MAX - 4096 ||
        (__int128)a.tokens * a.q_heads / 32 * sequences + (int64_t)a.batch * a.k_heads >
            INT32_MAX / 2 ||
        ((int64_t)a.keys / 32 * sequences + a.batch) * (__int128)a.k_heads > INT32_MAX / 2)
        return SGEMM_EMU_ERR_UNSUPPORTED;
    return SGEMM_EMU_OK;
}

int check_step(const attention_emu_step_t& a) {
    if (!known_dtype(a.dtype)) return SGEMM_EMU_ERR_UNSUPPORTED;
    if (a.batch < 0 || a.tokens < 0 || a.prefix < 0 || a.capacity < 0 || a.n_slots < 0 ||
        (a.slots == nullptr && a.batch > a.n_slots))
        return SGEMM_EMU_ERR_DIM;
    if (int rc = check_heads(a.q_heads, a.k_heads, a.size, a.scale)) return rc;
    if ((__int128)a.batch * a.tokens * a.q_heads > INT32_MAX / 2 || a.prefix > INT32_MAX - 4096 ||
        a.capacity > INT32_MAX - 4096)
        return SGEMM_EMU_ERR_UNSUPPORTED;
    return SGEMM_EMU_OK;
}

int check_workspace(int64_t need, const void* p, int64_t bytes) {
    if (need == 0) return SGEMM_EMU_OK;
    if (p == nullptr) return SGEMM_EMU_ERR_NULL;
    return bytes < need || (uintptr_t)p % 256 != 0 ? SGEMM_EMU_ERR_DIM : SGEMM_EMU_OK;
}

}  // namespace

extern "C" {

int64_t attention_emu_forward_workspace(const attention_emu_forward_t* a) {
    if (a == nullptr) return SGEMM_EMU_ERR_NULL;
    if (int rc = check_sequences(*a)) return rc;
    return attention_forward_workspace(*a);
}

int attention_emu_forward(const attention_emu_forward_t* args, hipStream_t stream) {
    if (args == nullptr) return SGEMM_EMU_ERR_NULL;
    const attention_emu_forward_t& a = *args;
    if (int rc = check_sequences(a)) return rc;
    if (!within_reach({a.q, a.k, a.v, a.o})) return SGEMM_EMU_ERR_UNSUPPORTED;
    if (a.batch == 0 || a.tokens == 0) return SGEMM_EMU_OK;
    if (!a.q.p || !a.o.p || (a.keys > 0 && (!a.k.p || !a.v.p))) return SGEMM_EMU_ERR_NULL;
    const bool packed = a.cu_seqlens != nullptr;
    const int64_t batch = packed ? 1 : a.batch, e = dtype_bytes(a.dtype);
    const Tensor q{a.q, batch, a.tokens, a.q_heads, a.size, e};
    const Tensor k{a.k, batch, a.keys, a.k_heads, a.size, e};
    const Tensor v{a.v, batch, a.keys, a.k_heads, a.size, e};
    const Tensor o{a.o, batch, a.tokens, a.q_heads, a.size, e};
    const Tensor lse{a.lse, batch, a.tokens, a.q_heads, 1, 4};
    const int64_t need = attention_forward_workspace(a);
    if (int rc = check_workspace(need, a.workspace, a.workspace_bytes)) return rc;
    const __int128 bounds = ((__int128)a.batch + 1) * 4;
    if (int rc = check_tensors({q, k, v}, {o, lse},
                               {array(a.cu_seqlens, bounds), array(a.cu_keys, bounds)},
                               {array(a.workspace, need)}))
        return rc;
    return done(launch_attention_forward(a, stream));
}

int64_t attention_emu_backward_workspace(const attention_emu_backward_t* a) {
    if (a == nullptr) return SGEMM_EMU_ERR_NULL;
    if (int rc = check_sequences(*a)) return rc;
    return attention_backward_workspace(*a);
}

int attention_emu_backward(const attention_emu_backward_t* args, hipStream_t stream) {
    if (args == nullptr) return SGEMM_EMU_ERR_NULL;
    const attention_emu_backward_t& a = *args;
    if (int rc = check_sequences(a)) return rc;
    if (!within_reach({a.q, a.k, a.v, a.o, a.d_o, a.dq, a.dk, a.dv}))
        return SGEMM_EMU_ERR_UNSUPPORTED;
    if (a.batch == 0) return SGEMM_EMU_OK;
    if (a.tokens > 0 && (!a.q.p || !a.o.p || !a.lse.p || !a.d_o.p || !a.dq.p))
        return SGEMM_EMU_ERR_NULL;
    if (a.keys > 0 && (!a.k.p || !a.v.p || !a.dk.p || !a.dv.p)) return SGEMM_EMU_ERR_NULL;
    const bool packed = a.cu_seqlens != nullptr;
    const int64_t batch = packed ? 1 : a.batch, e = dtype_bytes(a.dtype);
    const Tensor q{a.q, batch, a.tokens, a.q_heads, a.size, e};
    const Tensor k{a.k, batch, a.keys, a.k_heads, a.size, e};
    const Tensor v{a.v, batch, a.keys, a.k_heads, a.size, e};
    const Tensor o{a.o, batch, a.tokens, a.q_heads, a.size, e};
    const Tensor lse{a.lse, batch, a.tokens, a.q_heads, 1, 4};
    const Tensor d_o{a.d_o, batch, a.tokens, a.q_heads, a.size, e};
    const Tensor dq{a.dq, batch, a.tokens, a.q_heads, a.size, e};
    const Tensor dk{a.dk, batch, a.keys, a.k_heads, a.size, e};
    const Tensor dv{a.dv, batch, a.keys, a.k_heads, a.size, e};
    const int64_t need = attention_backward_workspace(a);
    if (int rc = check_workspace(need, a.workspace, a.workspace_bytes)) return rc;
    const __int128 bounds = ((__int128)a.batch + 1) * 4;
    if (int rc = check_tensors({q, k, v, o, lse, d_o}, {dq, dk, dv},
                               {array(a.cu_seqlens, bounds), array(a.cu_keys, bounds)},
                               {array(a.workspace, need)}))
        return rc;
    return done(launch_attention_backward(a, stream));
}

int64_t attention_emu_step_workspace(const attention_emu_step_t* a) {
    if (a == nullptr) return SGEMM_EMU_ERR_NULL;
    if (int rc = check_step(*a)) return rc;
    return attention_step_workspace(*a);
}

int attention_emu_step(const attention_emu_step_t* args, hipStream_t stream) {
    if (args == nullptr) return SGEMM_EMU_ERR_NULL;
    const attention_emu_step_t& a = *args;
    if (int rc = check_step(a)) return rc;
    if (!within_reach({a.q, a.prefix_k, a.prefix_v, a.k, a.v, a.o}))
        return SGEMM_EMU_ERR_UNSUPPORTED;
    if (a.batch == 0 || a.tokens == 0) return SGEMM_EMU_OK;
    if (!a.q.p || !a.o.p || !a.lengths || (a.prefix > 0 && (!a.prefix_k.p || !a.prefix_v.p)) ||
        (a.n_slots > 0 && a.capacity > 0 && (!a.k.p || !a.v.p)))
        return SGEMM_EMU_ERR_NULL;
    const int64_t e = dtype_bytes(a.dtype);
    const Tensor q{a.q, a.batch, a.tokens, a.q_heads, a.size, e};
    const Tensor pk{a.prefix_k, 1, a.prefix, a.k_heads, a.size, e};
    const Tensor pv{a.prefix_v, 1, a.prefix, a.k_heads, a.size, e};
    const Tensor k{a.k, a.n_slots, a.capacity, a.k_heads, a.size, e};
    const Tensor v{a.v, a.n_slots, a.capacity, a.k_heads, a.size, e};
    const Tensor o{a.o, a.batch, a.tokens, a.q_heads, a.size, e};
    const int64_t need = attention_step_workspace(a);
    if (int rc = check_workspace(need, a.workspace, a.workspace_bytes)) return rc;
    if (int rc = check_tensors(
            {q, pk, pv, k, v}, {o},
            {array(a.lengths, (__int128)a.batch * 4), array(a.slots, (__int128)a.batch * 4)},
            {array(a.workspace, need)}))
        return rc;
    return done(launch_attention_step(a, stream));
}

}  // extern "C"
