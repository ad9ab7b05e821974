// The gated delta rule over whole sequences: the chunk form's kernels and
// workspace.
#include "delta.h"

namespace sgemm_emu {

int64_t delta_forward_workspace(const delta_emu_forward_t& a) {
    return delta_chunks(a.batch, a.tokens, a.cu_seqlens != nullptr) * a.v_heads *
           DeltaRecord::kForward;
}

hipError_t launch_delta_forward(const delta_emu_forward_t& a, hipStream_t stream) {
    DeltaChunks c{};
    c.dtype = a.dtype, c.batch = a.batch, c.tokens = a.tokens;
    c.k_heads = a.k_heads, c.v_heads = a.v_heads, c.k_size = a.k_size, c.v_size = a.v_size;
    c.scale = a.scale;
    c.cu_seqlens = a.cu_seqlens;
    c.q = a.q, c.k = a.k, c.v = a.v, c.g = a.g, c.beta = a.beta, c.o = a.o;
    c.initial = a.initial, c.final_state = a.final_state;
    c.records = static_cast<char*>(a.workspace);
    c.record_bytes = DeltaRecord::kForward;
    c.chunks = (int)delta_chunks(a.batch, a.tokens, a.cu_seqlens != nullptr);
    c.wide = delta_wide(a.dtype, a.k_size, {a.q, a.k});
    c.wide_values = delta_wide(a.dtype, a.v_size, {a.v});
    if (hipError_t e = launch_delta_prep(c, stream)) return e;
    return launch_delta_chain(c, stream);
}

namespace {

int64_t rounded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// What the gradient keeps per chunk and value head, in bytes: the record, S and
// its gradient, U and the gradient of its right side.
struct BackwardParts {
    int64_t tasks, records, states, updates;
    int64_t total() const { return records + 2 * states + 2 * updates; }
};

BackwardParts backward_parts(const delta_emu_backward_t& a) {
    BackwardParts b;
    b.tasks = delta_chunks(a.batch, a.tokens, a.cu_seqlens != nullptr) * a.v_heads;
    b.records = b.tasks * DeltaRecord::kBackward;
    b.states = rounded(b.tasks * ((a.k_size + 15) / 16 * 16) * a.v_size * 4);
    b.updates = rounded(b.tasks * kDeltaChunk * a.v_size * 4);
    return b;
}

}  // namespace

int64_t delta_backward_workspace(const delta_emu_backward_t& a) {
    return backward_parts(a).total();
}

hipError_t launch_delta_backward(const delta_emu_backward_t& a, hipStream_t stream) {
    const BackwardParts b = backward_parts(a);
    char* at = static_cast<char*>(a.workspace);
    DeltaChunks c{};
    c.dtype = a.dtype, c.batch = a.batch, c.tokens = a.tokens;
    c.k_heads = a.k_heads, c.v_heads = a.v_heads, c.k_size = a.k_size, c.v_size = a.v_size;
    c.scale = a.scale;
    c.cu_seqlens = a.cu_seqlens;
    c.q = a.q, c.k = a.k, c.v = a.v, c.g = a.g, c.beta = a.beta, c.d_o = a.d_o;
    c.dq = a.dq, c.dk = a.dk, c.dv = a.dv, c.dg = a.dg, c.dbeta = a.dbeta;
    c.initial = a.initial, c.dfinal = a.dfinal, c.dinitial = a.dinitial;
    c.records = at;
    c.record_bytes = DeltaRecord::kBackward;
    c.states = reinterpret_cast<float*>(at + b.records);
    c.dstates = reinterpret_cast<float*>(at + b.records + b.states);
    c.updates = reinterpret_cast<float*>(at + b.records + 2 * b.states);
    c.dsides = reinterpret_cast<float*>(at + b.records + 2 * b.states + b.updates);
    c.chunks = (int)(b.tasks / a.v_heads);
    c.backward = true;
    c.wide = delta_wide(a.dtype, a.k_size, {a.q, a.k});
    c.wide_values = delta_wide(a.dtype, a.v_size, {a.v, a.d_o});
    if (hipError_t e = launch_delta_prep(c, stream)) return e;
    if (c.v_size > 0) {
        if (hipError_t e = launch_delta_chain(c, stream)) return e;
        if (hipError_t e = launch_delta_chain_back(c, stream)) return e;
    }
    return launch_delta_gradient(c, stream);
}

}  // namespace sgemm_emu
