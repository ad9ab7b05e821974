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
    c.wide = delta_wide(a);
    if (hipError_t e = launch_delta_prep(c, stream)) return e;
    return launch_delta_chain(c, stream);
}

}  // namespace sgemm_emu
