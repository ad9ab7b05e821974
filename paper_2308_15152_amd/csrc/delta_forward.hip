// The gated delta rule over whole sequences.
#include "delta.h"
#include "mixing.hpp"

namespace sgemm_emu {

int64_t delta_forward_workspace(const delta_emu_forward_t&) { return 0; }

hipError_t launch_delta_forward(const delta_emu_forward_t& a, hipStream_t stream) {
    DeltaStep s{};
    s.dtype = a.dtype, s.batch = a.batch, s.tokens = a.tokens;
    s.k_heads = a.k_heads, s.v_heads = a.v_heads, s.k_size = a.k_size, s.v_size = a.v_size;
    s.scale = a.scale;
    s.cu_seqlens = a.cu_seqlens;
    s.q = a.q, s.k = a.k, s.v = a.v, s.g = a.g, s.beta = a.beta, s.o = a.o;
    s.from = a.initial, s.to = a.final_state;
    s.state_stride = (int64_t)a.v_heads * a.k_size * a.v_size;
    s.n_slots = a.batch;
    return launch_delta_step(s, stream);
}

}  // namespace sgemm_emu
