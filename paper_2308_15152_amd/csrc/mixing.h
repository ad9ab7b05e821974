// Declarations shared by the token mixing operators: rotary positions and the
// gated delta rule.
#pragma once

#include <stdint.h>

#include <hip/hip_runtime.h>

#include "mixing_emu.h"

namespace sgemm_emu {

// Arguments are validated before these are called.
hipError_t launch_rotary(const rotary_emu_t& a, hipStream_t stream);
hipError_t launch_rotary_table(int rows, int rot, double base, double factor, double original,
                               double low, double high, double amplitude, float* cos_table,
                               float* sin_table, hipStream_t stream);

// One call of the rule's recurrent form.
struct DeltaStep {
    int dtype, batch, tokens, k_heads, v_heads, k_size, v_size;
    float scale;
    sgemm_emu_view_t q, k, v, g, beta, o;
    const float* from;  // states before, or null (zero)
    float* to;          // states after, or null
    int64_t state_stride;
    const int* slots;  // state of each sequence, or null (its own number)
    int n_slots;
};

hipError_t launch_delta_step(const DeltaStep& a, hipStream_t stream);

}  // namespace sgemm_emu
