// Declarations shared by the attention kernels.
#pragma once

#include <stdint.h>

#include <hip/hip_runtime.h>

#include "attention_emu.h"

namespace sgemm_emu {

constexpr int kAttentionMostSize = 128;
// Token strides up to this: the kernels address a tile's rows with 32-bit offsets.
constexpr int64_t kAttentionMostStride = 1 << 22;

// Bytes of workspace; arguments are validated before these are called.
int64_t attention_forward_workspace(const attention_emu_forward_t& a);
int64_t attention_backward_workspace(const attention_emu_backward_t& a);
int64_t attention_step_workspace(const attention_emu_step_t& a);

hipError_t launch_attention_forward(const attention_emu_forward_t& a, hipStream_t stream);
hipError_t launch_attention_backward(const attention_emu_backward_t& a, hipStream_t stream);
hipError_t launch_attention_step(const attention_emu_step_t& a, hipStream_t stream);

}  // namespace sgemm_emu
