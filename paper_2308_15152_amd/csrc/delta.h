// The gated delta rule over sequences: sizes, workspaces and launches.
#pragma once

#include "mixing.h"

namespace sgemm_emu {

constexpr int kDeltaMaxK = 128;  // largest key size
constexpr int kDeltaChunk = 64;  // tokens of a chunk
// Chunks x value heads of one call: one block each, one launch.
constexpr int64_t kDeltaMostTasks = 1 << 22;

// Chunks that the sequences of a call can have.  Sequence n's chunks are
// numbered from chunk_base(n); packed sequences leave at most one number
// between them unused.
inline int64_t delta_chunks(int64_t batch, int64_t tokens, bool packed) {
    if (packed) return tokens / kDeltaChunk + batch;
    return batch * ((tokens + kDeltaChunk - 1) / kDeltaChunk);
}

int64_t delta_forward_workspace(const delta_emu_forward_t& a);
hipError_t launch_delta_forward(const delta_emu_forward_t& a, hipStream_t stream);

}  // namespace sgemm_emu
