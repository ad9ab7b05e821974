// The gated delta rule over sequences: the chunk form's workspace and launches.
//
// Tokens go in chunks of 64.  With G the running sum of g inside a chunk, E_ts =
// e^{G_t - G_s} for s <= t and S the state before the chunk,
//   A = diag(beta) strict_lower(E . K K^T),   T = (I + A)^-1,
//   U = T diag(beta) (V - diag(e^G) K S),
//   O = scale (diag(e^G) Q S + lower(E . Q K^T) U),
//   S' = e^{G_64} S + K^T diag(e^{G_64 - G}) U.
// T and P = scale lower(E . Q K^T) depend on one chunk only: a first kernel
// makes them for all chunks at once (delta_prep.hip).  A second one walks the
// chunks of every sequence in order, 16 columns of S to a wave
// (delta_chain.hip).
//
// The gradient walks forward the same way, keeping S and U, and then back with
// the gradient D of the state after the chunk,
//   dU = P^T dO + diag(e^{G_64 - G}) K D,   dY = T^T dU,   dV = diag(beta) dY,
//   D before = e^{G_64} D + scale (diag(e^G) Q)^T dO - (diag(e^G) K)^T dV,
// (delta_back.hip), after which every chunk's dQ, dK, dbeta and dg depend on
// that chunk only (delta_gradient.hip).
#pragma once

#include <initializer_list>

#include "mixing.h"

namespace sgemm_emu {

constexpr int kDeltaMaxK = 128;  // largest key size
constexpr int kDeltaChunk = 64;  // tokens of a chunk
constexpr int kDeltaMaxV = 1 << 16;
constexpr int64_t kDeltaMostStride = 1 << 22;  // of tokens, in elements
// Chunks x value heads of one call (one block each, one launch), and sequences x value
// heads x groups of columns: two blocks of a walk take a group, and a launch has less than
// 2^32 threads.
constexpr int64_t kDeltaMostTasks = 1 << 21;
constexpr int kDeltaMostThreads = 768;  // of a walk's block
static_assert(2 * kDeltaMostTasks * kDeltaMostThreads < int64_t{1} << 32, "one launch");

// Columns of the state that a block of a walk takes (delta_chain.hip, delta_back.hip), where
// there are enough blocks for all CUs; with fewer, it may take 16.
struct DeltaColumns {
    int outputs, states, steps, back;
};

inline DeltaColumns delta_columns(int dtype, int k_size) {
    const bool large_f32 = dtype == SGEMM_EMU_F32 && k_size > 64;
    return {large_f32 ? 16 : 32, 32, large_f32 ? 32 : 64, large_f32 ? 16 : 32};
}

// Sequences of up to this many tokens go token by token (delta_step.hip).  Kernel times, 128 x
// 128 in bfloat16: 16 tokens of 16 heads 17.8 us against 16.7 in chunks, which are a launch
// more, and of 1024 heads 97 against 126; 24 tokens 25 against 17, and 143 against 127.
constexpr int kDeltaFewTokens = 16;

inline bool delta_few_tokens(const delta_emu_forward_t& a) {
    return a.cu_seqlens == nullptr && a.tokens <= kDeltaFewTokens;
}

// Chunks that the sequences of a call can have.  Packed sequences: sequence n's
// are numbered from first row / 64 + n, which leaves at most one number
// between two sequences unused.
inline int64_t delta_chunks(int64_t batch, int64_t tokens, bool packed) {
    if (packed) return tokens / kDeltaChunk + batch;
    return batch * ((tokens + kDeltaChunk - 1) / kDeltaChunk);
}

// What the first kernel leaves for one chunk of one value head, in bytes.
// Matrices are fp16 operand fragments of v_mfma_f32_16x16x32_f16 (1 KiB: 16
// bytes a lane) of the six (16-row tile, 32-column step) pairs that a lower (or,
// transposed, upper) triangular 64 x 64 matrix fills, hi fragments before
// lo ones; rows are scaled by powers of two.
struct DeltaRecord {
    enum Factor {   // rows of 64 floats
        kPt,         // inverse row scale of P^T
        kQueryRise,  // scale e^G / query scale
        kT,          // inverse row scales of T diag(beta), P
        kP,
        kRise,   // e^G / key scale, NaN where beta is not finite
        kTail,   // e^{G_64 - G} / key scale
        kDecay,  // [0]: e^{G_64}
        kBeta,   // beta
        kTt,     // inverse row scale of T^T
        kKeyScale,  // 2^a: a key row times it has its largest entry in [2^14, 2^15)
        kQueryScale,
        kFactors
    };
    // what the walks take of them: forward, back, and back's products ahead
    static constexpr int kFirstChain = kQueryRise, kChain = kDecay + 1 - kQueryRise;
    static constexpr int kFirstBack = kRise, kBack = kTt + 1 - kRise;
    static constexpr int kFirstAhead = kPt, kAhead = kQueryRise + 1 - kPt;
    static constexpr int kMatrix = 6 * 1024;             // one part of one matrix
    static constexpr int kFactorBytes = kFactors * 256;  // at the record's start
    static constexpr int kAtSums = kFactorBytes;         // G, 64 doubles
    static constexpr int kAtT = kAtSums + 512;           // two parts
    static constexpr int kAtP = kAtT + 2 * kMatrix;      // two parts
    static constexpr int kForward = kAtP + 2 * kMatrix;
    static constexpr int kAtTt = kAtP;  // the backward form has no P
    static constexpr int kAtPt = kAtTt + 2 * kMatrix;
    static constexpr int kBackward = kAtPt + 2 * kMatrix;
};

// Arguments of the chunk kernels.
struct DeltaChunks {
    int dtype, batch, tokens, k_heads, v_heads, k_size, v_size;
    float scale;
    const int* cu_seqlens;
    sgemm_emu_view_t q, k, v, g, beta, o;
    const float* initial;
    float* final_state;
    char* records;        // of chunk c, value head h: at (c v_heads + h) record_bytes
    int64_t record_bytes;
    int chunks;
    bool backward;        // records of the backward form
    // what the walk over the chunks keeps for the gradient, per chunk and
    // value head: S before the chunk (k_size x v_size) and U (64 x v_size)
    float* states;
    float* updates;
    bool wide;            // 16-byte loads of q's and k's rows
    // gradients: d_o, dfinal and what the walk back keeps per chunk: the
    // gradients of S after it and of diag(beta) (V - ...), the right side of U
    sgemm_emu_view_t d_o, dq, dk, dv, dg, dbeta;
    const float* dfinal;
    float* dinitial;
    float* dstates;
    float* dsides;
    bool wide_values;     // 16-byte loads of v's and d_o's rows
    // Long sequences of few heads are cut into parts of `part_chunks` chunks (0:
    // not cut), which are walked at the same time: a part takes the state S to
    // M S + N.  Per part and value head: N, then the state before the part
    // (k_size x v_size), and M (rows x rows, rows = k_size up to a multiple of 16).
    int part_chunks, parts;
    float* part_states;
    float* part_steps;
    float* part_dstates;  // the same of the walk back
};

// Parts that the sequences of a call can have; numbered as chunks are.
inline int64_t delta_parts(int64_t batch, int64_t tokens, bool packed, int64_t part_chunks) {
    const int64_t chunks = delta_chunks(batch, tokens, packed);
    if (packed) return chunks / part_chunks + batch;
    return batch == 0 ? 0 : batch * ((chunks / batch + part_chunks - 1) / part_chunks);
}

// Whether rows of `size` elements of these views can be loaded 16 bytes at a
// time.
inline bool delta_wide(int dtype, int size, std::initializer_list<sgemm_emu_view_t> views) {
    const int64_t n = dtype == SGEMM_EMU_F32 ? 4 : 8;
    for (const sgemm_emu_view_t& v : views)
        if ((uintptr_t)v.p % 16 || v.batch % n || v.token % n || v.head % n) return false;
    return size % 8 == 0;
}

hipError_t launch_delta_prep(const DeltaChunks& a, hipStream_t stream);
// What a walk writes: the outputs; the state and U of every chunk (or, back,
// the state's gradient and dY); or nothing but N and M of every part.
enum DeltaWalk { kDeltaOutputs, kDeltaStates, kDeltaParts };
hipError_t launch_delta_chain(const DeltaChunks& a, DeltaWalk walk, hipStream_t stream);
hipError_t launch_delta_chain_back(const DeltaChunks& a, DeltaWalk walk, hipStream_t stream);
// The states before every part from the first one's: part_states (back: the
// gradients after every part from the last one's, with M^T: part_dstates).
hipError_t launch_delta_join(const DeltaChunks& a, bool back, hipStream_t stream);
hipError_t launch_delta_gradient(const DeltaChunks& a, hipStream_t stream);

int64_t delta_forward_workspace(const delta_emu_forward_t& a);
hipError_t launch_delta_forward(const delta_emu_forward_t& a, hipStream_t stream);
int64_t delta_backward_workspace(const delta_emu_backward_t& a);
hipError_t launch_delta_backward(const delta_emu_backward_t& a, hipStream_t stream);

}  // namespace sgemm_emu
