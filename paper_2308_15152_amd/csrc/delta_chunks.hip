// The gated delta rule over whole sequences: workspaces and the order of the
// chunk form's kernels.
#include "delta.h"

namespace sgemm_emu {

namespace {

int64_t rounded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// Chunks of a part that the sequences are cut into, 0 if they are not.  A walk
// takes about the same time per chunk whatever the number of its blocks up to one per CU,
// and the parts cost a walk more, over k_size more columns, and the join.  The estimate
// below uses measured times (us, 128 x 128 states in bfloat16; for other types and sizes
// it takes them as they are, which was checked at the last case below only): a chunk takes
// 2.3 (few blocks) to 3.3 (on all CUs) in the walk for outputs, 2.3 to 2.6 for states, 2.8
// for N and M, 3.3 to 4.4 back; a part 3 in the join, and each of these launches 5.  Walks and
// joins: 32768 tokens of 8 heads 403 in 8 parts, 1163 not cut; 4096 tokens of 64 heads 329 in
// two, 204 not cut; their gradient with 32 heads 438 in two, 361 not cut; that of 1001
// tokens of 18 heads of 64 x 96 in float32 111 in three, 88 not cut.
template <class A>
int part_chunks_of(const A& a, bool backward) {
    if (a.batch == 0 || a.tokens == 0 || a.v_size == 0) return 0;
    constexpr double kCus = 256, kOutputs = 2.7, kStates = 2.4, kSteps = 2.8, kBack = 3.8,
                     kJoin = 3.0, kStart = 5.0;
    const DeltaColumns c = delta_columns(a.dtype, a.k_size);
    const auto blocks = [&](int64_t columns, int each) {  // of all sequences and heads
        return (double)((columns + each - 1) / each) * a.v_heads * a.batch;
    };
    const auto rounds = [&](double n) {
        return n <= kCus ? 1.0 : (double)((int64_t)((n + kCus - 1) / kCus));
    };
    // chunks of a sequence; of packed ones, whose lengths are not known here, the mean
    const int64_t chunks = a.cu_seqlens ? (a.tokens / kDeltaChunk + a.batch) / a.batch
                                        : (a.tokens + kDeltaChunk - 1) / kDeltaChunk;
    const double steps = blocks(a.v_size, c.steps) + blocks(a.k_size, c.steps);
    double best = 0;
    int64_t chosen = 0;
    for (int64_t parts = 1; parts <= 64 && parts <= chunks; ++parts) {
        const int64_t m = (chunks + parts - 1) / parts;
        const double p = (double)((chunks + m - 1) / m);
        double launches = backward ? 2 : 1;  // of walks and joins
        double walk = backward ? rounds(p * blocks(a.v_size, c.states)) * kStates +
                                     rounds(p * blocks(a.v_size, c.back)) * kBack
                               : rounds(p * blocks(a.v_size, c.outputs)) * kOutputs;
        double time = 0;
        if (parts > 1) {
            walk += rounds((backward ? p : p - 1) * steps) * kSteps;
            if (backward) walk += rounds((p - 1) * blocks(a.v_size, c.back)) * kBack;
            time = (backward ? 2 : 1) * kJoin * p;
            launches *= 3;
        }
        time += walk * m + kStart * launches;
        if (parts == 1) {
            best = 0.9 * time;  // worth the trouble
        } else if (time < best) {
            best = time;
            chosen = m;
        }
    }
    return (int)chosen;
}

// Byte offsets in the workspace.
struct Plan {
    bool packed;
    int chunks, part_chunks, parts;
    int64_t record_bytes, states, dstates, updates, dsides, part_states, part_dstates, part_steps,
        total;
};

template <class A>
Plan plan_of(const A& a, bool backward) {
    Plan p{};
    p.packed = a.cu_seqlens != nullptr;
    p.chunks = (int)delta_chunks(a.batch, a.tokens, p.packed);
    p.part_chunks = part_chunks_of(a, backward);
    if (p.part_chunks > 0)
        p.parts = (int)delta_parts(a.batch, a.tokens, p.packed, p.part_chunks);
    p.record_bytes = backward ? DeltaRecord::kBackward : DeltaRecord::kForward;
    const int64_t tasks = (int64_t)p.chunks * a.v_heads, walks = (int64_t)p.parts * a.v_heads;
    const int64_t rows = (a.k_size + 15) / 16 * 16;
    const auto take = [&](int64_t bytes) {
        const int64_t at = p.total;
        p.total += rounded(bytes);
        return at;
    };
    take(tasks * p.record_bytes);
    if (backward) {
        p.states = take(tasks * rows * a.v_size * 4);
        p.dstates = take(tasks * rows * a.v_size * 4);
        p.updates = take(tasks * kDeltaChunk * a.v_size * 4);
        p.dsides = take(tasks * kDeltaChunk * a.v_size * 4);
    }
    if (p.parts > 0) {
        p.part_states = take(walks * a.k_size * a.v_size * 4);
        p.part_steps = take(walks * rows * rows * 4);
        if (backward) p.part_dstates = take(walks * a.k_size * a.v_size * 4);
    }
    return p;
}

template <class A>
DeltaChunks arguments(const A& a, const Plan& p) {
    char* at = static_cast<char*>(a.workspace);
    DeltaChunks c{};
    c.dtype = a.dtype, c.batch = a.batch, c.tokens = a.tokens;
    c.k_heads = a.k_heads, c.v_heads = a.v_heads, c.k_size = a.k_size, c.v_size = a.v_size;
    c.scale = a.scale;
    c.cu_seqlens = a.cu_seqlens;
    c.q = a.q, c.k = a.k, c.v = a.v, c.g = a.g, c.beta = a.beta;
    c.initial = a.initial;
    c.records = at;
    c.record_bytes = p.record_bytes;
    c.chunks = p.chunks;
    c.part_chunks = p.part_chunks, c.parts = p.parts;
    c.part_states = reinterpret_cast<float*>(at + p.part_states);
    c.part_steps = reinterpret_cast<float*>(at + p.part_steps);
    c.wide = delta_wide(a.dtype, a.k_size, {a.q, a.k});
    return c;
}

}  // namespace

int64_t delta_forward_workspace(const delta_emu_forward_t& a) {
    return delta_few_tokens(a) ? 0 : plan_of(a, false).total;
}

int64_t delta_backward_workspace(const delta_emu_backward_t& a) { return plan_of(a, true).total; }

hipError_t launch_delta_forward(const delta_emu_forward_t& a, hipStream_t stream) {
    if (delta_few_tokens(a)) {
        DeltaStep s{};
        s.dtype = a.dtype, s.batch = a.batch, s.tokens = a.tokens;
        s.k_heads = a.k_heads, s.v_heads = a.v_heads, s.k_size = a.k_size, s.v_size = a.v_size;
        s.scale = a.scale;
        s.q = a.q, s.k = a.k, s.v = a.v, s.g = a.g, s.beta = a.beta, s.o = a.o;
        s.from = a.initial, s.to = a.final_state;
        s.state_stride = (int64_t)a.v_heads * a.k_size * a.v_size;
        s.n_slots = a.batch;
        return launch_delta_step(s, stream);
    }
    const Plan p = plan_of(a, false);
    DeltaChunks c = arguments(a, p);
    c.o = a.o;
    c.final_state = a.final_state;
    c.wide_values = delta_wide(a.dtype, a.v_size, {a.v});
    hipError_t e = launch_delta_prep(c, stream);
    if (e == hipSuccess && p.parts > 0) {
        e = launch_delta_chain(c, kDeltaParts, stream);
        if (e == hipSuccess) e = launch_delta_join(c, false, stream);
    }
    if (e == hipSuccess) e = launch_delta_chain(c, kDeltaOutputs, stream);
    return e;
}

hipError_t launch_delta_backward(const delta_emu_backward_t& a, hipStream_t stream) {
    const Plan p = plan_of(a, true);
    char* at = static_cast<char*>(a.workspace);
    DeltaChunks c = arguments(a, p);
    c.d_o = a.d_o;
    c.dq = a.dq, c.dk = a.dk, c.dv = a.dv, c.dg = a.dg, c.dbeta = a.dbeta;
    c.dfinal = a.dfinal, c.dinitial = a.dinitial;
    c.states = reinterpret_cast<float*>(at + p.states);
    c.dstates = reinterpret_cast<float*>(at + p.dstates);
    c.updates = reinterpret_cast<float*>(at + p.updates);
    c.dsides = reinterpret_cast<float*>(at + p.dsides);
    c.part_dstates = reinterpret_cast<float*>(at + p.part_dstates);
    c.backward = true;
    c.wide_values = delta_wide(a.dtype, a.v_size, {a.v, a.d_o});
    hipError_t e = launch_delta_prep(c, stream);
    const auto then = [&](auto&& launch) {
        if (e == hipSuccess) e = launch();
    };
    if (a.v_size > 0) {
        if (p.parts > 0) {
            then([&] { return launch_delta_chain(c, kDeltaParts, stream); });
            then([&] { return launch_delta_join(c, false, stream); });
        }
        then([&] { return launch_delta_chain(c, kDeltaStates, stream); });
        if (p.parts > 0) {
            then([&] { return launch_delta_chain_back(c, kDeltaParts, stream); });
            then([&] { return launch_delta_join(c, true, stream); });
        }
        then([&] { return launch_delta_chain_back(c, kDeltaStates, stream); });
    }
    then([&] { return launch_delta_gradient(c, stream); });
    return e;
}

}  // namespace sgemm_emu
