// FP32 rows as two FP16 planes and a power of two.  Bound by memory: 4 bytes an element are
// read and 4 written (the row's padding, too): 9.4 us for the four inputs of a gradient of
// 3 x 1001 tokens with 6 heads and 1234 keys with 2, of 80.  The products that they are for take a
// third of FP16's rate instead of an eighth: that gradient 175 us for 910 with FP32 products.
#include "attention_split.h"

#include "attention_rows.hpp"
#include "attention_tile.hpp"

namespace sgemm_emu {

namespace {

constexpr int kThreads = 256;

struct SplitArgs {
    Splitter::Job jobs[4];
    int first[5];  // blocks of the jobs before
    int size;
};

// kLanes lanes to a row, 8 elements each.
template <int kLanes, bool kVec>
__global__ __launch_bounds__(kThreads) void attention_split_kernel(SplitArgs a, int first_block) {
    const int block = first_block + (int)blockIdx.x;
    int i = 0;
    while (block >= a.first[i + 1]) ++i;
    const Splitter::Job& job = a.jobs[i];
    const int64_t row = (int64_t)(block - a.first[i]) * (kThreads / kLanes) + threadIdx.x / kLanes;
    const bool there = row < job.rows;
    const int c = threadIdx.x % kLanes;
    const int64_t token = there ? row / job.heads : 0;
    const int head = there ? (int)(row - token * job.heads) : 0;
    const int64_t n = token / job.tokens, t = token - n * job.tokens;
    const float* x = static_cast<const float*>(job.x.p) + n * job.x.batch + t * job.x.token +
                     head * job.x.head;
    float v[8];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const Frag<float> y = load_chunk<float, kVec>(x, 2 * c + j, a.size, there);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * j + e] = y[e];
    }
    // the exponent of the largest finite element
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t bits = __float_as_uint(v[j]) & 0x7fffffff;
        if (bits < 0x7f800000) most = max(most, bits);
    }
#pragma unroll
    for (int d = 1; d < kLanes; d *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, d));
    const int e = max((int)(most >> 23), 15);  // (2^-112 and below: no larger factor)
    const float by = __uint_as_float((uint32_t)(268 - e) << 23);
    Frag<f16_t> hi, lo;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float y = v[j] * by;
        hi[j] = from_f32<f16_t>(y);
        const float rest = y - to_f32(hi[j]);
        // (what is not finite is so in hi)
        lo[j] = from_f32<f16_t>(__builtin_fabsf(y) < __builtin_inff() ? rest : 0.0f);
    }
    if (!there) return;
    f16_t* to = static_cast<f16_t*>(job.to.planes.p) + row * (2 * 8 * kLanes) + 8 * c;
    *reinterpret_cast<Frag<f16_t>*>(to) = hi;
    *reinterpret_cast<Frag<f16_t>*>(to + 8 * kLanes) = lo;
    if (c == 0) job.to.factors[row] = __uint_as_float((uint32_t)(e - 14) << 23);
}

int64_t plane_bytes(int64_t rows, int size) { return rows * 2 * plane_width(size) * 2; }

}  // namespace

int64_t split_bytes(int64_t tokens, int heads, int size) {
    const int64_t rows = tokens * heads;
    return (plane_bytes(rows, size) + rows * 4 + 255) / 256 * 256;
}

SplitTensor Splitter::add(const sgemm_emu_view_t& x, int batch, int tokens, int heads) {
    const int64_t rows = (int64_t)batch * tokens * heads, width = 2 * plane_width(size_);
    SplitTensor s{{at_, tokens * heads * width, heads * width, width},
                  reinterpret_cast<float*>(at_ + plane_bytes(rows, size_))};
    jobs_[count_++] = {x, s, tokens, heads, rows};
    at_ += split_bytes((int64_t)batch * tokens, heads, size_);
    return s;
}

hipError_t Splitter::launch(hipStream_t stream) const {
    SplitArgs a{};
    a.size = size_;
    const int lanes = plane_width(size_) / 8;
    bool vec = size_ % 4 == 0;
    int64_t blocks = 0;
    for (int i = 0; i < 4; ++i) {
        a.first[i] = (int)blocks;
        if (i < count_) {
            a.jobs[i] = jobs_[i];
            blocks += (jobs_[i].rows * lanes + kThreads - 1) / kThreads;
            vec = vec && rows_aligned16(jobs_[i].x, 4);
        }
        a.first[i + 1] = (int)blocks;
    }
    const auto go = [&](auto kernel) { return launch_blocks(kernel, blocks, kThreads, stream, a); };
    if (lanes == 8)
        return vec ? go(attention_split_kernel<8, true>) : go(attention_split_kernel<8, false>);
    return vec ? go(attention_split_kernel<16, true>) : go(attention_split_kernel<16, false>);
}

}  // namespace sgemm_emu
