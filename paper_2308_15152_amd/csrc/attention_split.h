// FP32 tensors split into FP16 planes in a workspace, for the kernels that multiply them.
#pragma once

#include "attention.h"

namespace sgemm_emu {

// A tensor's planes: views of rows of hi and, one plane's width behind, lo, and what each
// row (token, head) was divided by.
struct SplitTensor {
    sgemm_emu_view_t planes;
    float* factors;  // [token in all][head]
};

// Elements of a plane's row.
inline int plane_width(int size) { return size <= 64 ? 64 : 128; }

// Bytes of a tensor's planes and factors (a multiple of 256).
int64_t split_bytes(int64_t tokens, int heads, int size);

// Up to four tensors of `size` elements, with their places in a workspace.
class Splitter {
public:
    Splitter(int size, void* workspace) : size_(size), at_((char*)workspace) {}
    // Planes of x, (batch, tokens, heads).
    SplitTensor add(const sgemm_emu_view_t& x, int batch, int tokens, int heads);
    hipError_t launch(hipStream_t stream) const;

    struct Job {
        sgemm_emu_view_t x;
        SplitTensor to;
        int tokens, heads;
        int64_t rows;
    };

private:
    int size_;
    char* at_;
    int count_ = 0;
    Job jobs_[4];
};

}  // namespace sgemm_emu
