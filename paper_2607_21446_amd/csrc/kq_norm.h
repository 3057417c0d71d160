// Internal interface of the norm operator (kq_norm.hip) to the C-ABI layer.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kq {

constexpr int64_t kNormMaxColumns = 16384;  // a row stays in the registers of one workgroup

// Sizes already validated by the caller.  Vectors of a batch: row b at b * stride.
struct NormParams {
    const void* x;         // [M, d]
    const void* residual;  // [M, d] or null
    const void* gate;      // [B, d] or null
    const void* scale;
    const void* shift;
    int64_t gate_stride, scale_stride, shift_stride;
    const void* weight;       // [d] or null
    const void* post_weight;  // [d] or null
    int64_t M, d;
    int64_t rows;        // rows of a batch, M / B
    int norm, post;      // 0 none, 1 rms, 2 layer
    float alpha, eps;
    int x16, stream16, vec16;  // 1: bf16, 0: fp32
    void* h;  // [M, d] or null
    void* y;  // [M, d] or null (norm 0)
    // backward: h is read, x may be null
    const void* dy;         // [M, d], type of x
    const void* dh;         // [M, d] or null, type of the stream
    void* dx;               // [M, d] or null, type of x
    void* dresidual;        // [M, d] or null, type of the stream
    float *dgate, *dscale, *dshift;  // [B, d] or null
    float *dweight, *dpost_weight;   // [d] or null
    float* partial;         // [B, chunks, 3, d]
    int64_t batches;
    // filled in by the launcher: workgroups of a batch; waves that share a row and rows that a workgroup
    // works on at once
    int64_t chunks;
    int waves, teams;
};

// Workgroups of a batch in the backward pass, each with its partial sums.
int64_t norm_chunks(int64_t M, int64_t batches, int64_t d);
hipError_t launch_block_norm(NormParams p, hipStream_t st);
hipError_t launch_block_norm_backward(NormParams p, hipStream_t st);

}  // namespace kq
