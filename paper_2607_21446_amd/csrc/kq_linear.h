// Internal interface of the W4A4 linear layers (kq_linear.hip) to the C-ABI layer.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kq_kernels.h"

namespace kq {

enum class Act { None = 0, Gelu = 1, GeluTanh = 2, Silu = 3, Relu = 4, Swiglu = 5 };

// out[m] = residual[m] + gate_b act(product[m] + bias), or row_scale[m] act(product[m] + bias_e).
// Sizes already validated by the caller.
struct LinearParams {
    GemmParams g{};  // operands and sizes (M: rows of the product); no C
    Act act = Act::None;
    int vec16 = 0;   // bias and gate: 1 bf16, 0 fp32
    int out16 = 0;   // out and residual: 1 bf16, 0 fp32
    const void* bias = nullptr;  // [N], or [E, N]
    const void* gate = nullptr;  // row b at b * gate_stride, of rows b gate_rows .. (b + 1) gate_rows - 1
    int64_t gate_stride = 0, gate_rows = 1;
    const float* row_scale = nullptr;  // [M]
    const void* residual = nullptr;    // [M, ldr]
    int64_t ldr = 0;
    void* out = nullptr;  // [M, ldo]; N / 2 columns with Swiglu
    int64_t ldo = 0;
    // grouped: rows offsets[e] .. offsets[e + 1] - 1 take expert e's weight, b_codes + e N K / 2
    const int32_t* offsets = nullptr;
    int64_t experts = 0;
    int stream_out = 0;  // filled in by the launcher: the output is stored past the caches
};

hipError_t launch_mxfp4_linear(LinearParams p, hipStream_t st);  // hipErrorInvalidConfiguration: more than one launch holds
// Workgroups of a grouped call's largest launch, against the grid limit.
int64_t mxfp4_grouped_workgroups(const LinearParams& p);

}  // namespace kq
