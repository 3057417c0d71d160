// W4A16 linear layers: a few rows of 16- or 32-bit activations and an MXFP4
// weight,
//     out = residual + gate act(x deq(B)^T + bias).
// The weight's values are exact in bf16, so the product runs on the bf16 matrix
// cores with the weight as operand A: 16 of its rows x 32 columns, lane (r, g) =
// row r (r = lane % 16, g = lane / 16), x's rows as operand B.  The order of
// columns in the sum is free: a lane takes the 16 bytes of a block of 32 of its
// row, four blocks a wave and step.  x in 32 bits goes in as three bf16 terms
// (8 + 8 + 8 bits: exact).
//
// Bound by the weight's read.  A workgroup's waves share a tile of 16 rows and
// take its columns in turn, and add their sums in LDS.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "kq_act.h"
#include "kq_mx.h"
#include "kq_serve.h"

namespace kq {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kVecWaves = 8;
constexpr int kVecRows = 16;  // of a workgroup, of the weight and of x

// Eight values of x as bf16 terms.
template <bool X16, int TERMS>
__device__ __forceinline__ void load_terms(const void* x, int64_t at, bf16x8 (&t)[TERMS]) {
    if constexpr (X16) {
        typedef uint32_t W __attribute__((ext_vector_type(4), aligned(2)));
        const W w = *reinterpret_cast<const W*>(static_cast<const uint16_t*>(x) + at);
        t[0] = __builtin_bit_cast(bf16x8, u32x4v{w[0], w[1], w[2], w[3]});
    } else {
        typedef float W __attribute__((ext_vector_type(4), aligned(4)));
        const W a = *reinterpret_cast<const W*>(static_cast<const float*>(x) + at);
        const W b = *reinterpret_cast<const W*>(static_cast<const float*>(x) + at + 4);
        float f[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
#pragma unroll
        for (int n = 0; n < TERMS; ++n) {
            u32x4v w;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                w[k] = __builtin_amdgcn_perm(__float_as_uint(f[2 * k + 1]), __float_as_uint(f[2 * k]), 0x07060302u);
                f[2 * k] -= bf16_low(w[k]);
                f[2 * k + 1] -= bf16_high(w[k]);
            }
            t[n] = __builtin_bit_cast(bf16x8, w);
        }
    }
}

__device__ __forceinline__ float value_of(const void* p, int is16, int64_t at) {
    return is16 ? bf16_low(static_cast<const uint16_t*>(p)[at]) : static_cast<const float*>(p)[at];
}

template <bool X16>
__global__ __launch_bounds__(64 * kVecWaves) void matvec_kernel(MatvecParams p) {
    constexpr int kTerms = X16 ? 1 : 3;
    const LinearParams& l = p.l;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * kVecRows, m0 = (int64_t)blockIdx.y * kVecRows;
    const int64_t row = min(n0 + r, l.g.N - 1);
    const int blocks = (int)(l.g.K / 32);
    const uint8_t* const codes = l.g.b_codes + row * (l.g.K / 2);
    const uint8_t* const scales = l.g.b_scales + row * blocks;
    const bool live = m0 + r < l.g.M;
    const int64_t xrow = (m0 + r) * p.ldx;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int b0 = 4 * wave; b0 < blocks; b0 += 4 * kVecWaves) {
        const int b = b0 + g;
        u32x4v w = {0u, 0u, 0u, 0u};
        uint32_t s = 127u;
        bf16x8 x[4][kTerms];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int n = 0; n < kTerms; ++n) x[k][n] = __builtin_bit_cast(bf16x8, u32x4v{0u, 0u, 0u, 0u});
        if (b < blocks) {
            w = *reinterpret_cast<const u32x4v*>(codes + 16 * (int64_t)b);
            s = scales[b];
            if (live) {
#pragma unroll
                for (int k = 0; k < 4; ++k) load_terms<X16, kTerms>(p.x, xrow + 32 * (int64_t)b + 8 * k, x[k]);
            }
        }
        const float sc = mx_scale(s);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bf16x8 a = __builtin_bit_cast(
                bf16x8, u32x4v{e2m1_pair<0>(w[k], sc), e2m1_pair<1>(w[k], sc), e2m1_pair<2>(w[k], sc), e2m1_pair<3>(w[k], sc)});
#pragma unroll
            for (int n = 0; n < kTerms; ++n) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, x[k][n], acc, 0, 0, 0);
        }
    }
    __shared__ float sums[kVecWaves][kVecRows][kVecRows + 1];  // [wave][row of x][row of the weight]
#pragma unroll
    for (int k = 0; k < 4; ++k) sums[wave][r][4 * g + k] = acc[k];
    __syncthreads();
    with_act(l.act, [&](auto a) __attribute__((always_inline)) {
        constexpr Act A = decltype(a)::value;
        constexpr int kWide = A == Act::Swiglu ? 2 : 1, kOut = kVecRows / kWide;
        const int i = threadIdx.x;
        if (i >= kVecRows * kOut) return;
        const int m = i / kOut, n = kWide * (i % kOut);
        if (m0 + m >= l.g.M || n0 + n >= l.g.N) return;
        float v[kWide];
#pragma unroll
        for (int j = 0; j < kWide; ++j) {
            v[j] = 0.f;
#pragma unroll
            for (int w = 0; w < kVecWaves; ++w) v[j] += sums[w][m][n + j];
            if (l.bias) v[j] += value_of(l.bias, l.vec16, n0 + n + j);
        }
        float y = activate<A>(v[0]);
        if constexpr (kWide == 2) y *= v[1];
        const int64_t column = (n0 + n) / kWide;
        if (l.gate) y *= value_of(l.gate, l.vec16, (m0 + m) / l.gate_rows * l.gate_stride + column);
        if (l.residual) y += value_of(l.residual, l.out16, (m0 + m) * l.ldr + column);
        const int64_t at = (m0 + m) * l.ldo + column;
        if (l.out16) static_cast<__bf16*>(l.out)[at] = (__bf16)y;
        else static_cast<float*>(l.out)[at] = y;
    });
}

}  // namespace

hipError_t launch_matvec(const MatvecParams& p, hipStream_t st) {
    const dim3 grid((unsigned)((p.l.g.N + kVecRows - 1) / kVecRows), (unsigned)((p.l.g.M + kVecRows - 1) / kVecRows));
    if (p.x16) matvec_kernel<true><<<grid, 64 * kVecWaves, 0, st>>>(p);
    else matvec_kernel<false><<<grid, 64 * kVecWaves, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace kq
