// The residual stream's update and the norms before and after a block, and
// their gradients:
//     u = x, or norm(x) post_weight;   h = residual + alpha gate u;
//     y = norm(h) weight (1 + scale) + shift.
// One pass: a row is loaded once, stays in registers in 32 bits through both
// norms and is written once; y comes from the 32-bit h.  Bound by HBM.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "kq_norm.h"

namespace kq {

namespace {

// Eight values at any alignment of their elements (rows of an odd width start anywhere).
typedef uint32_t u32x4e __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4e __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }

// The first n (<= 8) of the eight values at p; the rest `fill`.
__device__ __forceinline__ void load8(const uint16_t* p, int n, float (&v)[8], float fill = 0.f) {
    if (n >= 8) {
        const u32x4e w = *reinterpret_cast<const u32x4e*>(p);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k] = __uint_as_float(w[k] << 16);
            v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k < n ? bf16_value(p[k]) : fill;
    }
}
__device__ __forceinline__ void load8(const float* p, int n, float (&v)[8], float fill = 0.f) {
    if (n >= 8) {
        const f32x4e a = *reinterpret_cast<const f32x4e*>(p), b = *reinterpret_cast<const f32x4e*>(p + 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[k] = a[k];
            v[4 + k] = b[k];
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k < n ? p[k] : fill;
    }
}
// Of a vector of the call's vector type, from element `at`.
__device__ __forceinline__ void load8(const void* p, int v16, int64_t at, int n, float (&v)[8]) {
    if (v16) load8(static_cast<const uint16_t*>(p) + at, n, v);
    else load8(static_cast<const float*>(p) + at, n, v);
}

__device__ __forceinline__ void store8(uint16_t* p, int n, const float (&v)[8]) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    u32x4e w;
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)v[2 * k], (__bf16)v[2 * k + 1]});
    if (n >= 8) {
        *reinterpret_cast<u32x4e*>(p) = w;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n) p[k] = (uint16_t)(w[k / 2] >> (16 * (k & 1)));
    }
}
__device__ __forceinline__ void store8(float* p, int n, const float (&v)[8]) {
    if (n >= 8) {
        *reinterpret_cast<f32x4e*>(p) = f32x4e{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4e*>(p + 4) = f32x4e{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n) p[k] = v[k];
    }
}

template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, ROWS, 0xf, false));
}

// Sum over the wave's lanes, the same for all of them.
__device__ __forceinline__ float wave_sum(float v) {
    v = dpp_add<0x128, 0xf>(v);  // row_ror: every lane of a row of 16 has the row's sum
    v = dpp_add<0x124, 0xf>(v);
    v = dpp_add<0x122, 0xf>(v);
    v = dpp_add<0x121, 0xf>(v);
    v = dpp_add<0x142, 0xa>(v);  // rows 0 and 2 onto 1 and 3, then 1 onto 2 and 3
    v = dpp_add<0x143, 0xc>(v);
    return __uint_as_float(__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

// N sums over the W waves that share a row.  red: N floats for each of the W waves, not written
// again before another barrier has passed.
template <int W, int N>
__device__ __forceinline__ void row_sums(float (&s)[N], float* red, int wave) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = wave_sum(s[i]);
    if (W == 1) return;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) red[wave * N + i] = s[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float t = red[i];
#pragma unroll
        for (int w = 1; w < W; ++w) t += red[w * N + i];
        s[i] = t;
    }
}

template <bool H16>
using Stored = typename std::conditional<H16, uint16_t, float>::type;

// Makes v the normed row: v - mean (layer) times the returned 1 / sqrt(mean square + eps).
// Elements past the row's end come and leave as zeros.  red: 2 W floats.
template <int W, int NV>
__device__ __forceinline__ void normalize(float (&v)[NV][8], const int (&n)[NV], int kind, float inv_d, float eps, float* red,
                                          int wave) {
    if (kind == 2) {
        float s[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int k = 0; k < 8; ++k) s[0] += v[j][k];
        row_sums<W, 1>(s, red, wave);
        const float mean = s[0] * inv_d;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[j][k] = k < n[j] ? v[j][k] - mean : 0.f;
    }
    float q[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) q[0] = fmaf(v[j][k], v[j][k], q[0]);
    row_sums<W, 1>(q, red + W, wave);
    const float r = 1.0f / sqrtf(fmaf(q[0], inv_d, eps));
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[j][k] *= r;
}

// Rows of W waves, NV vectors of eight values a lane; with W 1 the workgroup's four waves take a
// row each.
template <bool X16, bool S16, int W, int NV>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void block_norm_kernel(const NormParams p) {
    typedef Stored<X16> TX;
    typedef Stored<S16> TS;
    __shared__ float red[4 * W];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = W == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
    if (row >= p.M) return;  // a whole wave, and W > 1 has none
    const int t = W == 1 ? threadIdx.x & 63 : threadIdx.x, d = (int)p.d;
    const int64_t base = row * p.d, b = row / p.rows;
    const float inv_d = 1.0f / (float)d;
    int col[NV], n[NV];
    float v[NV][8], o[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        col[j] = 8 * (t + 64 * W * j);
        n[j] = min(8, d - col[j]);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[j][k] = o[j][k] = 0.f;
        if (n[j] > 0) load8(static_cast<const TX*>(p.x) + base + col[j], n[j], v[j]);
    }
    if (p.residual) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (n[j] > 0) load8(static_cast<const TS*>(p.residual) + base + col[j], n[j], o[j]);
    }
    if (p.post) {
        normalize<W, NV>(v, n, p.post, inv_d, p.eps, red, wave);
        if (p.post_weight) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float w[8];
                if (n[j] > 0) {
                    load8(p.post_weight, p.vec16, col[j], n[j], w);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[j][k] *= w[k];
                }
            }
        }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (n[j] <= 0) continue;
        if (p.gate) {
            float g[8];
            load8(p.gate, p.vec16, b * p.gate_stride + col[j], n[j], g);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[j][k] *= g[k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) v[j][k] = fmaf(p.alpha, v[j][k], o[j][k]);
        if (p.h) store8(static_cast<TS*>(p.h) + base + col[j], n[j], v[j]);
    }
    if (!p.y) return;
    normalize<W, NV>(v, n, p.norm, inv_d, p.eps, red + 2 * W, wave);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (n[j] <= 0) continue;
        float w[8];
        if (p.weight) {
            load8(p.weight, p.vec16, col[j], n[j], w);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[j][k] *= w[k];
        }
        if (p.scale) {
            load8(p.scale, p.vec16, b * p.scale_stride + col[j], n[j], w);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[j][k] = fmaf(v[j][k], w[k], v[j][k]);
        }
        if (p.shift) {
            load8(p.shift, p.vec16, b * p.shift_stride + col[j], n[j], w);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[j][k] += w[k];
        }
        store8(static_cast<TX*>(p.y) + base + col[j], n[j], v[j]);
    }
}

// ------------------------------------------------------------------ gradients
//     m = weight (1 + scale), n = norm(h), g = dy m
//     D = dh + r (g - [mean g] - n mean(g n))                     dresidual
//     du = alpha gate D, gx = du post_weight
//     dx = rx (gx - [mean gx] - xn mean(gx xn))                   du without a post norm
// and, per batch, the column sums of dy, dy n and D xn (xn: x or its norm), from which all vectors'
// gradients follow.  A workgroup of R teams of W waves walks a chunk of a batch's rows, R rows at a
// time, with the three sums of its columns in registers; the teams' sums meet in LDS in order, the
// chunks' in norm_grad_kernel, so nothing depends on timing.
template <bool X16, bool S16, bool POST, int W, int R, int NV>
__global__ __launch_bounds__(64 * W * R) void block_norm_backward_kernel(const NormParams p) {
    typedef Stored<X16> TX;
    typedef Stored<S16> TS;
    constexpr int COLS = 512 * W * NV;
    __shared__ float red[2][R][8 * W];
    __shared__ float meet[R > 1 ? R : 1][R > 1 ? COLS : 1];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = wave / W, tw = wave % W;
    const int t = threadIdx.x - 64 * W * team, d = (int)p.d;
    const int64_t b = blockIdx.x / p.chunks, c = blockIdx.x % p.chunks;
    const int64_t first = b * p.rows + c * p.rows / p.chunks, end = b * p.rows + (c + 1) * p.rows / p.chunks;
    const float inv_d = 1.0f / (float)d;
    int col[NV], n[NV];
    float s_dy[NV][8], s_dyn[NV][8], s_dx[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        col[j] = 8 * (t + 64 * W * j);
        n[j] = min(8, d - col[j]);
#pragma unroll
        for (int k = 0; k < 8; ++k) s_dy[j][k] = s_dyn[j][k] = s_dx[j][k] = 0.f;
    }
    const bool layer = p.norm == 2, post_layer = POST && p.post == 2;
    int turn = 0;
    for (int64_t at = first; at < end; at += R, turn ^= 1) {
        const int64_t row = at + team;
        const bool mine = row < end;  // the teams stay together: a team past the end works on zeros
        const int64_t base = row * p.d;
        float* const mem = red[turn][team];
        float h[NV][8], g[NV][8], x[NV][8], dh[NV][8];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int k = 0; k < 8; ++k) h[j][k] = g[j][k] = x[j][k] = dh[j][k] = 0.f;
            if (mine && n[j] > 0) {
                load8(static_cast<const TS*>(p.h) + base + col[j], n[j], h[j]);
                load8(static_cast<const TX*>(p.dy) + base + col[j], n[j], g[j]);
                if (p.x) load8(static_cast<const TX*>(p.x) + base + col[j], n[j], x[j]);
                if (p.dh) load8(static_cast<const TS*>(p.dh) + base + col[j], n[j], dh[j]);
            }
        }
        if (layer || post_layer) {
            float s[2] = {0.f, 0.f};
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    s[0] += h[j][k];
                    if (POST) s[1] += x[j][k];
                }
            row_sums<W, 2>(s, mem, tw);
            const float mh = layer ? s[0] * inv_d : 0.f, mx = post_layer ? s[1] * inv_d : 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    h[j][k] = k < n[j] ? h[j][k] - mh : 0.f;
                    if (POST) x[j][k] = k < n[j] ? x[j][k] - mx : 0.f;
                }
        }
        // the columns' sums of dy, then g = dy m
        float q[4] = {0.f, 0.f, 0.f, 0.f};
        float dyh[NV][8];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float w[8], m[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) m[k] = 1.f;
            if (n[j] > 0) {
                if (p.weight) load8(p.weight, p.vec16, col[j], n[j], m);
                if (p.scale) {
                    load8(p.scale, p.vec16, b * p.scale_stride + col[j], n[j], w);
#pragma unroll
                    for (int k = 0; k < 8; ++k) m[k] = fmaf(m[k], w[k], m[k]);
                }
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                s_dy[j][k] += g[j][k];
                dyh[j][k] = g[j][k] * h[j][k];
                g[j][k] *= m[k];
                q[0] = fmaf(h[j][k], h[j][k], q[0]);
                q[1] += g[j][k];
                q[2] = fmaf(g[j][k], h[j][k], q[2]);
                if (POST) q[3] = fmaf(x[j][k], x[j][k], q[3]);
            }
        }
        row_sums<W, 4>(q, mem + 2 * W, tw);
        // (a team past the end has zeros, and with eps 0 no factors)
        const float r = mine ? 1.0f / sqrtf(fmaf(q[0], inv_d, p.eps)) : 0.f;
        const float rx = !POST ? 1.f : mine ? 1.0f / sqrtf(fmaf(q[3], inv_d, p.eps)) : 0.f;
        const float mg = layer ? q[1] * inv_d : 0.f, mgn = q[2] * r * inv_d;
        float e[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float gt[8], D[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) gt[k] = 1.f;
            if (n[j] > 0 && p.gate) load8(p.gate, p.vec16, b * p.gate_stride + col[j], n[j], gt);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float nn = h[j][k] * r;
                s_dyn[j][k] = fmaf(dyh[j][k], r, s_dyn[j][k]);
                D[k] = fmaf(r, g[j][k] - mg - nn * mgn, dh[j][k]);
                if (POST) x[j][k] *= rx;
                s_dx[j][k] = fmaf(D[k], x[j][k], s_dx[j][k]);
            }
            if (mine && n[j] > 0 && p.dresidual) store8(static_cast<TS*>(p.dresidual) + base + col[j], n[j], D);
#pragma unroll
            for (int k = 0; k < 8; ++k) g[j][k] = p.alpha * gt[k] * D[k];
            if (POST) {
                if (n[j] > 0 && p.post_weight) {
                    load8(p.post_weight, p.vec16, col[j], n[j], gt);
#pragma unroll
                    for (int k = 0; k < 8; ++k) g[j][k] *= gt[k];
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (k >= n[j]) g[j][k] = 0.f;
                    e[0] += g[j][k];
                    e[1] = fmaf(g[j][k], x[j][k], e[1]);
                }
            } else if (mine && n[j] > 0 && p.dx) {
                store8(static_cast<TX*>(p.dx) + base + col[j], n[j], g[j]);
            }
        }
        if (POST) {
            row_sums<W, 2>(e, mem + 6 * W, tw);
            const float m0 = post_layer ? e[0] * inv_d : 0.f, m1 = e[1] * inv_d;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
#pragma unroll
                for (int k = 0; k < 8; ++k) g[j][k] = rx * (g[j][k] - m0 - x[j][k] * m1);
                if (mine && n[j] > 0 && p.dx) store8(static_cast<TX*>(p.dx) + base + col[j], n[j], g[j]);
            }
        }
    }
    // the teams' sums, in order
    float* const out = p.partial + (int64_t)blockIdx.x * 3 * p.d;
    auto put = [&](int which, const float (&s)[NV][8]) {
        if (R == 1) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (n[j] > 0) store8(out + which * p.d + col[j], n[j], s[j]);
            return;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (n[j] > 0) {
#pragma unroll
                for (int k = 0; k < 8; ++k) meet[R > 1 ? team : 0][R > 1 ? col[j] + k : 0] = s[j][k];
            }
        __syncthreads();
        for (int i = threadIdx.x; i < d; i += 64 * W * R) {
            float v = meet[0][R > 1 ? i : 0];
#pragma unroll
            for (int w = 1; w < R; ++w) v += meet[R > 1 ? w : 0][R > 1 ? i : 0];
            out[which * p.d + i] = v;
        }
    };
    put(0, s_dy);
    put(1, s_dyn);
    put(2, s_dx);
}

// The vectors' gradients from the chunks' column sums.  32 columns a workgroup, 32 threads a column.
// blockIdx.y < batches: one batch's dshift, dscale and dgate; == batches: dweight and dpost_weight.
__global__ __launch_bounds__(1024) void norm_grad_kernel(const NormParams p) {
    __shared__ float sum[3][32][33];
    const int cx = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + cx;
    const bool in = c < p.d, all = blockIdx.y == p.batches;
    auto vec = [&](const void* q, int64_t at) { return p.vec16 ? bf16_value(static_cast<const uint16_t*>(q)[at]) : static_cast<const float*>(q)[at]; };
    const int64_t from = all ? 0 : blockIdx.y * p.chunks, to = all ? p.batches * p.chunks : from + p.chunks;
    float s[3] = {0.f, 0.f, 0.f};
    if (in) {
#pragma unroll 4
        for (int64_t i = from + part; i < to; i += 32) {
            const float* const src = p.partial + i * 3 * p.d + c;
            float f1 = 1.f, f2 = 1.f;
            if (all) {
                if (p.scale) f1 += vec(p.scale, i / p.chunks * p.scale_stride + c);
                if (p.gate) f2 = vec(p.gate, i / p.chunks * p.gate_stride + c);
            }
            s[0] += src[0];
            s[1] = fmaf(f1, src[p.d], s[1]);
            s[2] = fmaf(f2, src[2 * p.d], s[2]);
        }
    }
#pragma unroll
    for (int w = 0; w < 3; ++w) sum[w][part][cx] = s[w];
    __syncthreads();
    if (part >= 3 || !in) return;
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) v += sum[part][i][cx];
    if (all) {
        if (part == 1 && p.dweight) p.dweight[c] = v;
        if (part == 2 && p.dpost_weight) p.dpost_weight[c] = p.alpha * v;
        return;
    }
    const int64_t to_c = blockIdx.y * p.d + c;
    if (part == 0 && p.dshift) p.dshift[to_c] = v;
    if (part == 1 && p.dscale) p.dscale[to_c] = p.weight ? v * vec(p.weight, c) : v;
    if (part == 2 && p.dgate) p.dgate[to_c] = p.alpha * (p.post_weight ? v * vec(p.post_weight, c) : v);
}

template <bool X16, bool S16>
hipError_t launch_forward(const NormParams& p, hipStream_t st) {
    const int64_t vecs = (p.d + 7) / 8;
#define KQ_NORM(W, NV)                                                                                                  \
    do {                                                                                                                \
        hipLaunchKernelGGL((block_norm_kernel<X16, S16, W, NV>), dim3((unsigned)(W == 1 ? (p.M + 3) / 4 : p.M)),          \
                           dim3(W == 1 ? 256 : 64 * W), 0, st, p);                                                       \
        return hipGetLastError();                                                                                       \
    } while (0)
    if (p.M >= 1024 || vecs <= 64) {
        if (vecs <= 64) KQ_NORM(1, 1);
        if (vecs <= 128) KQ_NORM(1, 2);
        if (vecs <= 192) KQ_NORM(1, 3);
        if (vecs <= 256) KQ_NORM(1, 4);
        if (vecs <= 384) KQ_NORM(1, 6);
    }
    if (vecs <= 256) KQ_NORM(4, 1);
    if (vecs <= 512) KQ_NORM(4, 2);
    if (vecs <= 1024) KQ_NORM(4, 4);
    KQ_NORM(16, 2);
#undef KQ_NORM
}

// Columns that W waves hold with 2 and with 3 vectors a lane.
template <class F>
hipError_t by_width(int64_t d, F f) {
    const int64_t vecs = (d + 7) / 8;
    int w = 1;
    for (; w < 16; w *= 2) {
        if (vecs <= 128 * w) return f(w, 2);
        if (vecs <= 192 * w) return f(w, 3);
    }
    return f(16, 2);
}

constexpr int kBackwardWaves = 8;  // of a workgroup, where a row needs no more

template <bool X16, bool S16, bool POST>
hipError_t launch_backward(const NormParams& p, hipStream_t st) {
    const dim3 grid((unsigned)(p.batches * p.chunks));
    return by_width(p.d, [&](int w, int nv) {
#define KQ_NORM(W, NV)                                                                                                            \
    if (w == W && nv == NV) {                                                                                                     \
        constexpr int R = W < kBackwardWaves ? kBackwardWaves / W : 1;                                                            \
        hipLaunchKernelGGL((block_norm_backward_kernel<X16, S16, POST, W, R, NV>), grid, dim3(64 * W * R), 0, st, p);              \
    }
        KQ_NORM(1, 2) KQ_NORM(1, 3) KQ_NORM(2, 2) KQ_NORM(2, 3) KQ_NORM(4, 2) KQ_NORM(4, 3) KQ_NORM(8, 2) KQ_NORM(8, 3)
        KQ_NORM(16, 2)
#undef KQ_NORM
        return hipGetLastError();
    });
}

}  // namespace

int64_t norm_chunks(int64_t M, int64_t batches, int64_t d) {
    int64_t chunks = 1;
    (void)by_width(d, [&](int w, int) {
        const int64_t teams = w < kBackwardWaves ? kBackwardWaves / w : 1;
        const int64_t rows = M / batches;
        chunks = std::max<int64_t>(1, std::min<int64_t>((rows + teams - 1) / teams, 512 / batches));
        return hipSuccess;
    });
    return chunks;
}

hipError_t launch_block_norm(const NormParams& p, hipStream_t st) {
    if (p.x16) return p.stream16 ? launch_forward<true, true>(p, st) : launch_forward<true, false>(p, st);
    return p.stream16 ? launch_forward<false, true>(p, st) : launch_forward<false, false>(p, st);
}

hipError_t launch_block_norm_backward(const NormParams& p, hipStream_t st) {
    hipError_t e;
    if (p.post) {
        if (p.x16) e = p.stream16 ? launch_backward<true, true, true>(p, st) : launch_backward<true, false, true>(p, st);
        else e = p.stream16 ? launch_backward<false, true, true>(p, st) : launch_backward<false, false, true>(p, st);
    } else {
        if (p.x16) e = p.stream16 ? launch_backward<true, true, false>(p, st) : launch_backward<true, false, false>(p, st);
        else e = p.stream16 ? launch_backward<false, true, false>(p, st) : launch_backward<false, false, false>(p, st);
    }
    const bool grads = p.dgate || p.dscale || p.dshift, weights = p.dweight || p.dpost_weight;
    if (e != hipSuccess || (!grads && !weights)) return e;
    const dim3 grid((unsigned)((p.d + 31) / 32), (unsigned)(p.batches + (weights ? 1 : 0)));
    hipLaunchKernelGGL(norm_grad_kernel, grid, dim3(1024), 0, st, p);
    return hipGetLastError();
}

}  // namespace kq
