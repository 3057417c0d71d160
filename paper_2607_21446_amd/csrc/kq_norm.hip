// The residual stream's update and the norms before and after a block, and
// their gradients:
//     u = x, or norm(x) post_weight;   h = residual + alpha gate u;
//     y = norm(h) weight (1 + scale) + shift.
// One pass: a row is loaded once, stays in registers in 32 bits through both
// norms and is written once; y comes from the 32-bit h.  Bound by HBM: 4608 x
// 3072 in bf16 (113 MB) takes 21.9 us, 5.2 TB/s, which is a large copy's rate.
// Rows of more than 8192 columns take 1024 threads of 128 registers, which only
// the forward pass of bf16 rows of whole vectors keeps without spills (4608 x
// 12288: 90 us, 5.0 TB/s; with an fp32 stream and two norms 206, 3.3 TB/s;
// gradients 481, 1.4 TB/s).
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

template <bool B16>
using Stored = typename std::conditional<B16, uint16_t, float>::type;

// Eight values as they are stored.
template <bool B16>
struct Raw {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    typedef typename std::conditional<B16, u32x4e, f32x4e>::type Mem;  // at any alignment of the elements
    typename std::conditional<B16, u32x4, f32x4>::type v[B16 ? 1 : 2];
    // Waits for the load here.
    __device__ __forceinline__ void settle() {
        asm volatile("" : "+v"(v[0]));
        if (!B16) asm volatile("" : "+v"(v[B16 ? 0 : 1]));
    }
};

// The eight values at `at`, of which n (1 to 8) are inside the row: fewer as the eight that end with the
// row's last (shifted once they are used, so that nothing waits for the load here).  Rows of less than
// eight values one by one.
template <bool B16>
__device__ __forceinline__ Raw<B16> load_raw(const void* base, int64_t at, int n, int d) {
    Raw<B16> r;
    const Stored<B16>* p = static_cast<const Stored<B16>*>(base) + at;
    if (n < 8 && d < 8) {
        r = Raw<B16>{};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (k >= n) break;
            if constexpr (B16) r.v[0][k / 2] |= (uint32_t)p[k] << (16 * (k & 1));
            else r.v[k / 4][k % 4] = p[k];
        }
        return r;
    }
    if (n < 8) p -= 8 - n;
    r.v[0] = *reinterpret_cast<const typename Raw<B16>::Mem*>(p);
    if (!B16) r.v[B16 ? 0 : 1] = *reinterpret_cast<const typename Raw<B16>::Mem*>(p + 4);
    return r;
}
template <bool B16>
__device__ __forceinline__ void values(const Raw<B16>& r, int n, int d, float (&f)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if constexpr (B16) f[k] = __uint_as_float(k & 1 ? r.v[0][k / 2] & 0xffff0000u : r.v[0][k / 2] << 16);
        else f[k] = r.v[k / 4][k % 4];
    }
    if (n < 8 && n > 0 && d >= 8) {
        const int by = 8 - n;
#pragma unroll
        for (int step = 4; step > 0; step >>= 1)
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (by & step) f[k] = k + step < 8 ? f[k + step] : 0.f;
    }
}

template <bool B16>
__device__ __forceinline__ Raw<B16> packed(const float (&f)[8]) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    Raw<B16> r;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if constexpr (!B16) r.v[k / 4][k % 4] = f[k];
        else if (k % 2 == 0) r.v[0][k / 2] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)f[k], (__bf16)f[k + 1]});
    }
    return r;
}
// The first n of eight values (n >= 1).
template <bool B16>
__device__ __forceinline__ void store_raw(void* base, int64_t at, int n, const Raw<B16>& r) {
    Stored<B16>* const p = static_cast<Stored<B16>*>(base) + at;
    if (n >= 8) {
        *reinterpret_cast<typename Raw<B16>::Mem*>(p) = r.v[0];
        if (!B16) *reinterpret_cast<typename Raw<B16>::Mem*>(p + 4) = r.v[B16 ? 0 : 1];
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (k >= n) break;
            if constexpr (B16) p[k] = (uint16_t)(r.v[0][k / 2] >> (16 * (k & 1)));
            else p[k] = r.v[k / 4][k % 4];
        }
    }
}

// A workgroup is R teams of W waves; a team has a row at a time, lane t of it the columns 8 (t + 64 W j)
// .. + 7 for j < NV.  A workgroup's rows are all of one batch, so the batch's vectors stay in registers, and the
// next row is loaded while this one is worked on.  Workgroups take rows in turn: at any time they work on
// neighbouring rows (a run of rows each: 4608 x 3072 23.3 us, 22.6 so; gradients of 18432 x 1152 63.3 and 61.5).
// WHOLE: d is a multiple of 8.
template <int NV, bool WHOLE>
struct Place {
    int W, R, team, wave;   // of the workgroup; this wave's team and its place there
    int d;
    int col[NV];            // first columns
    int left[NV];           // columns of the row from there on (may be <= 0)
    int b;                  // batch
    int64_t row, end, step; // the team's first row, the batch's end, rows from one of the team's to the next
    float count, inv_d;     // columns of this wave; 1 / d
    __device__ __forceinline__ explicit Place(const NormParams& p) {
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        W = p.waves;
        R = p.teams;
        team = w / W;
        wave = w - team * W;
        const int t = 64 * wave + (threadIdx.x & 63);
        d = (int)p.d;
        int in_wave = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            col[j] = 8 * (t + 64 * W * j);
            left[j] = d - col[j];
            in_wave += min(512, max(0, d - 512 * (wave + W * j)));
        }
        count = (float)in_wave;
        inv_d = 1.0f / (float)d;
        b = (int)(blockIdx.x / (uint32_t)p.chunks);
        const uint32_t c = blockIdx.x - (uint32_t)b * (uint32_t)p.chunks;
        row = (int64_t)b * p.rows + c * R + team;
        end = ((int64_t)b + 1) * p.rows;
        step = p.chunks * R;
    }
    __device__ __forceinline__ bool any(int j) const { return left[j] > 0; }
    __device__ __forceinline__ int n(int j) const { return WHOLE ? 8 : left[j]; }             // with any(j)
    // Makes v[j] zeros past the row's end.
    __device__ __forceinline__ void clip(int j, float (&v)[8]) const {
        if (WHOLE) return;  // a vector is inside or outside as a whole: see add()
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k < left[j] ? v[k] : 0.f;
    }
    // s += t, a sum over vector j, if it is inside the row.
    __device__ __forceinline__ void add(int j, float t, float& s) const { s += !WHOLE || left[j] > 0 ? t : 0.f; }
    // This lane's sum of the values inside the row (past its end they are zeros or, with WHOLE, anything).
    __device__ __forceinline__ float total(const float (&v)[NV][8]) const {
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            add(j, ((v[j][0] + v[j][1]) + (v[j][2] + v[j][3])) + ((v[j][4] + v[j][5]) + (v[j][6] + v[j][7])), s);
        return s;
    }
    __device__ __forceinline__ float squares(const float (&v)[NV][8]) const {
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float t[2] = {v[j][0] * v[j][0], v[j][1] * v[j][1]};
#pragma unroll
            for (int k = 2; k < 8; ++k) t[k & 1] = fmaf(v[j][k], v[j][k], t[k & 1]);
            add(j, t[0] + t[1], s);
        }
        return s;
    }
};

constexpr int kMaxWaves = 16, kTeamWaves = 8;
// One round of a row's sums, 8 numbers of every wave; rounds alternate, so that a slot is written again
// only after another barrier.
typedef float Slots[kMaxWaves][8];

// N values of this wave to its team.  One barrier.
template <int N>
__device__ __forceinline__ void publish(const float (&mine)[N], float* slot) {
    static_assert(N <= 8, "a slot");
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) slot[i] = mine[i];
    }
    __syncthreads();
}

__device__ __forceinline__ float inverse_root(float q, float inv_d, float eps) { return __builtin_amdgcn_rsqf(fmaf(q, inv_d, eps)); }

// Makes v a row's values less a LayerNorm's mean in this wave, and gives what is left of the row's mean (rest, to be
// added to v) and the sum of squares about it.  The waves sum about their own means m_w, so that one round does:
// sum (v - mean)^2 = sum_w [q_w + n_w (m_w - mean)^2].  What v holds past the row's end is no part of the sums.
template <int NV, bool WHOLE>
__device__ __forceinline__ float centre(float (&v)[NV][8], const Place<NV, WHOLE>& at, bool layer, Slots& s, float& rest) {
    float own[3] = {0.f, 0.f, at.count};  // mean, squares, columns
    rest = 0.f;
    if (layer) {
        own[0] = wave_sum(at.total(v)) / at.count;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[j][k] -= own[0];
            at.clip(j, v[j]);
        }
    }
    own[1] = wave_sum(at.squares(v));
    if (at.W == 1) return own[1];
    publish(own, s[at.team * at.W + at.wave]);
    float sum = 0.f, q = 0.f;
    for (int w = 0; w < at.W; ++w) {
        const float* const o = s[at.team * at.W + w];
        sum = fmaf(o[0], o[2], sum);
        q += o[1];
    }
    if (layer) {
        const float mean = sum * at.inv_d;
        for (int w = 0; w < at.W; ++w) {
            const float* const o = s[at.team * at.W + w];
            const float off = o[0] - mean;
            q = fmaf(o[2] * off, off, q);
        }
        rest = own[0] - mean;
    }
    return q;
}

template <bool X16, bool S16, bool WHOLE, int NV, int THREADS>
__global__ __launch_bounds__(THREADS) void block_norm_kernel(const NormParams p) {
    __shared__ Slots slots[4];
    const Place<NV, WHOLE> at(p);
    struct Loaded {
        Raw<X16> x[NV];
        Raw<S16> r[NV];
        __device__ __forceinline__ void settle() {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                x[j].settle();
                r[j].settle();
            }
        }
    };
    auto load = [&](int64_t row, Loaded& l) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (row < at.end && at.any(j)) {
                l.x[j] = load_raw<X16>(p.x, row * p.d + at.col[j], at.n(j), at.d);
                if (p.residual) l.r[j] = load_raw<S16>(p.residual, row * p.d + at.col[j], at.n(j), at.d);
            }
    };
    Loaded next{};
    load(at.row, next);
    float gp[NV][8], m[NV][8], sh[NV][8];  // alpha gate post_weight; weight (1 + scale); shift
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            gp[j][k] = p.alpha;
            m[j][k] = 1.f;
            sh[j][k] = 0.f;
        }
        if (!at.any(j)) continue;
        if (p.gate) {
            load8(p.gate, p.vec16, at.b * p.gate_stride + at.col[j], at.n(j), w);
#pragma unroll
            for (int k = 0; k < 8; ++k) gp[j][k] *= w[k];
        }
        if (p.post_weight) {
            load8(p.post_weight, p.vec16, at.col[j], at.n(j), w);
#pragma unroll
            for (int k = 0; k < 8; ++k) gp[j][k] *= w[k];
        }
        if (p.weight) load8(p.weight, p.vec16, at.col[j], at.n(j), m[j]);
        if (p.scale) {
            load8(p.scale, p.vec16, at.b * p.scale_stride + at.col[j], at.n(j), w);
#pragma unroll
            for (int k = 0; k < 8; ++k) m[j][k] = fmaf(m[j][k], w[k], m[j][k]);
        }
        if (p.shift) load8(p.shift, p.vec16, at.b * p.shift_stride + at.col[j], at.n(j), sh[j]);
    }
    int turn = 0;
    // the teams stay together (the rounds' barriers): one past the chunk's end works on what it has
    for (int64_t row = at.row; row - at.team < at.end; row += at.step, turn ^= 1) {
        float v[NV][8], o[NV][8];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            values(next.x[j], at.n(j), at.d, v[j]);
            values(next.r[j], at.n(j), at.d, o[j]);
        }
        load(row + at.step, next);
        __builtin_amdgcn_sched_barrier(0);  // the next row's loads stay ahead of this one's work
        const bool mine = row < at.end;
        if (p.post) {
            float rest;
            const float q = centre(v, at, p.post == 2, slots[2 * turn], rest);
            const float r = inverse_root(q, at.inv_d, p.eps);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[j][k] = (v[j][k] + rest) * r;
                if (p.post == 2) at.clip(j, v[j]);  // rest reaches past the row's end too, where the second norm sums zeros
            }
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[j][k] = fmaf(gp[j][k], v[j][k], o[j][k]);
        }
        Raw<S16> h[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) h[j] = packed<S16>(v[j]);
        // Loads and stores are waited for in order: the next row's loads are waited for before this row's stores,
        // which then have the next row's work to finish in.
        auto store_h = [&] {
            next.settle();
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (mine && at.any(j) && p.h) store_raw<S16>(p.h, row * p.d + at.col[j], at.n(j), h[j]);
        };
        if (!p.y) {
            store_h();
            continue;
        }
        float rest;
        const float q = centre(v, at, p.norm == 2, slots[2 * turn + 1], rest);
        const float r = inverse_root(q, at.inv_d, p.eps);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[j][k] = fmaf((v[j][k] + rest) * r, m[j][k], sh[j][k]);
        }
        store_h();
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (mine && at.any(j)) store_raw<X16>(p.y, row * p.d + at.col[j], at.n(j), packed<X16>(v[j]));
    }
}

// ------------------------------------------------------------------ gradients
//     m = weight (1 + scale), n = norm(h), g = dy m
//     D = dh + r (g - [mean g] - n mean(g n))                     dresidual
//     du = alpha gate D, gx = du post_weight
//     dx = rx (gx - [mean gx] - xn mean(gx xn))                   du without a post norm
// and, per batch, the column sums of dy, dy n and D xn (xn: x or its norm), from which all vectors'
// gradients follow.  A team walks its rows with the three sums of its columns in registers; the teams'
// sums meet in LDS in order, the chunks' in norm_grad_kernel, so nothing depends on timing.
template <bool X16, bool S16, bool POST, bool WHOLE, int NV, int THREADS>
__global__ __launch_bounds__(THREADS) void block_norm_backward_kernel(const NormParams p) {
    __shared__ Slots slots[4];
    __shared__ float meet[512 * kTeamWaves * NV];  // R rows of sums, R > 1 only with R W <= kTeamWaves
    const Place<NV, WHOLE> at(p);
    const int d = (int)p.d, me = at.team * at.W + at.wave;
    const bool layer = p.norm == 2, post_layer = POST && p.post == 2;
    float m[NV][8], gp[NV][8];  // weight (1 + scale); alpha gate post_weight
    float s_dy[NV][8], s_dyn[NV][8], s_dx[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            s_dy[j][k] = s_dyn[j][k] = s_dx[j][k] = 0.f;
            m[j][k] = 1.f;
            gp[j][k] = p.alpha;
        }
        if (!at.any(j)) continue;
        if (p.gate) {
            load8(p.gate, p.vec16, at.b * p.gate_stride + at.col[j], at.n(j), w);
#pragma unroll
            for (int k = 0; k < 8; ++k) gp[j][k] *= w[k];
        }
        if (POST && p.post_weight) {
            load8(p.post_weight, p.vec16, at.col[j], at.n(j), w);
#pragma unroll
            for (int k = 0; k < 8; ++k) gp[j][k] *= w[k];
        }
        if (p.weight) load8(p.weight, p.vec16, at.col[j], at.n(j), m[j]);
        if (p.scale) {
            load8(p.scale, p.vec16, at.b * p.scale_stride + at.col[j], at.n(j), w);
#pragma unroll
            for (int k = 0; k < 8; ++k) m[j][k] = fmaf(m[j][k], w[k], m[j][k]);
        }
    }
    struct Loaded {
        Raw<X16> g[NV], x[NV];
        Raw<S16> h[NV], dh[NV];
        __device__ __forceinline__ void settle() {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                g[j].settle();
                x[j].settle();
                h[j].settle();
                dh[j].settle();
            }
        }
    };
    auto load = [&](int64_t row, Loaded& l) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (row < at.end) {
                if (at.any(j)) {
                    const int64_t i = row * p.d + at.col[j];
                    l.h[j] = load_raw<S16>(p.h, i, at.n(j), at.d);
                    l.g[j] = load_raw<X16>(p.dy, i, at.n(j), at.d);
                    if (p.x) l.x[j] = load_raw<X16>(p.x, i, at.n(j), at.d);
                    if (p.dh) l.dh[j] = load_raw<S16>(p.dh, i, at.n(j), at.d);
                }
            } else {  // zeros add nothing to the sums
                l.h[j] = Raw<S16>{};
                l.g[j] = Raw<X16>{};
                l.x[j] = Raw<X16>{};
                l.dh[j] = Raw<S16>{};
            }
        }
    };
    Loaded next{};
    load(at.row, next);
    int turn = 0;
    for (int64_t row = at.row; row - at.team < at.end; row += at.step, turn ^= 1) {
        const bool mine = row < at.end;
        float h[NV][8], g[NV][8], x[NV][8], dh[NV][8];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            values(next.h[j], at.n(j), at.d, h[j]);
            values(next.g[j], at.n(j), at.d, g[j]);
            values(next.x[j], at.n(j), at.d, x[j]);
            values(next.dh[j], at.n(j), at.d, dh[j]);
        }
        load(row + at.step, next);
        __builtin_amdgcn_sched_barrier(0);  // the next row's loads stay ahead of this one's work
        // own: h's mean and squares about it in this wave, sum g m, sum g m (h - mean), x's first two, columns
        float own[7] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, at.count};
        if (layer) {
            own[0] = wave_sum(at.total(h)) / at.count;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
#pragma unroll
                for (int k = 0; k < 8; ++k) h[j][k] -= own[0];
                at.clip(j, h[j]);
            }
        }
        if (post_layer) {
            own[4] = wave_sum(at.total(x)) / at.count;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
#pragma unroll
                for (int k = 0; k < 8; ++k) x[j][k] -= own[4];
                at.clip(j, x[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 8; ++k) {  // (dy is zero past the row's end)
                const float gm = g[j][k] * m[j][k];
                s_dy[j][k] += g[j][k];
                t[0] = fmaf(h[j][k], h[j][k], t[0]);
                t[1] += gm;
                t[2] = fmaf(gm, h[j][k], t[2]);
                if (POST) t[3] = fmaf(x[j][k], x[j][k], t[3]);
            }
            at.add(j, t[0], own[1]);
            own[2] += t[1];
            own[3] += t[2];
            if (POST) at.add(j, t[3], own[5]);
        }
        own[1] = wave_sum(own[1]);
        if (layer) own[2] = wave_sum(own[2]);
        own[3] = wave_sum(own[3]);
        if (POST) own[5] = wave_sum(own[5]);
        float qh = own[1], G = own[2], gh = own[3], qx = own[5], rest = 0.f, xrest = 0.f;
        if (at.W > 1) {
            Slots& s = slots[2 * turn];
            publish(own, s[me]);
            float sh = 0.f, sx = 0.f;
            qh = G = gh = qx = 0.f;
            for (int w = 0; w < at.W; ++w) {
                const float* const o = s[at.team * at.W + w];
                sh = fmaf(o[0], o[6], sh);
                qh += o[1];
                G += o[2];
                gh += o[3];
                if (POST) {
                    sx = fmaf(o[4], o[6], sx);
                    qx += o[5];
                }
            }
            if (layer || post_layer) {
                const float mean = sh * at.inv_d, xmean = sx * at.inv_d;
                for (int w = 0; w < at.W; ++w) {
                    const float* const o = s[at.team * at.W + w];
                    const float off = o[0] - mean;
                    qh = fmaf(o[6] * off, off, qh);
                    gh = fmaf(off, o[2], gh);
                    if (POST) {
                        const float xoff = o[4] - xmean;
                        qx = fmaf(o[6] * xoff, xoff, qx);
                    }
                }
                rest = own[0] - mean;  // (0 without the layer norm: every wave's mean is 0)
                xrest = own[4] - xmean;
            }
        }
        // (a team past the end has zeros, and with eps 0 no factors)
        const float r = mine ? inverse_root(qh, at.inv_d, p.eps) : 0.f;
        const float rx = !POST ? 1.f : mine ? inverse_root(qx, at.inv_d, p.eps) : 0.f;
        float e[2] = {0.f, 0.f};
        Raw<S16> dres[NV];
        // D = dh + r (g m - mean(g m) - n mean(g m n)) = dh + r g m + a n + c
        const float a = -r * gh * r * at.inv_d, c = layer ? -r * G * at.inv_d : 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float D[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float n = (h[j][k] + rest) * r;
                s_dyn[j][k] = fmaf(g[j][k], n, s_dyn[j][k]);
                D[k] = fmaf(a, n, fmaf(r, g[j][k] * m[j][k], dh[j][k] + c));
                if (POST) x[j][k] = (x[j][k] + xrest) * rx;
                s_dx[j][k] = fmaf(D[k], x[j][k], s_dx[j][k]);
                g[j][k] = gp[j][k] * D[k];
            }
            if (POST) {
                at.clip(j, g[j]);
                float t[2] = {0.f, 0.f};
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    t[0] += g[j][k];
                    t[1] = fmaf(g[j][k], x[j][k], t[1]);
                }
                at.add(j, t[0], e[0]);
                at.add(j, t[1], e[1]);
            }
            dres[j] = packed<S16>(D);
        }
        if (POST) {
            if (post_layer) e[0] = wave_sum(e[0]);
            e[1] = wave_sum(e[1]);
            if (at.W > 1) {
                Slots& s = slots[2 * turn + 1];
                publish(e, s[me]);
                e[0] = e[1] = 0.f;
                for (int w = 0; w < at.W; ++w) {
                    e[0] += s[at.team * at.W + w][0];
                    e[1] += s[at.team * at.W + w][1];
                }
            }
            const float m0 = post_layer ? e[0] * at.inv_d : 0.f, m1 = e[1] * at.inv_d;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
#pragma unroll
                for (int k = 0; k < 8; ++k) g[j][k] = rx * (g[j][k] - m0 - x[j][k] * m1);
            }
        }
        next.settle();  // before the stores, as in the forward kernel
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (!mine || !at.any(j)) continue;
            const int64_t i = row * p.d + at.col[j];
            if (p.dresidual) store_raw<S16>(p.dresidual, i, at.n(j), dres[j]);
            if (p.dx) store_raw<X16>(p.dx, i, at.n(j), packed<X16>(g[j]));
        }
    }
    // the teams' sums, in order
    float* const out = p.partial + (int64_t)blockIdx.x * 3 * p.d;
    auto put = [&](int which, const float (&s)[NV][8]) {
        if (at.R == 1) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (at.any(j)) store_raw<false>(out, which * p.d + at.col[j], at.n(j), packed<false>(s[j]));
            return;
        }
        const int stride = 512 * NV * at.W;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int k = 0; k < 8; ++k) meet[at.team * stride + at.col[j] + k] = s[j][k];
        __syncthreads();
        for (int i = threadIdx.x; i < d; i += blockDim.x) {
            float v = 0.f;
            for (int w = 0; w < at.R; ++w) v += meet[w * stride + i];
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

// How a call's rows are dealt out: vectors of eight a lane, waves that share a row, rows a workgroup works on
// at once, workgroups of a batch.
struct Shape {
    int vectors, waves, teams;
    int64_t chunks;
};

// most: vectors a lane may have; even: one, where two would leave lanes without one; fit: workgroups' waves that a CU holds at once; team_waves: of a workgroup, where
// a row needs no more.
Shape shape_of(int64_t d, int64_t rows, int64_t batches, int most, bool even, int fit, int team_waves) {
    const int64_t vecs = (d + 7) / 8;
    Shape s{};
    s.waves = (int)((vecs + 64 * most - 1) / (64 * most));
    if (even && 2 * s.waves > (vecs + 63) / 64 && vecs <= 64 * 8) s.waves = (int)((vecs + 63) / 64);
    s.vectors = (int)((vecs + 64 * s.waves - 1) / (64 * s.waves));
    s.teams = std::max(1, team_waves / s.waves);
    const int64_t groups = std::max<int64_t>(1, 256 * std::max(1, fit / (s.waves * s.teams)) / batches);
    s.chunks = std::max<int64_t>(1, std::min<int64_t>(groups, (rows + s.teams - 1) / s.teams));
    return s;
}

// Measured, us.  Forward, vectors a lane and waves on a CU, 4608 x 3072 and 8190 x 1155 (both norms, fp32
// stream): 1, 16 25.0, 27.4; 1, 20 30.1, 32.9; 2, 12 22.6, 28.3; 2, 16 22.9, 27.3 (1155 columns take one vector either
// way).  A wave's own work a row (its sums, their exchange) is the same for two vectors as for one, and past what
// the registers let a CU hold at once the workgroups come in rounds.  Gradients, vectors, waves on a CU and of a
// workgroup, 18432 x 1152 and 4096 x 2240 (both norms, fp32 stream): 1, 12, 4 65.6, 60.0; 1, 16, 4 63.5, 63.3; 2, 8, 8
// 66.3, 50.0; 2, 8, 4 61.5, 46.5: every workgroup leaves three sums a column for norm_grad_kernel.
constexpr int kForwardMost = 2, kForwardFit = 12, kForwardTeam = 1;
constexpr int kBackwardMost = 2, kBackwardFit = 8, kBackwardTeam = 4;

Shape forward_shape(int64_t d, int64_t rows, int64_t batches) {
    const bool few = rows * batches <= 256 && d <= 512 * kMaxWaves;
    return shape_of(d, rows, batches, few ? 1 : kForwardMost, true, kForwardFit, kForwardTeam);
}
Shape backward_shape(int64_t d, int64_t rows, int64_t batches) {
    return shape_of(d, rows, batches, kBackwardMost, false, kBackwardFit, kBackwardTeam);
}

void deal(NormParams& p, const Shape& s) {
    p.waves = s.waves;
    p.teams = s.teams;
    p.chunks = s.chunks;
}

// f(X16, S16, WHOLE) as integral constants.
template <class F>
void by_type(const NormParams& p, F f) {
    auto with_whole = [&](auto x, auto s) {
        if (p.d % 8 == 0) f(x, s, std::true_type{});
        else f(x, s, std::false_type{});
    };
    if (p.x16) p.stream16 ? with_whole(std::true_type{}, std::true_type{}) : with_whole(std::true_type{}, std::false_type{});
    else p.stream16 ? with_whole(std::false_type{}, std::true_type{}) : with_whole(std::false_type{}, std::false_type{});
}

}  // namespace

int64_t norm_chunks(int64_t M, int64_t batches, int64_t d) { return backward_shape(d, M / batches, batches).chunks; }

hipError_t launch_block_norm(NormParams p, hipStream_t st) {
    const Shape s = forward_shape(p.d, p.rows, p.batches);
    deal(p, s);
    const dim3 grid((unsigned)(p.batches * p.chunks)), block(64 * s.waves * s.teams);
    by_type(p, [&](auto x, auto h, auto whole) {
#define KQ_NORM(NV, THREADS)                                                                                                   \
    hipLaunchKernelGGL((block_norm_kernel<decltype(x)::value, decltype(h)::value, decltype(whole)::value, NV, THREADS>), grid, \
                       block, 0, st, p)
        if (s.vectors == 1) KQ_NORM(1, 1024);
        else if (s.waves <= 8) KQ_NORM(2, 512);
        else KQ_NORM(2, 1024);
#undef KQ_NORM
    });
    return hipGetLastError();
}

hipError_t launch_block_norm_backward(NormParams p, hipStream_t st) {
    const Shape s = backward_shape(p.d, p.rows, p.batches);
    deal(p, s);
    const dim3 groups((unsigned)(p.batches * p.chunks)), block(64 * s.waves * s.teams);
    by_type(p, [&](auto x, auto h, auto whole) {
#define KQ_NORM(POST, NV, THREADS)                                                                                                   \
    hipLaunchKernelGGL((block_norm_backward_kernel<decltype(x)::value, decltype(h)::value, POST, decltype(whole)::value, NV, THREADS>), \
                       groups, block, 0, st, p)
#define KQ_NORM_POST(NV, THREADS)              \
    do {                                       \
        if (p.post) KQ_NORM(true, NV, THREADS); \
        else KQ_NORM(false, NV, THREADS);       \
    } while (0)
        if (s.vectors == 1) KQ_NORM_POST(1, 512);
        else if (s.waves <= 8) KQ_NORM_POST(2, 512);
        else KQ_NORM_POST(2, 1024);
#undef KQ_NORM_POST
#undef KQ_NORM
    });
    hipError_t e = hipGetLastError();
    const bool grads = p.dgate || p.dscale || p.dshift, weights = p.dweight || p.dpost_weight;
    if (e != hipSuccess || (!grads && !weights)) return e;
    const dim3 grid((unsigned)((p.d + 31) / 32), (unsigned)(p.batches + (weights ? 1 : 0)));
    hipLaunchKernelGGL(norm_grad_kernel, grid, dim3(1024), 0, st, p);
    return hipGetLastError();
}

}  // namespace kq
