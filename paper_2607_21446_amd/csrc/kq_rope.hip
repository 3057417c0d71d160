// Rotary positions with one to four axes, and their gradient.  Pair p of a row
// (x_a, x_b) belongs to an axis with position t and turns by t f_p:
//     y_a = x_a cos - x_b sin,   y_b = x_b cos + x_a sin;
// the gradient is the rotation back.  Angles, their sines and cosines are in
// 64 bits: a position of 10^6 at f = 1 keeps 2^-33 of a radian, where 32 bits
// keep 2^-4.  The rotation is in 32 bits.
//
// A workgroup makes the sines of its tokens once, in LDS, and its heads share
// them.  Bound by HBM, an element is read and written once: 4608 x 48 x 128 in
// bf16 22.7 us, 18000 x 16 x 72 in fp32 31.9 us, 5.0 and 5.2 TB/s; one token by
// a launch's and its loads' latencies (2.5 us).  Rows that go a pair a step (see
// the launch) are bound by their small accesses: 48.8 us for the second size
// with axes of 18.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "kq_serve.h"

namespace kq {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeTableBytes = 32768;

// cos and sin of z, |z| <= pi / 4, by their power series in 64 bits: what they leave out is below 2^-41 of them.  Rounded
// once.  (In 32 bits, from an angle rounded to 32 bits, they were off by up to 1.5 of the last place, in the same time.)
__device__ __forceinline__ void sincos_small(double z, float* s, float* c) {
    const double w = z * z;
    double a = fma(w, 1.0 / 6227020800.0, -1.0 / 39916800.0);
    a = fma(w, a, 1.0 / 362880.0);
    a = fma(w, a, -1.0 / 5040.0);
    a = fma(w, a, 1.0 / 120.0);
    a = fma(w, a, -1.0 / 6.0);
    *s = (float)fma(z * w, a, z);
    double b = fma(w, 1.0 / 479001600.0, -1.0 / 3628800.0);
    b = fma(w, b, 1.0 / 40320.0);
    b = fma(w, b, -1.0 / 720.0);
    b = fma(w, b, 1.0 / 24.0);
    b = fma(w, b, -0.5);
    *c = (float)fma(w, b, 1.0);
}

// Pair p's axis, and its frequency in quarter turns a position.
__device__ __forceinline__ double quarter_turns(const RopeParams& p, int pair, int* axis) {
    constexpr double kQuarter = 0.63661977236758134308;  // 2 / pi
    int a = 0, from = 0;
    while (a + 1 < p.axes && pair >= p.end[a]) from = p.end[a++];
    *axis = a;
    if (p.freqs) return p.freqs[pair] * kQuarter;
    const int n = p.end[a] - from;  // theta^(-2i / d) with d = 2n
    return exp2(-(double)(pair - from) / n * p.log2_theta) * kQuarter;
}

__device__ __forceinline__ double position(const RopeParams& p, int64_t at) {
    switch (p.pos_type) {
        case Position::Int32: return static_cast<const int32_t*>(p.positions)[at];
        case Position::Int64: return (double)static_cast<const int64_t*>(p.positions)[at];
        case Position::Fp32: break;
    }
    return static_cast<const float*>(p.positions)[at];
}

// N elements as they are stored, A bytes aligned.
template <bool B16, int N, int A>
struct Row;
template <int N, int A>
struct Row<true, N, A> {
    typedef uint16_t E;
    typedef uint16_t V __attribute__((ext_vector_type(N), aligned(A)));
    static __device__ __forceinline__ float value(uint16_t e) { return __uint_as_float((uint32_t)e << 16); }
    static __device__ __forceinline__ uint16_t stored(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
};
template <int N, int A>
struct Row<false, N, A> {
    typedef float E;
    typedef float V __attribute__((ext_vector_type(N), aligned(A)));
    static __device__ __forceinline__ float value(float e) { return e; }
    static __device__ __forceinline__ float stored(float f) { return f; }
};

// U pairs a step: 2 U elements side by side, or U and U.  With U = 1 rows are aligned to their elements only.
// Eight waves a SIMD: the sines' constants take registers for six, and 18000 x 16 x 72 in fp32 with axes of 18 took 65 us for 47.
template <bool B16, int U, bool HALVES>
__global__ __launch_bounds__(kRopeThreads, 8) void rope_kernel(RopeParams p) {
    constexpr int kSize = B16 ? 2 : 4;
    constexpr int kAlign = U == 1 ? kSize : U * kSize < 16 ? U * kSize : 16;
    typedef Row<B16, HALVES ? U : 2 * U, kAlign> R;
    typedef typename R::E E;
    typedef typename R::V V;
    extern __shared__ float2 table[];  // [tokens, pairs]: cos, sin
    const int pairs = p.end[p.axes - 1], t0n = p.tokens;
    const int64_t t0 = (int64_t)blockIdx.x * t0n;
    const int nt = (int)min((int64_t)t0n, p.T - t0);
    const int h0 = (int)(blockIdx.y * p.heads), nh = min((int)p.heads, p.H - h0);
    for (int i = threadIdx.x; i < nt * pairs; i += kRopeThreads) {
        const int t = i / pairs, pair = i - t * pairs;
        int axis;
        const double f = quarter_turns(p, pair, &axis);
        const double turns = position(p, (t0 + t) * p.pos_stride + axis) * f;
        const double whole = rint(turns);
        float s, c;
        sincos_small((turns - whole) * 1.57079632679489661923, &s, &c);
        const int q = (int)(whole - 4.0 * floor(whole * 0.25));  // 0 .. 3
        const float u = q & 1 ? s : c, w = q & 1 ? c : s;
        const float cs = q == 1 || q == 2 ? -u : u, sn = q >= 2 ? -w : w;
        table[i] = make_float2(cs, p.backward ? -sn : sn);
    }
    __syncthreads();
    const int steps = p.D / 2 / U;  // of a row: pairs / U turn, the rest go through
    const int turning = pairs / U, all = nt * nh * steps;
    const bool over = p.x == p.y && p.x_token == p.y_token && p.x_head == p.y_head;
    for (int i = threadIdx.x; i < all; i += kRopeThreads) {
        const int row = i / steps, u = i - row * steps, t = row / nh, h = h0 + row - t * nh;
        const E* const x = static_cast<const E*>(p.x) + (t0 + t) * p.x_token + h * p.x_head;
        E* const y = static_cast<E*>(p.y) + (t0 + t) * p.y_token + h * p.y_head;
        if (u >= turning) {
            if (over) continue;
            const int at = 2 * U * u;
            typedef typename Row<B16, 2 * U, kAlign>::V W;
            *reinterpret_cast<W*>(y + at) = *reinterpret_cast<const W*>(x + at);
            continue;
        }
        const float2* const cs = table + t * pairs + u * U;
        if constexpr (HALVES) {
            V a = *reinterpret_cast<const V*>(x + U * u), b = *reinterpret_cast<const V*>(x + pairs + U * u);
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const float f = R::value(a[k]), g = R::value(b[k]);
                a[k] = R::stored(fmaf(f, cs[k].x, -(g * cs[k].y)));
                b[k] = R::stored(fmaf(g, cs[k].x, f * cs[k].y));
            }
            *reinterpret_cast<V*>(y + U * u) = a;
            *reinterpret_cast<V*>(y + pairs + U * u) = b;
        } else {
            V a = *reinterpret_cast<const V*>(x + 2 * U * u);
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const float f = R::value(a[2 * k]), g = R::value(a[2 * k + 1]);
                a[2 * k] = R::stored(fmaf(f, cs[k].x, -(g * cs[k].y)));
                a[2 * k + 1] = R::stored(fmaf(g, cs[k].x, f * cs[k].y));
            }
            *reinterpret_cast<V*>(y + 2 * U * u) = a;
        }
    }
}

// Rows start at multiples of 16 bytes.
bool aligned_rows(const RopeParams& p) {
    const uint64_t all = (uint64_t)p.x_token | p.x_head | p.y_token | p.y_head;
    return ((uintptr_t)p.x | (uintptr_t)p.y) % 16 == 0 && all % (p.is16 ? 8 : 4) == 0;
}

template <bool B16, int U>
void launch_rope_of(const RopeParams& p, dim3 grid, size_t lds, hipStream_t st) {
    if (p.halves) rope_kernel<B16, U, true><<<grid, kRopeThreads, lds, st>>>(p);
    else rope_kernel<B16, U, false><<<grid, kRopeThreads, lds, st>>>(p);
}

}  // namespace

hipError_t launch_rope(RopeParams p, hipStream_t st) {
    const int pairs = p.end[p.axes - 1], rest = p.D / 2 - pairs;
    // sines are made by all threads, and by few workgroups for the same token, as long as there are workgroups enough
    p.tokens = std::max(1, std::min(kRopeThreads / std::max(pairs, 1), kRopeTableBytes / (8 * std::max(pairs, 1))));
    while (p.tokens > 1 && ((p.T + p.tokens - 1) / p.tokens < 1024 || (int64_t)p.tokens * p.H * p.D > (1 << 26))) p.tokens /= 2;
    p.heads = p.H;
    const int64_t along = (p.T + p.tokens - 1) / p.tokens;
    if (along < 512) {  // a workgroup's threads a step each at least
        const int64_t least = std::max<int64_t>(1, 8 * kRopeThreads / p.D);
        p.heads = std::max<int64_t>(least, (p.H * along + 511) / 512);
    }
    p.heads = std::min<int64_t>(p.heads, p.H);
    const unsigned across = (unsigned)((p.H + p.heads - 1) / p.heads);
    const size_t lds = std::max<size_t>(8, (size_t)p.tokens * pairs * 8);
    // Four pairs a step where rows start at multiples of 16 bytes, and the pairs that turn and the rest are multiples of four:
    // one pair a step takes 47 and 39 us for the calls above.
    const bool wide = pairs % 4 == 0 && rest % 4 == 0 && aligned_rows(p);
    const int size = p.is16 ? 2 : 4, pos_size = p.pos_type == Position::Int64 ? 8 : 4;
    in_launches(p.T, p.tokens, kRopeThreads, [&](int64_t from, int64_t n) {
        RopeParams l = p;
        l.T = n;
        l.x = static_cast<const uint8_t*>(p.x) + from * p.x_token * size;
        l.y = static_cast<uint8_t*>(p.y) + from * p.y_token * size;
        l.positions = static_cast<const uint8_t*>(p.positions) + from * p.pos_stride * pos_size;
        const dim3 grid((unsigned)((n + p.tokens - 1) / p.tokens), across);
        if (p.is16) {
            if (wide) launch_rope_of<true, 4>(l, grid, lds, st);
            else launch_rope_of<true, 1>(l, grid, lds, st);
        } else {
            if (wide) launch_rope_of<false, 4>(l, grid, lds, st);
            else launch_rope_of<false, 1>(l, grid, lds, st);
        }
    });
    return hipGetLastError();
}

}  // namespace kq
