// W4A16 linear layers: a few rows of 16- or 32-bit activations and an MXFP4
// weight,
//     out = residual + gate act(x deq(B)^T + bias).
// The weight's values are exact in bf16, so the product runs on the bf16 matrix
// cores with the weight as operand A: 16 of its rows x 32 columns, lane (r, g) =
// row r (r = lane % 16, g = lane / 16), x's rows as operand B.  The order of
// columns in the sum is free: a lane takes the 16 bytes of a block of 32 of its
// row, which has one scale.  x in 32 bits goes in as three bf16 terms (8 + 8 + 8
// bits: exact).
//
// Bound by the weight's read where that is 25 MB and more (one bf16 row through
// 4096 x 12288: 7.5 us, 3.6 TB/s), by a launch's and its loads' latencies below it
// (4096 x 4096: 4.6 us), and with 16 rows in 32 bits by LDS (below).  Three forms,
// by what x takes:
//   narrow    K below 2048: a workgroup's waves take the columns of 16 rows in
//             turn, x as the operands need it; also whatever fits no other form,
//             which is every call of more than 16 rows: the weight is read for
//             each 16 of them, a row a lane (12288 x 12288 in bf16: 16 rows 25 us
//             in slices, 17 76, 32 99, 64 194);
//   resident  all of x's rows (16 at most) fit in LDS: as above with x in LDS,
//             as terms, and the weight's loads 64 bytes a row;
//   slices    they do not: workgroups take 512 columns of many rows of the
//             weight, x's slice in LDS, and a second launch adds the slices' sums.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "kq_act.h"
#include "kq_mx.h"
#include "kq_serve.h"

namespace kq {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4e __attribute__((ext_vector_type(4), aligned(2)));  // at any alignment of the elements

#define KQ_INLINE __attribute__((always_inline))

constexpr int kVecRows = 16;   // of a workgroup, of the weight and of x
constexpr int kVecWaves = 8;   // of a workgroup
constexpr int kStepBlocks = 4;    // of a wave's step: 128 columns
constexpr int kSliceBlocks = 16;  // of a slice: 512 columns
constexpr int kSumThreads = 64;   // of the slices' second launch
constexpr int kAhead = 2;           // steps that a wave has loaded or is loading
// LDS of x's rows.  (16 bf16 rows of 4096: 6.0 us resident, 8.2 in slices; one fp32 row of 12288: 9.7 and 14.8.)
constexpr int kResidentBytes = 136 << 10;
constexpr int kResidentColumns = 2048;  // from here on: one row through 1152 x 1152 takes 3.1 us resident, 2.7 narrow

template <int I, int N, class Fn>
__device__ __forceinline__ void unrolled(Fn f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        unrolled<I + 1, N>(f);
    }
}

template <bool X16>
constexpr int kTerms = X16 ? 1 : 3;

// Eight values in 32 bits as three bf16 operands whose sum they are.
__device__ __forceinline__ void three_terms(float (&f)[8], u32x4v (&t)[3]) {
#pragma unroll
    for (int n = 0; n < 3; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            t[n][i] = __builtin_amdgcn_perm(__float_as_uint(f[2 * i + 1]), __float_as_uint(f[2 * i]), 0x07060302u);
            f[2 * i] -= bf16_low(t[n][i]);
            f[2 * i + 1] -= bf16_high(t[n][i]);
        }
}
// Eight values of x as operands.
template <bool X16>
__device__ __forceinline__ void load_terms(const uint8_t* p, u32x4v (&t)[kTerms<X16>]) {
    const u32x4v a = u32x4v(*reinterpret_cast<const u32x4e*>(p));
    if constexpr (X16) {
        t[0] = a;
    } else {
        const u32x4v b = u32x4v(*reinterpret_cast<const u32x4e*>(p + 16));
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i] = __uint_as_float(a[i]);
            f[4 + i] = __uint_as_float(b[i]);
        }
        three_terms(f, t);
    }
}

// Eight codes as an operand.
__device__ __forceinline__ bf16x8 weight_operand(uint32_t c, float scale) {
    return __builtin_bit_cast(
        bf16x8, u32x4v{e2m1_pair<0>(c, scale), e2m1_pair<1>(c, scale), e2m1_pair<2>(c, scale), e2m1_pair<3>(c, scale)});
}

// What the epilogue of an element (of two of the weight's rows with Swiglu) reads beside the sums, as stored.  Loaded before
// the sums are made.
struct Beside {
    uint32_t bias[2], gate, residual;
    static __device__ __forceinline__ uint32_t at(const void* p, int is16, int64_t i) {
        return is16 ? static_cast<const uint16_t*>(p)[i] : static_cast<const uint32_t*>(p)[i];
    }
    static __device__ __forceinline__ float value(uint32_t v, int is16) { return __uint_as_float(is16 ? v << 16 : v); }
    // Of row m of x and row n of the weight (n even with Swiglu).
    __device__ __forceinline__ void load(const LinearParams& l, int64_t m, int64_t n) {
        const bool two = l.act == Act::Swiglu;
        if (l.bias) {
            bias[0] = at(l.bias, l.vec16, n);
            if (two) bias[1] = at(l.bias, l.vec16, n + 1);
        }
        if (two) n >>= 1;
        if (l.gate) gate = at(l.gate, l.vec16, m / l.gate_rows * l.gate_stride + n);
        if (l.residual) residual = at(l.residual, l.out16, m * l.ldr + n);
    }
};

// The result of the sums of row m of x and row n (and n + 1 with Swiglu, n even) of the weight.
template <Act A>
__device__ __forceinline__ void finish(const LinearParams& l, int64_t m, int64_t n, float v, float u, const Beside& e) {
    if (l.bias) v += Beside::value(e.bias[0], l.vec16);
    float y = activate<A>(v);
    if constexpr (A == Act::Swiglu) {
        if (l.bias) u += Beside::value(e.bias[1], l.vec16);
        y *= u;
        n >>= 1;
    }
    if (l.gate) y *= Beside::value(e.gate, l.vec16);
    if (l.residual) y += Beside::value(e.residual, l.out16);
    const int64_t at = m * l.ldo + n;
    if (l.out16) static_cast<__bf16*>(l.out)[at] = (__bf16)y;
    else static_cast<float*>(l.out)[at] = y;
}

// A thread's element of a tile's result: row m of x, row n of the weight; none where m is negative.
struct TilePlace {
    int64_t m = -1, n = 0;
    Beside beside;
    __device__ __forceinline__ TilePlace(const LinearParams& l, int64_t m0, int64_t n0) {
        const int wide = l.act == Act::Swiglu ? 2 : 1, out = kVecRows / wide, i = threadIdx.x;
        const int64_t row = m0 + i / out, column = n0 + wide * (i % out);
        if (i >= kVecRows * out || row >= l.g.M || column >= l.g.N) return;
        m = row;
        n = column;
        beside.load(l, m, n);
    }
};

// The waves' sums of a tile in one, and its epilogue.
__device__ __forceinline__ void finish_tile(const LinearParams& l, int64_t m0, int64_t n0, const f32x4& acc, const TilePlace& at) {
    __shared__ float sums[kVecWaves][kVecRows][kVecRows + 1];  // [wave][row of x][row of the weight]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int k = 0; k < 4; ++k) sums[wave][lane & 15][4 * (lane >> 4) + k] = acc[k];
    __syncthreads();
    if (at.m < 0) return;
    with_act(l.act, [&](auto a) KQ_INLINE {
        constexpr Act A = decltype(a)::value;
        const int m = (int)(at.m - m0), n = (int)(at.n - n0);
        float v[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < (A == Act::Swiglu ? 2 : 1); ++j)
#pragma unroll
            for (int w = 0; w < kVecWaves; ++w) v[j] += sums[w][m][n + j];
        finish<A>(l, at.m, at.n, v[0], v[1], at.beside);
    });
}

// ------------------------------------------------------------ narrow

// A lane's block of the weight and of x.
template <bool X16>
struct Block {
    static constexpr int kBytes = X16 ? 16 : 32;  // of eight values
    u32x4v w;
    uint32_t s;
    u32x4v x[4][X16 ? 1 : 2];
    __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, const uint8_t* row, int b, bool in, bool live) {
        w = u32x4v{0u, 0u, 0u, 0u};
        s = 127u;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < (X16 ? 1 : 2); ++i) x[k][i] = u32x4v{0u, 0u, 0u, 0u};
        if (!in) return;
        w = *reinterpret_cast<const u32x4v*>(codes + 16 * (int64_t)b);
        s = scales[b];
        if (!live) return;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < (X16 ? 1 : 2); ++i)
                x[k][i] = u32x4v(*reinterpret_cast<const u32x4e*>(row + (4 * (int64_t)b + k) * kBytes + 16 * i));
    }
    __device__ __forceinline__ void add(f32x4& acc) const {
        const float sc = mx_scale(s);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bf16x8 a = weight_operand(w[k], sc);
            u32x4v t[kTerms<X16>];
            if constexpr (X16) {
                t[0] = x[k][0];
            } else {
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(x[k][i / 4][i % 4]);
                three_terms(f, t);
            }
#pragma unroll
            for (int n = 0; n < kTerms<X16>; ++n) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, t[n]), acc, 0, 0, 0);
        }
    }
};

template <bool X16>
__global__ __launch_bounds__(64 * kVecWaves) void matvec_narrow_kernel(MatvecParams p) {
    const LinearParams& l = p.l;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * kVecRows, m0 = (int64_t)blockIdx.y * kVecRows, row = min(n0 + r, l.g.N - 1);
    const int blocks = (int)(l.g.K / 32);
    const uint8_t* const codes = l.g.b_codes + row * (l.g.K / 2);
    const uint8_t* const scales = l.g.b_scales + row * blocks;
    const bool live = m0 + r < l.g.M;
    const uint8_t* const xrow = static_cast<const uint8_t*>(p.x) + (live ? m0 + r : 0) * p.ldx * (X16 ? 2 : 4);
    constexpr int kStep = 4 * kVecWaves;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    Block<X16> a, b;  // one is worked on while the other is in flight
    int at = 4 * wave;
    if (at < blocks) a.load(codes, scales, xrow, at + g, at + g < blocks, live);
    const TilePlace place(l, m0, n0);
    while (at < blocks) {
        const int next = at + kStep, after = next + kStep;
        if (next < blocks) b.load(codes, scales, xrow, next + g, next + g < blocks, live);
        a.add(acc);
        if (next >= blocks) break;
        if (after < blocks) a.load(codes, scales, xrow, after + g, after + g < blocks, live);
        b.add(acc);
        at = after;
    }
    finish_tile(l, m0, n0, acc, place);
}

// ------------------------------------------------------------ x in LDS

// A step of a wave: four blocks of 16 of the weight's rows.  Four neighbouring lanes read a row's 64 bytes, and an exchange
// gives lane (r, g) its own row's block g.  (A row a lane, as the operand needs it, costs the cache an access for every lane:
// 16 bf16 rows and a weight of 12288 x 12288 took 49 us so.)
struct Step {
    u32x4v w;
    uint32_t s;
    // codes, scales: of the row lane / 4; b0: the first block.  Blocks past the last are read as the last (and dropped later).
    __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, int b0, int blocks) {
        const int b = min(b0 + (int)(threadIdx.x & 3), blocks - 1);
        w = *reinterpret_cast<const u32x4v*>(codes + 16 * (int64_t)b);
        s = scales[b];
    }
    __device__ __forceinline__ void settle() {
        const int from = (16 * (int)(threadIdx.x & 15) + 4 * ((int)(threadIdx.x & 63) >> 4));  // four times the lane
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)w[i]);
        s = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)s);
    }
};

// x's rows in LDS as terms: row r's block b of `blocks` from r stride + b terms 64 on, a block's terms one after another.
// Rows are 16 bytes more than a multiple of 128 apart, so that eight lanes' rows lie in different banks.
template <bool X16>
__device__ __forceinline__ int lds_stride(int blocks) {
    return blocks * kTerms<X16> * 64 + 16 + (blocks * kTerms<X16> & 1) * 64;
}
// Blocks b0 .. b0 + blocks - 1 of `rows` rows.
template <bool X16>
__device__ __forceinline__ void stage_rows(uint8_t* xs, int stride, const uint8_t* x, int64_t row_bytes, int rows, int b0, int blocks) {
    const int each = 4 * blocks, all = rows * each;  // eights of values
    constexpr int kBytes = X16 ? 16 : 32, kAtOnce = X16 ? 4 : 2;
    for (int i = threadIdx.x; i < all; i += kAtOnce * 64 * kVecWaves) {
        u32x4v t[kAtOnce][kTerms<X16>];
        int to[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int at = min(i + j * 64 * kVecWaves, all - 1), row = at / each, e = at - row * each;
            load_terms<X16>(x + row * row_bytes + ((int64_t)b0 * 4 + e) * kBytes, t[j]);
            to[j] = row * stride + (e >> 2) * (kTerms<X16> * 64) + (e & 3) * 16;
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
            for (int n = 0; n < kTerms<X16>; ++n) *reinterpret_cast<u32x4v*>(xs + to[j] + 64 * n) = t[j][n];
    }
}

// A step's products in two sums: lane (r, g)'s block g of the weight, of which `left` exist, with x's at `from`.
template <bool X16>
__device__ __forceinline__ void add_step(f32x4 (&acc)[2], Step& w, const uint8_t* from, int left) {
    u32x4v t[4][kTerms<X16>];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int n = 0; n < kTerms<X16>; ++n) t[k][n] = *reinterpret_cast<const u32x4v*>(from + n * 64 + 16 * k);
    w.settle();
    if (left < kStepBlocks) {
        asm volatile("");  // a branch: the last step only
        const bool in = (int)((threadIdx.x & 63) >> 4) < left;
        w.s = in ? w.s : 127u;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            w.w[k] = in ? w.w[k] : 0u;
#pragma unroll
            for (int n = 0; n < kTerms<X16>; ++n) t[k][n] = in ? t[k][n] : u32x4v{0u, 0u, 0u, 0u};
        }
    }
    const float sc = mx_scale(w.s);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const bf16x8 a = weight_operand(w.w[k], sc);
#pragma unroll
        for (int n = 0; n < kTerms<X16>; ++n)
            acc[k & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, t[k][n]), acc[k & 1], 0, 0, 0);
    }
}

template <bool X16>
__global__ __launch_bounds__(64 * kVecWaves) void matvec_resident_kernel(MatvecParams p) {
    extern __shared__ uint8_t xs[];
    const LinearParams& l = p.l;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * kVecRows, row = min(n0 + (lane >> 2), l.g.N - 1);
    const int blocks = (int)(l.g.K / 32), rows = (int)l.g.M, stride = lds_stride<X16>(blocks);
    const uint8_t* const codes = l.g.b_codes + row * (l.g.K / 2);
    const uint8_t* const scales = l.g.b_scales + row * blocks;
    constexpr int kStep = kStepBlocks * kVecWaves;
    f32x4 acc[2] = {};
    Step w[kAhead];
    int b0 = kStepBlocks * wave;
    unrolled<0, kAhead - 1>([&](auto stage) KQ_INLINE {
        if (b0 + stage * kStep < blocks) w[stage].load(codes, scales, b0 + stage * kStep, blocks);
    });
    stage_rows<X16>(xs, stride, static_cast<const uint8_t*>(p.x), p.ldx * (X16 ? 2 : 4), rows, 0, blocks);
    const TilePlace place(l, 0, n0);
    __syncthreads();
    const uint8_t* const mine = xs + min(r, rows - 1) * stride + g * (kTerms<X16> * 64);
    while (b0 < blocks) {
        bool more = true;
        unrolled<0, kAhead>([&](auto stage) KQ_INLINE {
            constexpr int now = stage, late = (stage + kAhead - 1) % kAhead;
            if (!more) return;
            const int at = b0 + (kAhead - 1) * kStep;
            if (at < blocks) w[late].load(codes, scales, at, blocks);
            add_step<X16>(acc, w[now], mine + b0 * (kTerms<X16> * 64), blocks - b0);
            b0 += kStep;
            more = b0 < blocks;
        });
    }
    finish_tile(l, 0, n0, acc[0] + acc[1], place);
}

// ------------------------------------------------------------ slices

// Word i of lane q of every four lanes becomes word q of lane i.
__device__ __forceinline__ void quad_transpose(uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d) {
    const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
    auto from1 = [](uint32_t v) KQ_INLINE { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true); };  // lane ^ 1
    auto from2 = [](uint32_t v) KQ_INLINE { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true); };  // lane ^ 2
    // (exchanges first: every lane takes part in them)
    const uint32_t fa = from1(a), fb = from1(b), fc = from1(c), fd = from1(d);
    const uint32_t a1 = odd ? fb : a, b1 = odd ? b : fa, c1 = odd ? fd : c, d1 = odd ? d : fc;
    const uint32_t ga = from2(a1), gb = from2(b1), gc = from2(c1), gd = from2(d1);
    a = high ? gc : a1;
    c = high ? c1 : ga;
    b = high ? gd : b1;
    d = high ? d1 : gb;
}

// A slice of 16 of the weight's rows: 16 blocks, four side by side a lane.  Loads as for a step, 64 bytes of a row by four
// neighbouring lanes: lane 4 i + q reads the block q + 4 (i / 4) of row 4 (i % 4) + k in load k, and the transpose of the four
// loads gives lane (r, g) its own row's blocks 4 g .. 4 g + 3.  (LDS is what this form waits for, x's 48 KB a tile in 32 bits:
// both launches took 16.7 us with a step's exchange, 15.8 with this one.)
struct Run {
    u32x4v w[4];  // after `settle`: block 4 g + k of row r
    uint32_t s;   // their scales
    // b0: the first block of 16, of which those before `blocks` exist; others are read as the last (and dropped later)
    __device__ __forceinline__ void load(const uint8_t* const (&codes)[4], const uint8_t* scales, int b0, int blocks) {
        const int lane = threadIdx.x & 63, mine = min(b0 + (lane & 3) + 4 * (lane >> 4), blocks - 1), own = b0 + 4 * (lane >> 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = *reinterpret_cast<const u32x4v*>(codes[k] + 16 * (int64_t)mine);
        if (b0 + 16 <= blocks) {
            typedef uint32_t W __attribute__((aligned(1)));
            s = *reinterpret_cast<const W*>(scales + own);
        } else {
            s = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) s |= (uint32_t)scales[min(own + k, blocks - 1)] << (8 * k);
        }
    }
    __device__ __forceinline__ void settle() {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t a = w[0][i], b = w[1][i], c = w[2][i], d = w[3][i];
            quad_transpose(a, b, c, d);
            w[0][i] = a;
            w[1][i] = b;
            w[2][i] = c;
            w[3][i] = d;
        }
    }
};

// A run's products in two sums: lane (r, g)'s blocks 4 g .. 4 g + 3 of the weight, those before `left` existing, with x's
// at `from`.
template <bool X16>
__device__ __forceinline__ void add_run(f32x4 (&acc)[2], const Run& w, const uint8_t* from, int left) {
    unrolled<0, 4>([&](auto sub) KQ_INLINE {
        constexpr int S = sub;
        uint32_t c[4], s = w.s >> (8 * S) & 255u;
        u32x4v t[4][kTerms<X16>];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            c[k] = w.w[S][k];
#pragma unroll
            for (int n = 0; n < kTerms<X16>; ++n) t[k][n] = *reinterpret_cast<const u32x4v*>(from + (S * kTerms<X16> + n) * 64 + 16 * k);
        }
        if (left < kSliceBlocks) {
            asm volatile("");  // a branch: the last run only
            const bool in = 4 * (int)((threadIdx.x & 63) >> 4) + S < left;
            s = in ? s : 127u;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                c[k] = in ? c[k] : 0u;
#pragma unroll
                for (int n = 0; n < kTerms<X16>; ++n) t[k][n] = in ? t[k][n] : u32x4v{0u, 0u, 0u, 0u};
            }
        }
        const float sc = mx_scale(s);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bf16x8 a = weight_operand(c[k], sc);
#pragma unroll
            for (int n = 0; n < kTerms<X16>; ++n)
                acc[k & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, t[k][n]), acc[k & 1], 0, 0, 0);
        }
    });
}

// Where a lane's loads and its own row are in tile n0 of the weight.
struct WeightRows {
    const uint8_t *codes[4], *scales;
    __device__ __forceinline__ WeightRows(const GemmParams& g, int64_t n0) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int k = 0; k < 4; ++k) codes[k] = g.b_codes + min(n0 + 4 * (lane >> 2 & 3) + k, g.N - 1) * (g.K / 2);
        scales = g.b_scales + min(n0 + (lane & 15), g.N - 1) * (g.K / 32);
    }
};

// Slice blockIdx.y of the columns, for every gridDim.x-th eight tiles of the weight: a wave a tile.  16 rows in 32 bits through
// 12288 x 4096 take 12.7 us, the weight's 27 MB 5.3 of them, x's reads from LDS 3.8 at least; they do not overlap, since all
// workgroups are resident at once and do the same.  (Two tiles a wave, which share x's reads, leave two waves a SIMD and took
// 18 us for 16, both launches; x's loads issued before the weight's 16.8 for 15.9.)
template <bool X16>
__global__ __launch_bounds__(64 * kVecWaves) void matvec_slice_kernel(MatvecParams p) {
    extern __shared__ uint8_t xs[];
    const LinearParams& l = p.l;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int blocks = (int)(l.g.K / 32), rows = (int)l.g.M, b0 = kSliceBlocks * blockIdx.y, mine = min(blocks - b0, kSliceBlocks);
    constexpr int kStride = kSliceBlocks * kTerms<X16> * 64 + 16;
    const int64_t step = (int64_t)gridDim.x * kVecWaves * kVecRows;
    int64_t n0 = ((int64_t)blockIdx.x * kVecWaves + wave) * kVecRows;
    Run w, next;
    if (n0 < l.g.N) {
        const WeightRows at(l.g, n0);
        next.load(at.codes, at.scales, b0, blocks);
    }
    stage_rows<X16>(xs, kStride, static_cast<const uint8_t*>(p.x), p.ldx * (X16 ? 2 : 4), rows, b0, mine);
    __syncthreads();
    const uint8_t* const from = xs + min(r, rows - 1) * kStride + 4 * g * (kTerms<X16> * 64);
    float* const out = p.partial + ((int64_t)blockIdx.y * rows + r) * p.columns + 4 * g;
    for (; n0 < l.g.N; n0 += step) {
        w = next;
        if (n0 + step < l.g.N) {
            const WeightRows at(l.g, n0 + step);
            next.load(at.codes, at.scales, b0, blocks);
        }
        w.settle();
        f32x4 acc[2] = {};
        add_run<X16>(acc, w, from, mine);
        if (r < rows) *reinterpret_cast<f32x4*>(out + n0) = acc[0] + acc[1];
    }
}

// The slices' sums in one, in order, and the epilogue: four columns a thread.  (Of 24 slices of 16 x 4096: 4.5 us, 5.7 with
// the epilogue's operands loaded after the sums; 16 loads in flight instead of 8 took 6.6.)
__global__ __launch_bounds__(kSumThreads) void matvec_sum_kernel(MatvecParams p, int slices) {
    const LinearParams& l = p.l;
    const int64_t i = (int64_t)blockIdx.x * kSumThreads + threadIdx.x, each = p.columns / 4, m = i / each, n = 4 * (i - m * each);
    if (m >= l.g.M) return;
    Beside beside[4];
    const int wide = l.act == Act::Swiglu ? 2 : 1;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (n + k < l.g.N && k % wide == 0) beside[k].load(l, m, n + k);
    const f32x4* const from = reinterpret_cast<const f32x4*>(p.partial + m * p.columns + n);
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int s = 0; s < slices; ++s) v += from[s * l.g.M * each];
    with_act(l.act, [&](auto a) KQ_INLINE {
        constexpr Act A = decltype(a)::value;
        constexpr int kWide = A == Act::Swiglu ? 2 : 1;
#pragma unroll
        for (int k = 0; k < 4; k += kWide)
            if (n + k < l.g.N) finish<A>(l, m, n + k, v[k], v[k + kWide - 1], beside[k]);
    });
}

int64_t vec_slices(int64_t K) { return (K / 32 + kSliceBlocks - 1) / kSliceBlocks; }
int64_t vec_columns(int64_t N) { return (N + kVecRows - 1) / kVecRows * kVecRows; }

// Bytes of x's rows in LDS.
int64_t resident_bytes(int64_t M, int64_t K, bool x16) { return M * (K / 32 * (x16 ? 64 : 192) + 80); }

}  // namespace

// Only the slices' form has one.
int64_t matvec_workspace(int64_t M, int64_t N, int64_t K, bool x16) {
    if (M > kVecRows || K < kResidentColumns || vec_slices(K) > 65535 || resident_bytes(M, K, x16) <= kResidentBytes) return 0;
    return vec_slices(K) * M * vec_columns(N) * (int64_t)sizeof(float);
}

hipError_t launch_matvec(MatvecParams p, hipStream_t st) {
    const int64_t M = p.l.g.M, N = p.l.g.N, K = p.l.g.K, tiles = (N + kVecRows - 1) / kVecRows;
    const dim3 grid((unsigned)tiles, (unsigned)((M + kVecRows - 1) / kVecRows));
    const int64_t resident = resident_bytes(M, K, p.x16);
    if (M <= kVecRows && K >= kResidentColumns && resident <= kResidentBytes) {
        const size_t lds = resident + (kStepBlocks - 1) * (p.x16 ? 64 : 192);  // the last step reads whole steps, and drops blocks past x
        if (p.x16) matvec_resident_kernel<true><<<grid, 64 * kVecWaves, lds, st>>>(p);
        else matvec_resident_kernel<false><<<grid, 64 * kVecWaves, lds, st>>>(p);
    } else if (p.partial) {
        p.columns = vec_columns(N);
        const int64_t slices = vec_slices(K), eights = (tiles + kVecWaves - 1) / kVecWaves;
        // as many workgroups as the GPU holds, each with the same number of tiles a wave
        const int64_t turns = std::max<int64_t>(1, (eights * slices + 767) / 768);
        const dim3 shares((unsigned)((eights + turns - 1) / turns), (unsigned)slices);
        const size_t lds = resident_bytes(M, 32 * kSliceBlocks, p.x16);
        if (p.x16) matvec_slice_kernel<true><<<shares, 64 * kVecWaves, lds, st>>>(p);
        else matvec_slice_kernel<false><<<shares, 64 * kVecWaves, lds, st>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        matvec_sum_kernel<<<(unsigned)((M * (p.columns / 4) + kSumThreads - 1) / kSumThreads), kSumThreads, 0, st>>>(p, (int)slices);
    } else {
        if (p.x16) matvec_narrow_kernel<true><<<grid, 64 * kVecWaves, 0, st>>>(p);
        else matvec_narrow_kernel<false><<<grid, 64 * kVecWaves, 0, st>>>(p);
    }
    return hipGetLastError();
}

}  // namespace kq
