// Attention of one new token of every sequence over a paged cache:
//     out = softmax(scale q K^T) V
// over the sequence's tokens (or its last `window`), K and V in bf16, MXFP8 or
// MXFP4.  One pass over the cache with the running maximum and sum of the
// softmax; ragged sequences are shared out to workgroups in runs of equal length
// (kq_split.h), and those that are cut are joined by a second launch.
//
// A wave takes a tile of 32 tokens of one head of the cache and up to 16 of the
// query heads that share it.  Both products run on the bf16 matrix cores, which
// hold the cache's values of every format exactly:
//     S^T = K Q^T   A: 16 tokens x 32 columns, lane (r, g) = row r, eight columns
//     O^T = V^T P^T A: 16 columns x 32 tokens, lane (r, g) = column r, tokens 8 g .. 8 g + 7
// (r = lane % 16, g = lane / 16).  Row r of S^T's tile m is token
// 8 (r / 4) + 4 m + r % 4, so that a lane's eight results, rows 4 g .. 4 g + 3 of
// two tiles, are query r's scores of tokens 8 g .. 8 g + 7: P^T's operand as it
// is, without an exchange between lanes.  The order of the columns in S^T's sum
// is free, so each lane's columns of K are 16 bytes side by side; V's columns
// that a lane loads of its eight tokens are turned into operands by byte
// permutations.  Operands of 32 bits (the softmax's p, and q of that type) go in
// as three bf16 terms, which hold their 24 bits.  (p as two terms, within 2^-16
// of it, for bf16 results: 46 us for 49 with 64 ragged sequences of up to 8192
// tokens in MXFP4, 194 for 199 in the MXFP8 case below.)
//
// Bound by HBM for bf16 and MXFP8 (4 x 131072 tokens, 32 query heads over 8 of
// 128: 357 us for 2148 MB, 191 for 1107 MB, 6.0 and 5.8 TB/s).  MXFP4 takes
// about 10 us and its bytes at 5.2 TB/s (16 x 8192 tokens 37.7 us for 143 MB,
// 64 x 4096 65 for 286): lengths, page table, q and the first tiles, the waves'
// join and uneven ends of runs, and at 570 MB (4 x 131072) 128 to 137 us, with
// the vector units, which make bf16 of the codes, busy for 0.6 of the time and
// the matrix cores for 0.2.  For a few thousand tokens that first part is all,
// with the second launch (one sequence of 1000 tokens: 9.3 + 3.9 us).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "kq_mx.h"
#include "kq_serve.h"
#include "kq_split.h"

namespace kq {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kAttnWaves = 4;
constexpr int kAttnThreads = 64 * kAttnWaves;
constexpr int kMostGroups = 1280;  // workgroups of a launch, where each has its run
constexpr int kRowTile = 16;       // query heads of a workgroup

template <CacheFormat F>
constexpr int kBits = F == CacheFormat::Bf16 ? 16 : F == CacheFormat::Mxfp8 ? 8 : 4;

constexpr int least(int a, int b) { return a < b ? a : b; }

// N bytes (2, 4, 8 or 16) at p.
template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[(N + 3) / 4]) {
    if constexpr (N == 2) {
        w[0] = *reinterpret_cast<const uint16_t*>(p);
    } else if constexpr (N == 4) {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else if constexpr (N == 8) {
        const u32x2v v = *reinterpret_cast<const u32x2v*>(p);
        w[0] = v[0];
        w[1] = v[1];
    } else {
        const u32x4v v = *reinterpret_cast<const u32x4v*>(p);
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = v[k];
    }
}

// Values 2 I and 2 I + 1 of a row's loaded words, as bf16.
template <CacheFormat F, int I, int W>
__device__ __forceinline__ uint32_t pair_of(const uint32_t (&w)[W], float scale) {
    if constexpr (F == CacheFormat::Bf16) return w[I];
    else if constexpr (F == CacheFormat::Mxfp8) return e4m3_pair<I % 2>(w[I / 2], scale);
    else return e2m1_pair<I % 4>(w[I / 4], scale);
}

__device__ __forceinline__ bf16x8 operand(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_bit_cast(bf16x8, u32x4v{a, b, c, d});
}

// Eight values in 32 bits as TERMS bf16 operands whose sum they are (three; one for values of 16 bits): the leading bits as
// they stand, what is left rounded in the last.
template <int TERMS>
__device__ __forceinline__ void split_terms(const float (&v)[8], bf16x8 (&t)[TERMS]) {
    float f[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] = v[k];
#pragma unroll
    for (int n = 0; n < TERMS; ++n) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (n + 1 == TERMS) {
                w[k] = bf16_pair(f[2 * k], f[2 * k + 1]);
            } else {
                w[k] = __builtin_amdgcn_perm(__float_as_uint(f[2 * k + 1]), __float_as_uint(f[2 * k]), 0x07060302u);
                f[2 * k] -= bf16_low(w[k]);
                f[2 * k + 1] -= bf16_high(w[k]);
            }
        }
        t[n] = operand(w[0], w[1], w[2], w[3]);
    }
}

// The same over the four lanes of a query (r, r + 16, r + 32, r + 48).
__device__ __forceinline__ float query_max(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float query_sum(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The same over a wave.
template <int CTRL>
__device__ __forceinline__ float row_other(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, row_other<0x128>(v));  // row_ror 8, 4, 2, 1: every lane of a row of 16 has the row's
    v = fmaxf(v, row_other<0x124>(v));
    v = fmaxf(v, row_other<0x122>(v));
    return query_max(fmaxf(v, row_other<0x121>(v)));
}
__device__ __forceinline__ float wave_sum(float v) {
    v += row_other<0x128>(v);
    v += row_other<0x124>(v);
    v += row_other<0x122>(v);
    return query_sum(v + row_other<0x121>(v));
}

constexpr float kLowest = -3.402823466e38f;

// A uniform read of an array that the kernel does not write, by a scalar load.
typedef const __attribute__((address_space(4))) int32_t* const_i32_ptr;

// Where a tile's tokens are: rows of a head in the cache for its tokens 0 .. 15 and 16 .. 31.
struct Rows {
    int64_t at[2];
    // Tokens 32 t .. 32 t + 31 of head h, of which those before `end` exist.
    __device__ __forceinline__ Rows(const Cache& c, const int32_t* table, int h, int t, int end) {
        const int base = t * kTileTokens;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int token = base + 16 * i;
            const int32_t entry = ((const_i32_ptr)table)[page_index(token, end, c.page_shift)];
            at[i] = ((page_of(entry, c.pages) * c.heads + h) << c.page_shift) + (token & (c.page_size - 1));
        }
    }
};

// DC: columns of the matrix products, at least d; FULL: d itself (without it, widths of 64 and 128 take 11.6 us for 9.0 and
// 52.9 for 47.5: addresses that are not constants).  Lanes of columns past d load the row's last ones:
// q is 0 there, and those columns of the result are not stored.
template <CacheFormat F, int DC, bool FULL>
struct Tile {
    static constexpr int kE8 = kBits<F>;  // bytes of eight values
    // K: a lane's columns of unit u are kKw from 4 kKw u + kKw g on
    static constexpr int kSteps = DC / 32, kKs = least(kSteps, 16 / kE8), kKw = 8 * kKs, kKu = kSteps / kKs;
    static constexpr int kKb = kKs * kE8, kKwords = (kKb + 3) / 4;
    // V: a lane's columns of unit u are kVw from 16 kVw u + kVw r on
    static constexpr int kVc = DC / 16, kVw = least(kVc, F == CacheFormat::Bf16 ? 8 : 16), kVu = kVc / kVw;
    static constexpr int kVb = kVw * kE8 / 8, kVwords = (kVb + 3) / 4;
    static constexpr bool kScaled = F != CacheFormat::Bf16;

    uint32_t k[2][kKu][kKwords];
    uint32_t v[8][kVu][kVwords];
    uint32_t ks[2][kScaled ? kKu : 1];
    uint32_t vs[8][kScaled ? kVu : 1];

    // A lane's places in a tile's rows, the same for every tile.
    struct Lane {
        int k[kKu], ks[kKu], v[kVu], vs[kVu];
        int row, scales;  // bytes of a row, and of its scales
        bool low_k, low_v;
        __device__ __forceinline__ explicit Lane(const Cache& c) {
            const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4, d = FULL ? DC : c.d;
            row = d * kE8 / 8;
            scales = d / 32;
            low_k = r < 8;
            low_v = g < 2;
            const int tk = (8 * (r >> 2) + (r & 3)) % 16, tv = 8 * (g & 1);
#pragma unroll
            for (int u = 0; u < kKu; ++u) {
                const int column = min(4 * kKw * u + kKw * g, d - kKw);
                k[u] = tk * row + column * kE8 / 8;
                ks[u] = tk * scales + column / 32;
            }
#pragma unroll
            for (int u = 0; u < kVu; ++u) {
                const int column = min(16 * kVw * u + kVw * r, d - kVw);
                v[u] = tv * row + column * kE8 / 8;
                vs[u] = tv * scales + column / 32;
            }
        }
    };

    __device__ __forceinline__ void load(const Cache& c, const Lane& l, const Rows& rows) {
        const int row = FULL ? DC * kE8 / 8 : l.row, scales = FULL ? DC / 32 : l.scales;
        const uint8_t* const kp = l.low_k ? c.k + rows.at[0] * row : c.k + rows.at[1] * row;
        const uint8_t* const vp = l.low_v ? c.v + rows.at[0] * row : c.v + rows.at[1] * row;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int u = 0; u < kKu; ++u) load_words<kKb>(kp + l.k[u] + 4 * m * row, k[m][u]);
        if constexpr (kScaled) {
            const uint8_t* const sp = l.low_k ? c.k_scales + rows.at[0] * scales : c.k_scales + rows.at[1] * scales;
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int u = 0; u < kKu; ++u) ks[m][u] = sp[l.ks[u] + 4 * m * scales];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int u = 0; u < kVu; ++u) load_words<kVb>(vp + l.v[u] + j * row, v[j][u]);
        if constexpr (kScaled) {
            const uint8_t* const sp = l.low_v ? c.v_scales + rows.at[0] * scales : c.v_scales + rows.at[1] * scales;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int u = 0; u < kVu; ++u) vs[j][u] = sp[l.vs[u] + j * scales];
        }
    }

    // Values of tokens that do not count are zero, whatever the cache holds there.
    __device__ __forceinline__ void clear(int t, int from, int end) {
        const int token = t * kTileTokens + 8 * ((threadIdx.x & 63) >> 4);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool counts = token + j >= from && token + j < end;
#pragma unroll
            for (int u = 0; u < kVu; ++u) {
#pragma unroll
                for (int i = 0; i < kVwords; ++i) v[j][u][i] = counts ? v[j][u][i] : 0u;
                if (kScaled) vs[j][u] = counts ? vs[j][u] : 127u;
            }
        }
    }

    // Unit u's columns of step w of K's tile m.
    template <int W>
    __device__ __forceinline__ bf16x8 keys(int m, int u) const {
        const float s = kScaled ? mx_scale(ks[m][kScaled ? u : 0]) : 0.f;
        return operand(pair_of<F, 4 * W>(k[m][u], s), pair_of<F, 4 * W + 1>(k[m][u], s), pair_of<F, 4 * W + 2>(k[m][u], s),
                       pair_of<F, 4 * W + 3>(k[m][u], s));
    }
    // Columns 2 I and 2 I + 1 of V's unit u, eight tokens each.
    template <int I>
    __device__ __forceinline__ void values(int u, bf16x8 (&a)[2]) const {
        uint32_t x[8], lo[4], hi[4];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = pair_of<F, I>(v[j][u], kScaled ? mx_scale(vs[j][kScaled ? u : 0]) : 0.f);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            lo[j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x05040100u);
            hi[j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x07060302u);
        }
        a[0] = operand(lo[0], lo[1], lo[2], lo[3]);
        a[1] = operand(hi[0], hi[1], hi[2], hi[3]);
    }
};

template <int I, int N, class Fn>
__device__ __forceinline__ void unrolled(Fn f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        unrolled<I + 1, N>(f);
    }
}

// The column of O^T's tile n, row i.
template <class T>
__device__ __forceinline__ int value_column(int n, int i) {
    constexpr int w = T::kVw;
    return 16 * w * (n / w) + w * i + n % w;
}

#define KQ_INLINE __attribute__((always_inline))

// Waves of a SIMD that registers are kept for.  (MXFP4, 128 columns, 64 ragged sequences of up to 8192 tokens: 48 to 51 us with
// two, 47.5 with three; four spill.)
template <CacheFormat F, int DC, bool B16>
constexpr int kWavesHeld = !B16 ? 1 : DC > 128 ? 2 : F == CacheFormat::Mxfp4 || DC <= 64 ? 3 : 2;

template <CacheFormat F, int DC, bool B16, bool FULL>
__global__ __launch_bounds__(kAttnThreads, (kWavesHeld<F, DC, B16>)) void attn_kernel(AttnParams p) {
    typedef Tile<F, DC, FULL> T;
    constexpr int kQ = B16 ? 1 : 3, kP = 3;  // terms of q (exact in bf16, or 32 bits) and p
    // tiles that a wave has loaded or is loading (MXFP4, 128 columns, 64 ragged sequences: 47.5 us with one, 48 with two)
    constexpr int kAhead = F != CacheFormat::Mxfp4 && DC < 256 ? 2 : 1;
    extern __shared__ float shared[];  // [2, rows, d]: of waves 0 and 2, and 1 and 3
    __shared__ float stats[2][kAttnWaves][kRowTile];
    const Cache& c = p.c;
    const int d = FULL ? DC : c.d;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    Run run = find_run(p.lengths, (int)p.B, p.max_tokens, p.window, p.inverse, (int)blockIdx.x);
    const int row_tiles = (p.group + kRowTile - 1) / kRowTile;
    const int h = blockIdx.y / row_tiles, first_row = (blockIdx.y - h * row_tiles) * kRowTile;
    const int rows = min(p.group - first_row, kRowTile), head = h * p.group + first_row;
    const int64_t heads = (int64_t)c.heads * p.group;
    const typename T::Lane lanes(c);
    for (; run.tiles > 0; run.skip = 0) {
    // a piece: a sequence's tiles in this run, from `done` on
    const Span span(run.length, p.max_tokens, p.window);
    const int done = max(run.skip - kPieceTiles, 0), left = span.tiles() - done, before = max(kPieceTiles - run.skip, 0);
    const int tiles = run.tiles < left + before ? (int)run.tiles - before : left;
    run.tiles -= tiles + before;
    if (tiles <= 0) break;  // the run ends before the first
    const int32_t* const table = p.table + run.b * p.table_stride;
    auto where = [&](int t) KQ_INLINE { return Rows(c, table, h, t, span.end); };
    const int last = span.end > span.first ? span.first_tile() + done + tiles : 0;
    int t = span.first_tile() + done + wave;
    T tile[kAhead];
    unrolled<0, kAhead - 1>([&](auto stage) KQ_INLINE {
        if (t + stage * kAttnWaves < last) tile[stage].load(c, lanes, where(t + stage * kAttnWaves));
    });

    bf16x8 q[T::kSteps][kQ];
    unrolled<0, T::kSteps>([&](auto step) KQ_INLINE {
        constexpr int u = step / T::kKs, w = step % T::kKs;
        const int column = 4 * T::kKw * u + T::kKw * g + 8 * w;
        const int64_t at = run.b * p.q_seq + (head + min(r, rows - 1)) * p.q_head + min(column, d - 8);
        float f[8];
        if constexpr (B16) {
            typedef uint32_t W __attribute__((ext_vector_type(4), aligned(2)));
            const W w = *reinterpret_cast<const W*>(static_cast<const uint16_t*>(p.q) + at);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                f[2 * k] = bf16_low(w[k]);
                f[2 * k + 1] = bf16_high(w[k]);
            }
        } else {
            typedef float W __attribute__((ext_vector_type(4), aligned(4)));
            const W a = *reinterpret_cast<const W*>(static_cast<const float*>(p.q) + at);
            const W b = *reinterpret_cast<const W*>(static_cast<const float*>(p.q) + at + 4);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                f[k] = a[k];
                f[4 + k] = b[k];
            }
        }
        const bool live = r < rows && (FULL || column < d);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = live ? f[k] : 0.f;
        split_terms<kQ>(f, q[step]);
    });

    f32x4 o[T::kVc];
#pragma unroll
    for (int n = 0; n < T::kVc; ++n) o[n] = f32x4{0.f, 0.f, 0.f, 0.f};
    float most = kLowest, sum = 0.f;
    const float scale = p.scale * 1.44269504088896341f;  // scores in powers of two

    auto attend = [&](T& tile, int t) KQ_INLINE {
        float s[8];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            f32x4 a = {0.f, 0.f, 0.f, 0.f};
            unrolled<0, T::kSteps>([&](auto step) KQ_INLINE {
                constexpr int u = step / T::kKs, w = step % T::kKs;
                const bf16x8 k = tile.template keys<w>(m, u);
#pragma unroll
                for (int n = 0; n < kQ; ++n) a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[step][n], a, 0, 0, 0);
            });
#pragma unroll
            for (int k = 0; k < 4; ++k) s[4 * m + k] = a[k] * scale;
        }
        if (t * kTileTokens < span.first || (t + 1) * kTileTokens > span.end) {
            asm volatile("");  // a branch: tiles in between skip this
            tile.clear(t, span.first, span.end);
            const int token = t * kTileTokens + 8 * g;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (token + k < span.first || token + k >= span.end) s[k] = -INFINITY;
        }
        float top = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
        top = fmaxf(query_max(top), most);
        if (__any(top > most)) {
            const float f = __builtin_amdgcn_exp2f(most - top);
            sum *= f;
#pragma unroll
            for (int n = 0; n < T::kVc; ++n) o[n] *= f;
            most = top;
        }
        float e[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) e[k] = __builtin_amdgcn_exp2f(s[k] - most);
        sum += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
        bf16x8 pt[kP];
        split_terms<kP>(e, pt);
#pragma unroll
        for (int u = 0; u < T::kVu; ++u) {
            unrolled<0, T::kVw / 2>([&](auto pair) KQ_INLINE {
                bf16x8 a[2];
                tile.template values<pair>(u, a);
#pragma unroll
                for (int n = 0; n < kP; ++n) {
                    f32x4 &x = o[u * T::kVw + 2 * pair], &y = o[u * T::kVw + 2 * pair + 1];
                    x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[0], pt[n], x, 0, 0, 0);
                    y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[1], pt[n], y, 0, 0, 0);
                }
            });
        }
    };
    // the next tiles' loads are in flight while a tile is worked on
    while (t < last) {
        bool more = true;
        unrolled<0, kAhead>([&](auto stage) KQ_INLINE {
            constexpr int now = stage, late = (stage + kAhead - 1) % kAhead;
            if (!more) return;
            const int tn = t + (kAhead - 1) * kAttnWaves;
            if (tn < last) tile[late].load(c, lanes, where(tn));
            attend(tile[now], t);
            t += kAttnWaves;
            more = t < last;
        });
    }
    // the waves' results in one: the common maximum first, then sums
    sum = query_sum(sum);
    if (g == 0) {
        stats[0][wave][r] = most;
        stats[1][wave][r] = sum;
    }
    __syncthreads();
    float all = fmaxf(fmaxf(stats[0][0][r], stats[0][1][r]), fmaxf(stats[0][2][r], stats[0][3][r]));
    const float f = __builtin_amdgcn_exp2f(most - all);
    static_assert(kAttnWaves == 4, "two waves a place");
#pragma unroll
    for (int turn = 0; turn < 2; ++turn) {
        if (wave / 2 == turn && r < rows) {
#pragma unroll
            for (int n = 0; n < T::kVc; ++n)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int column = value_column<T>(n, 4 * g + k);
                    if (!FULL && column >= d) continue;
                    float& v = shared[((wave & 1) * rows + r) * d + column];
                    v = turn ? v + o[n][k] * f : o[n][k] * f;
                }
        }
        __syncthreads();
    }
    // a sequence in one run is done; one that is cut leaves its piece, and its first run the place of them all
    const bool begins = done == 0, whole = begins && tiles == left;
    if (begins && blockIdx.y == 0 && threadIdx.x == 0) {
        const int64_t over = left - tiles;  // in the runs that follow
        p.plan[2 * run.b] = blockIdx.x;
        p.plan[2 * run.b + 1] = over > 0 ? 2 + (int)((over - 1) / run.each) : 1;
    }
    const int64_t place = (2 * (int64_t)blockIdx.x + begins) * heads + head;
    for (int i = threadIdx.x; i < rows * d; i += kAttnThreads) {
        const int row = i / d, column = i - row * d;
        const float top = fmaxf(fmaxf(stats[0][0][row], stats[0][1][row]), fmaxf(stats[0][2][row], stats[0][3][row]));
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < kAttnWaves; ++w) total += stats[1][w][row] * __builtin_amdgcn_exp2f(stats[0][w][row] - top);
        float v = shared[row * d + column] + shared[(rows + row) * d + column];
        if (whole) {
            v = total != 0.f ? v / total : 0.f;
            const int64_t at = run.b * p.out_seq + (head + row) * p.out_head + column;
            if (B16) static_cast<__bf16*>(p.out)[at] = (__bf16)v;
            else static_cast<float*>(p.out)[at] = v;
            if (p.lse && column == 0)
                p.lse[run.b * heads + head + row] =
                    total != 0.f ? (top + __builtin_amdgcn_logf(total)) * 0.693147180559945309f : -INFINITY;
        } else {
            p.partial[(place + row) * d + column] = v;
            if (column == 0) {
                p.stats[2 * (place + row)] = top;
                p.stats[2 * (place + row) + 1] = total;
            }
        }
    }
    if (run.tiles <= 0) break;
    run.length = ((const_i32_ptr)p.lengths)[++run.b];
    __syncthreads();  // the next piece's waves write where these read
    }
}

// The pieces of a sequence in one, a workgroup a sequence and query head: its threads take four columns each of as many pieces
// at once as there are threads for.  3 to 5 us, of which most is the launch and three loads that wait for each other.
constexpr int kJoinThreads = 256;

template <bool B16>
__global__ __launch_bounds__(kJoinThreads) void attn_join_kernel(AttnParams p) {
    const int b = blockIdx.x, head = blockIdx.y, d = p.c.d, heads = p.c.heads * p.group;
    const int run = p.plan[2 * b], count = p.plan[2 * b + 1];
    if (count <= 1) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // piece 0 is at place 2 run + 1, piece i at 2 (run + i)
    auto piece = [&](int i) KQ_INLINE { return (2 * (int64_t)(run + i) + (i == 0)) * heads + head; };
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2* const stats = reinterpret_cast<const f32x2*>(p.stats);
    const int columns = d / 4, at = threadIdx.x / columns, column = threadIdx.x - at * columns, step = kJoinThreads / columns;
    const f32x4* const from = reinterpret_cast<const f32x4*>(p.partial) + column;
    const bool busy = at < step;
    auto load = [&](int i, f32x4* v, float* m) KQ_INLINE {
        *v = from[piece(i) * columns];
        *m = stats[piece(i)][0];
    };
    f32x4 now = {0.f, 0.f, 0.f, 0.f};
    float most = kLowest;
    if (busy && at < count) load(at, &now, &most);  // in flight while the maximum is found
    // every wave has the maximum of all pieces
    float top = kLowest, total = 0.f;
    for (int i = lane; i < count; i += 64) top = fmaxf(top, stats[piece(i)][0]);
    top = wave_max(top);
    if (wave == 0) {
        for (int i = lane; i < count; i += 64) {
            const f32x2 s = stats[piece(i)];
            total += s[1] * __builtin_amdgcn_exp2f(s[0] - top);
        }
        total = wave_sum(total);
    }
    f32x4 v = now * __builtin_amdgcn_exp2f(most - top);
    if (busy) {
#pragma unroll 4
        for (int i = at + step; i < count; i += step) {
            load(i, &now, &most);
            v += now * __builtin_amdgcn_exp2f(most - top);
        }
    }
    __shared__ f32x4 sums[kJoinThreads];
    __shared__ float all;
    sums[threadIdx.x] = v;
    if (threadIdx.x == 0) all = total;
    __syncthreads();
    total = all;
    if (at == 0) {
        const int n = min(step, count);
        for (int i = 1; i < n; ++i) v += sums[i * columns + column];
        const int64_t to = b * p.out_seq + head * p.out_head + 4 * column;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float f = total != 0.f ? v[k] / total : 0.f;
            if (B16) static_cast<__bf16*>(p.out)[to + k] = (__bf16)f;
            else static_cast<float*>(p.out)[to + k] = f;
        }
    }
    if (p.lse && threadIdx.x == 0)
        p.lse[(int64_t)b * heads + head] = total != 0.f ? (top + __builtin_amdgcn_logf(total)) * 0.693147180559945309f : -INFINITY;
}

// Runs that a head's tiles are cut into at most.
int64_t most_runs(int64_t heads, int64_t group) {
    return std::max<int64_t>(1, kMostGroups / (heads * ((group + kRowTile - 1) / kRowTile)));
}

int64_t round16(int64_t n) { return (n + 15) / 16 * 16; }

// Workgroups of a kernel that the GPU holds at once.
template <class K>
int resident_groups(K kernel, size_t lds) {
    int device = 0, units = 0, each = 0;
    if (hipGetDevice(&device) != hipSuccess || hipDeviceGetAttribute(&units, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess ||
        hipOccupancyMaxActiveBlocksPerMultiprocessor(&each, kernel, kAttnThreads, lds) != hipSuccess)
        return 512;
    return units * std::max(each, 1);
}

template <CacheFormat F, int DC, bool B16, bool FULL>
hipError_t launch_attn_of(AttnParams& p, int64_t most, hipStream_t st) {
    const size_t lds = sizeof(float) * 2 * std::min(p.group, kRowTile) * p.c.d;
    static const int resident = resident_groups(attn_kernel<F, DC, B16, FULL>, sizeof(float) * 2 * kRowTile * DC);
    const int rows = p.c.heads * ((p.group + kRowTile - 1) / kRowTile);
    p.runs = (int)std::max<int64_t>(1, std::min(std::min<int64_t>(resident / rows, most_runs(p.c.heads, p.group)), most));
    p.inverse = 1.0 / p.runs;
    attn_kernel<F, DC, B16, FULL><<<dim3((unsigned)p.runs, (unsigned)rows), kAttnThreads, lds, st>>>(p);
    return hipGetLastError();
}

template <CacheFormat F, int DC>
hipError_t launch_attn_width(AttnParams& p, int64_t most, hipStream_t st) {
    if (p.c.d == DC) return p.is16 ? launch_attn_of<F, DC, true, true>(p, most, st) : launch_attn_of<F, DC, false, true>(p, most, st);
    return p.is16 ? launch_attn_of<F, DC, true, false>(p, most, st) : launch_attn_of<F, DC, false, false>(p, most, st);
}

template <CacheFormat F>
hipError_t launch_attn_format(AttnParams& p, int64_t most, hipStream_t st) {
    if (p.c.d <= 64) return launch_attn_width<F, 64>(p, most, st);
    if (p.c.d <= 128) return launch_attn_width<F, 128>(p, most, st);
    return launch_attn_width<F, 256>(p, most, st);
}

}  // namespace

int64_t attn_workspace(int64_t B, int64_t heads, int64_t group, int64_t d) {
    const int64_t rows = run_slots(most_runs(heads, group)) * heads * group;
    return round16(8 * B) + round16(8 * rows) + round16(4 * rows * d);
}

hipError_t launch_attn(AttnParams p, hipStream_t st) {
    const int heads = p.c.heads * p.group;
    p.plan = reinterpret_cast<int32_t*>(p.workspace);
    p.stats = reinterpret_cast<float*>(p.workspace + round16(8 * p.B));
    p.partial = reinterpret_cast<float*>(p.workspace + round16(8 * p.B) + round16(8 * run_slots(most_runs(p.c.heads, p.group)) * heads));
    // no more runs than the longest sequences that the table holds can fill
    const int64_t seen = p.window > 0 && p.window < p.max_tokens ? std::min(p.window + kTileTokens - 1, p.max_tokens) : p.max_tokens;
    const int64_t longest = seen / kTileTokens + 1 + kPieceTiles;
    const int64_t most = (p.B * longest + kLeastTiles - 1) / kLeastTiles;
    hipError_t e = hipSuccess;
    switch (p.c.format) {
        case CacheFormat::Bf16: e = launch_attn_format<CacheFormat::Bf16>(p, most, st); break;
        case CacheFormat::Mxfp8: e = launch_attn_format<CacheFormat::Mxfp8>(p, most, st); break;
        case CacheFormat::Mxfp4: e = launch_attn_format<CacheFormat::Mxfp4>(p, most, st); break;
    }
    if (e != hipSuccess || p.runs == 1) return e;  // (one run cuts no sequence)
    const dim3 joins((unsigned)p.B, (unsigned)heads);
    if (p.is16) attn_join_kernel<true><<<joins, kJoinThreads, 0, st>>>(p);
    else attn_join_kernel<false><<<joins, kJoinThreads, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace kq
