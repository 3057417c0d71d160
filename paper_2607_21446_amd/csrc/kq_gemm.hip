// W4A4 MXFP4 GEMM: the consumer of the quantizer's output (Sec. 3.1 eq. (1),
// Sec. 3.4): C[M, N] (+)= deq(Xq)[M, K] . deq(Wq)[N, K]^T, both operands in
// the MXFP4 layout the quantizer writes -- codes [rows, K/2] (element 2i in
// the low nibble of byte i) and E8M0 scales [rows, K/32] -- so activations
// from kq_quantize* and weights from kq_weight_transform feed it unchanged.
//
// Matrix cores: v_mfma_scale_f32_32x32x64_f8f6f4 with both operands E2M1.  In
// that instruction lane l supplies row (A) or column (B) l % 32 and the 32
// K-values 32 (l / 32) .. 32 (l / 32) + 31 of the 64-wide K step, 16 bytes,
// plus one E8M0 byte for them: exactly one 32-element block and its scale in
// the quantizer's layout, so fragments are plain 16-byte loads and no
// re-layout or pre-shuffle of codes or scales is needed.  Products of E2M1
// values times the two scales are exact in fp32; the sum over K is
// accumulated in fp32 (order not specified).
//
// Kernels: a pipelined one on a 256 x 256 (eight waves) or 128 x 128 (four waves)
// tile of C, for K up to 2^24 (32-bit offsets within a tile), and one whose waves
// split K, on tiles of 32 x 32 to 64 x 64, for few tiles (and any K).  The tiles' sums
// are in kq_gemm_tile.h, what becomes of them here.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kq_gemm_tile.h"
#include "kq_kernels.h"

namespace kq {

namespace {

// Four consecutive fp32 C values of row m from column n.  (One vector access: as
// float4, four members, the compiler shared the last with the other branch.)
__device__ __forceinline__ void store_c4(const GemmParams& g, int64_t m, int64_t n, float4 v) {
    float* const c = g.C + m * g.ldc_out + n;
    if (n + 3 < g.N) {
        *reinterpret_cast<f32x4*>(c) = f32x4{v.x, v.y, v.z, v.w};
    } else {
        c[0] = v.x;
        if (n + 1 < g.N) c[1] = v.y;
        if (n + 2 < g.N) c[2] = v.z;
        if (n + 3 < g.N) c[3] = v.w;
    }
}

// The values they are added to: the bias, C (accumulate) or zeros; zeros past M and N.
__device__ __forceinline__ float4 base_c4(const GemmParams& g, int64_t m, int64_t n) {
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* const src = g.bias ? g.bias : g.accumulate ? g.C : nullptr;
    if (src && m < g.M && n < g.N) {
        const float* const b = src + m * g.ldc_out + n;
        if (n + 3 < g.N) {
            const f32x4 o = *reinterpret_cast<const f32x4*>(b);
            v = make_float4(o.x, o.y, o.z, o.w);
        } else {
            v.x = b[0];
            if (n + 1 < g.N) v.y = b[1];
            if (n + 2 < g.N) v.z = b[2];
            if (n + 3 < g.N) v.w = b[3];
        }
    }
    return v;
}

// Four consecutive bf16 C values.
__device__ __forceinline__ void store_b4(const GemmParams& g, int64_t m, int64_t n, float4 v) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    const bf16x4 b = {(__bf16)v.x, (__bf16)v.y, (__bf16)v.z, (__bf16)v.w};
    const uint2 w = __builtin_bit_cast(uint2, b);
    uint16_t* const c = g.C16 + m * g.ldc_out + n;
    if (n + 3 < g.N) {
        *reinterpret_cast<u32x2b*>(c) = u32x2b{w.x, w.y};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < g.N) c[e] = (uint16_t)((e < 2 ? w.x : w.y) >> (16 * (e & 1)));
    }
}

// Four consecutive values of the residual as two bf16 terms (zero past M and N, up to
// rows_pad and ldr); their squares are added to sq.
__device__ __forceinline__ void store_r4(const GemmParams& g, int64_t m, int64_t n, float4 v, double& sq) {
    const bool in = m < g.M;
    const float f[4] = {in && n < g.N ? v.x : 0.f, in && n + 1 < g.N ? v.y : 0.f, in && n + 2 < g.N ? v.z : 0.f,
                        in && n + 3 < g.N ? v.w : 0.f};
    uint32_t hi[2], lo[2];
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        const bf16x2 h2 = {(__bf16)f[e], (__bf16)f[e + 1]};
        const bf16x2 l2 = {(__bf16)(f[e] - (float)h2[0]), (__bf16)(f[e + 1] - (float)h2[1])};
        hi[e / 2] = __builtin_bit_cast(uint32_t, h2);
        lo[e / 2] = __builtin_bit_cast(uint32_t, l2);
        sq += (double)f[e] * (double)f[e] + (double)f[e + 1] * (double)f[e + 1];
    }
    *reinterpret_cast<uint2*>(g.rh + m * g.ldr + n) = make_uint2(hi[0], hi[1]);
    *reinterpret_cast<uint2*>(g.rl + m * g.ldr + n) = make_uint2(lo[0], lo[1]);
}

// The workgroup's sum of sq to its place (red: one entry per wave).
template <int WAVES>
__device__ __forceinline__ void block_squares(double sq, double* red, const GemmParams& g) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sq += __shfl_xor(sq, off);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sq;
    __syncthreads();
    if (threadIdx.x == 0) {
        double tot = red[0];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) tot += red[i];
        g.sq_part[blockIdx.x] = tot;
    }
}

}  // namespace

// The tile's accumulators, acc[i][j][4q + e] = C[mb0 + 32 (wm TM + j) + r][nb0 +
// 32 (wn TN + i) + 8 q + 4 h + e], to C through LDS, so that C (and the bias) is
// accessed along its rows, 512 bytes at a time, and not in 8- or 16-byte pieces
// of 32 rows (4608 x 12288 x 3072, bf16 / fp32: 141 / 155 us so, 119 / 131 along rows).
// Rows in LDS are 16 bytes apart from a multiple of 512 (256), so that the 16 rows of a
// write phase cover all banks.  When a tile of fp32 does not fit, it goes in NP passes of
// TN / NP of every wave's column tiles.
//
// OUT 0: fp32 (bias, accumulate); 1: bf16; 2: the residual v = bias + product as its
// two bf16 terms hi = bf16(v), lo = bf16(v - hi), zero in the padding columns and
// rows up to ldr and rows_pad, and the workgroup's sum of v^2 (fp64).
//
// BASE (the bias or C is added): all loads of a pass are issued before its stores (a
// wait for a load waits for every store issued before it too).
// 4096 x 5600 x 2240 and 18432 x 3072 x 3072 onto C, us: 104 and 220 with the loads
// among the stores, 88 and 188 so.
template <int WN, int WM, int TN, int TM, int OUT, bool BASE>
__device__ __forceinline__ void store_tile(const GemmParams& g, uint8_t* lds, int64_t nb0, int64_t mb0,
                                           const f32x16g (&acc)[TN][TM]) {
    typedef Tile<WN, WM, TN, TM> T;
    constexpr bool BF16 = OUT == 1;
    constexpr int ES = BF16 ? 2 : 4;
    constexpr int NP = (T::BM * (T::BN * ES + 16) <= (int)sizeof(typename T::Lds)) ? 1 : 2;
    constexpr int TP = TN / NP;                    // column tiles per wave and pass
    constexpr int RB = T::BN / NP * ES, RS = RB + 16;  // data and stride of a row in bytes
    static_assert(T::BM * RS <= (int)sizeof(typename T::Lds), "a pass fits LDS");
    constexpr int CPR = RB / 16, EPC = 16 / ES;    // 16-byte chunks per row, elements per chunk
    constexpr int STEP = 64 * T::WAVES / CPR;      // rows that the workgroup covers at a time
    constexpr int CH = T::BM / STEP;               // chunks per thread and pass
    static_assert(64 * T::WAVES % CPR == 0, "a thread keeps its column");
    const int t = threadIdx.x;
    const int wave = t >> 6, lane = t & 63;
    const int r = lane & 31, h = lane >> 5, wn = wave / WM, wm = wave % WM;
    const int last = (int)min<int64_t>(T::BM, g.M - mb0) - 1;  // the tile's last row of C
    // A thread takes one chunk of columns of every STEP-th row: whether the chunk is whole,
    // cut by N or past it is decided once a pass.  Decided for every chunk, in nested
    // branches, and so: 1000 x 1152 x 1152 onto C 12.3 and 8.8 us, fp32 8.6 and 7.8, bf16 7.3
    // and 7.0; 4096 x 5600 x 2240 onto C 76 and 67; 18432 x 3072 x 3072 onto C 169 and 151.
    const int trow = t / CPR, cl = t % CPR * EPC, seg = cl / (32 * TP);
    float4 base[BASE ? CH : 1];
    double sq = 0.0;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        // column of C of this thread's chunk: the pass holds TP tiles of each of the WN waves' column ranges
        const int64_t n = nb0 + seg * 32 * TN + 32 * p * TP + (cl - seg * 32 * TP);
        const bool whole = n + EPC <= g.N;
        if (p > 0) __syncthreads();
#pragma unroll
        for (int i = 0; i < TP; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                uint8_t* const dst = lds + (32 * (wm * TM + j) + r) * RS + (32 * (wn * TP + i) + 4 * h) * ES;
                const f32x16g& c = acc[p * TP + i][j];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (BF16) {
                        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                        const bf16x4 v = {(__bf16)c[4 * q], (__bf16)c[4 * q + 1], (__bf16)c[4 * q + 2], (__bf16)c[4 * q + 3]};
                        *reinterpret_cast<uint2*>(dst + 16 * q) = __builtin_bit_cast(uint2, v);
                    } else {
                        *reinterpret_cast<float4*>(dst + 32 * q) =
                            make_float4(c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]);
                    }
                }
            }
        __builtin_amdgcn_sched_barrier(0);  // the pass's accumulators are free for what is loaded
        if (BASE) {
            // rows past M load this thread's first row again (or the tile's first); not used
            const float* const src = (g.bias ? g.bias : g.C) + mb0 * g.ldc_out + n;
            const float* const first = src + (trow <= last ? trow : 0) * g.ldc_out;
#pragma unroll
            for (int k = 0; k < CH; ++k) base[k] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (whole) {
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    const float* const b = trow + k * STEP <= last ? first + k * STEP * g.ldc_out : first;
                    const f32x4 o = *reinterpret_cast<const f32x4*>(b);
                    base[k] = make_float4(o.x, o.y, o.z, o.w);
                }
            } else if (n < g.N) {
                const int left = (int)(g.N - 1 - n);  // 0 to 2; columns past N load the last one again
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    const float* const b = trow + k * STEP <= last ? first + k * STEP * g.ldc_out : first;
                    base[k] = make_float4(b[0], b[min(1, left)], b[left], 0.f);
                }
            }
        }
        __syncthreads();
        const uint8_t* const from = lds + trow * RS + 16 * (t % CPR);
        auto value = [&](int k) {
            float4 f = *reinterpret_cast<const float4*>(from + k * STEP * RS);
            if (BASE) f = make_float4(base[k].x + f.x, base[k].y + f.y, base[k].z + f.z, base[k].w + f.w);
            return f;
        };
        const int64_t at = (mb0 + trow) * g.ldc_out + n;
        if (OUT == 2) {
            if (n < g.ldr) {
#pragma unroll
                for (int k = 0; k < CH; ++k)
                    if (mb0 + trow + k * STEP < g.rows_pad) store_r4(g, mb0 + trow + k * STEP, n, value(k), sq);
            }
        } else if (whole) {
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                if (trow + k * STEP > last) break;
                if (BF16) {
                    const uint4 v = *reinterpret_cast<const uint4*>(from + k * STEP * RS);
                    *reinterpret_cast<u32x4b*>(g.C16 + at + k * STEP * g.ldc_out) = u32x4b{v.x, v.y, v.z, v.w};
                } else {
                    const float4 f = value(k);
                    *reinterpret_cast<f32x4*>(g.C + at + k * STEP * g.ldc_out) = f32x4{f.x, f.y, f.z, f.w};
                }
            }
        } else if (n < g.N) {
            const int left = (int)(g.N - 1 - n);
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                if (trow + k * STEP > last) break;
                if (BF16) {  // 1 to 7 values, as four, two and one
                    const uint4 v = *reinterpret_cast<const uint4*>(from + k * STEP * RS);
                    uint16_t* const c = g.C16 + at + k * STEP * g.ldc_out;
                    const int n = left + 1;
                    if (n & 4) *reinterpret_cast<u32x2b*>(c) = u32x2b{v.x, v.y};
                    if (n & 2) *reinterpret_cast<u32b*>(c + (n & 4)) = n & 4 ? v.z : v.x;
                    if (n & 1) c[n & 6] = (uint16_t)(n & 4 ? (n & 2 ? v.w : v.z) : (n & 2 ? v.y : v.x));
                } else {
                    const float4 f = value(k);
                    float* const c = g.C + at + k * STEP * g.ldc_out;
                    c[0] = f.x;
                    if (left >= 1) c[1] = f.y;
                    if (left >= 2) c[2] = f.z;
                }
            }
        }
    }
    if (OUT == 2) {
        __syncthreads();
        block_squares<T::WAVES>(sq, reinterpret_cast<double*>(lds), g);
    }
}

template <int TN, int TM, int W, int D>
__global__ __launch_bounds__(64 * W) void mxfp4_gemm_split_kernel(const GemmParams g, int64_t gx, int64_t gy) {
    constexpr int BN = 32 * TN, BM = 32 * TM, RS = BN + 4;
    __shared__ float sums[W * BM * RS];
    const int t = threadIdx.x;
    int64_t tn, tm;
    xcd_tile(gx, gy, tn, tm);
    const int64_t nb0 = tn * BN, mb0 = tm * BM;
    const int active = split_tile<TN, TM, W, D>(g, sums, nb0, mb0);
    const int64_t mend = g.rh ? g.rows_pad : g.M, nend = g.rh ? g.ldr : g.N;
    double sq = 0.0;
    for (int k = t; k < BM * BN / 4; k += 64 * W) {
        const int row = k / (BN / 4), col = 4 * (k % (BN / 4));
        const int64_t m = mb0 + row, n = nb0 + col;
        if (m >= mend || n >= nend) continue;
        const bool based = g.bias || g.accumulate;
        const float4 b = based ? base_c4(g, m, n) : make_float4(0.f, 0.f, 0.f, 0.f);
        float4 v = *reinterpret_cast<const float4*>(sums + row * RS + col);
        for (int w = 1; w < active; ++w) {
            const float4 o = *reinterpret_cast<const float4*>(sums + (w * BM + row) * RS + col);
            v = make_float4(v.x + o.x, v.y + o.y, v.z + o.z, v.w + o.w);
        }
        if (based) v = make_float4(b.x + v.x, b.y + v.y, b.z + v.z, b.w + v.w);
        if (g.C16) store_b4(g, m, n, v);
        else if (g.rh) store_r4(g, m, n, v, sq);
        else store_c4(g, m, n, v);
    }
    if (g.rh) {
        __shared__ double red[W];
        block_squares<W>(sq, red, g);
    }
}

// OUT, BASE: as store_tile (one kernel each: every epilogue in one is 78 KB of code).
template <int WN, int WM, int TN, int TM, bool PING, bool DMA_SCALES, int OUT, bool BASE>
__global__ __launch_bounds__(64 * WN * WM) void mxfp4_gemm_pipe_kernel(const GemmParams g, int64_t gx, int64_t gy) {
    typedef Tile<WN, WM, TN, TM> T;
    __shared__ typename T::Lds lds;
    int64_t tn, tm;
    xcd_tile(gx, gy, tn, tm);
    f32x16g acc[TN][TM];
    gemm_tile<WN, WM, TN, TM, PING, DMA_SCALES>(g, lds, tn * T::BN, tm * T::BM, acc);
    uint8_t* const stage = reinterpret_cast<uint8_t*>(&lds);
    store_tile<WN, WM, TN, TM, OUT, BASE>(g, stage, tn * T::BN, tm * T::BM, acc);
}

// The pipelined kernels index a tile's 256 rows with 32-bit byte offsets.
constexpr int64_t kPipeMaxK = int64_t(1) << 24;

// Tile of a call.  Measured, us (bf16 C, K 512 / 1152 / 3072 / 9600):
//   32 x 32 split (8 waves)     128 x  512: 3.4 / 3.8 /  7.0 / 11.0; 128 x 128 4.7 / 6.7 / 11.9 / 30.3
//   32 (M) x 64 (N) split       256 x 1152: 3.9 / 4.4 /  9.2 / 15.3; 32 x 32 3.9 / 4.5 / 10.9 / 19.0
//   64 x 64 split               512 x 2048: 5.0 / 6.0 / 12.2 / 24.9; 128 x 128 5.0 / 6.9 / 12.0 / 30.7
//   128 x 128 pipelined         512 x 4096: 5.4 / 7.4 / 12.9 / 32.0; 64 x 64 8.6 / 10.6 / 22.8 / 48.2
//                              4096 x 2048: 8.4 / 12.1 / 23.9 / 62.5; 256 x 256 11.2 / 15.1 / 25.8 / 63.8
//   256 x 256 pipelined        3000 x 3000: 11.1 / 15.5 / 25.8 / 63.9; 128 x 128 10.8 / 16.1 / 30.8 / 83.7
// So the smallest split tile that still gives a CU no more than one workgroup, and
// past 256 tiles of 64 x 64 the pipelined tile that needs fewer rounds (two 128 x
// 128 workgroups share a CU and take as long as one of 256 x 256).  But:
//
// K <= 1536: stores (and C, where it is added to) take as long as the products, and of two
// workgroups on a CU one stores while the other multiplies.  There 128 x 128 unless
// it needs twice the rounds.  128 x 128 over 256 x 256, in time, 39 sizes with more rounds but
// less than twice: K 1152 0.72 - 0.97, 1536 0.75 - 1.01, 1920 0.77 - 1.09, 2240 0.83 - 1.16
// (onto C 0.72 - 0.95, 0.75 - 0.96, 0.78 - 0.98, 0.83 - 1.04); with twice the rounds 0.83 - 1.10 at
// 1152, 0.86 - 1.14 at 1536.  For the residual, which moves 8 bytes an element and has the
// most work besides, at any number of rounds: the calibration step by 256 x 256 and 128 x
// 128 tiles, us: 9216 x 512 x 2048 158, 147; 6000 x 1024 x 2900 223, 204; 4096 x 1152 x 4608
// 271, 259; 18432 x 1152 x 3072 626, 614; 8192 x 1536 x 3072 387, 381; 18432 x 3072 x 3072 1295, 1300.
// K <= 128, a single stage: 128 x 128 always (0.79 - 1.03).
//
// N <= 32 with more than 256 tiles of 32 x 32 (C is four times narrower than a 128 x 128
// tile): 32 x 32 tiles of two waves, many on a CU.  Not the residual, whose sums of
// squares have room for one a tile of 64 x 64.  128 x 128 and so, us, K 64 / 480 / 1152 /
// 3072: 18432 x 32 4.2 / 5.5 / 6.8 / 12.2 and 3.8 / 4.3 / 5.7 / 15.6; 70000 x 8 onto C
// 11.1 / 14.5 / 20.3 / 33.9 and 6.7 / 8.0 / 13.5 / 33.7.
enum class GemmTile { Thin32, Split32, Split32x64, Split64, Pipe128, Pipe256 };

static GemmTile gemm_tile_of(const GemmParams& g) {
    auto tiles = [&](int64_t tm, int64_t tn) { return ((g.M + tm - 1) / tm) * ((g.N + tn - 1) / tn); };
    if (tiles(32, 32) <= 256) return GemmTile::Split32;
    if (g.N <= 32 && g.K <= 1152 && !g.rh) return GemmTile::Thin32;
    if (tiles(32, 64) <= 256) return GemmTile::Split32x64;
    if (tiles(64, 64) <= 256 || g.K > kPipeMaxK) return GemmTile::Split64;
    const int64_t rounds128 = (tiles(128, 128) + 511) / 512, rounds256 = (tiles(256, 256) + 255) / 256;
    if (g.K <= 1536 && (g.rh || rounds128 < 2 * rounds256)) return GemmTile::Pipe128;
    return g.K <= 128 || rounds128 <= rounds256 ? GemmTile::Pipe128 : GemmTile::Pipe256;
}

int64_t mxfp4_gemm_workgroups(const GemmParams& g) {
    auto tiles = [&](int64_t tm, int64_t tn) { return ((g.M + tm - 1) / tm) * ((g.N + tn - 1) / tn); };
    switch (gemm_tile_of(g)) {
        case GemmTile::Thin32:
        case GemmTile::Split32: return tiles(32, 32);
        case GemmTile::Split32x64: return tiles(32, 64);
        case GemmTile::Split64: return tiles(64, 64);
        case GemmTile::Pipe128: return tiles(128, 128);
        default: return tiles(256, 256);
    }
}

template <int TN, int TM, int W, int D>
static void launch_split(const GemmParams& g, hipStream_t st) {
    const int64_t gx = (g.N + 32 * TN - 1) / (32 * TN), gy = (g.M + 32 * TM - 1) / (32 * TM);
    hipLaunchKernelGGL((mxfp4_gemm_split_kernel<TN, TM, W, D>), dim3((unsigned)(gx * gy)), dim3(64 * W), 0, st, g, gx, gy);
}

template <int WN, int WM, int TN, int TM, bool PING, bool DMA_SCALES>
static void launch_pipe_out(const GemmParams& g, hipStream_t st) {
    typedef Tile<WN, WM, TN, TM> T;
    const int64_t gx = (g.N + T::BN - 1) / T::BN, gy = (g.M + T::BM - 1) / T::BM;
    const dim3 grid((unsigned)(gx * gy)), b(64 * T::WAVES);
#define KQ_PIPE(OUT, BASE) \
    hipLaunchKernelGGL((mxfp4_gemm_pipe_kernel<WN, WM, TN, TM, PING, DMA_SCALES, OUT, BASE>), grid, b, 0, st, g, gx, gy)
    if (g.C16) KQ_PIPE(1, false);
    else if (g.rh) KQ_PIPE(2, true);
    else if (g.bias || g.accumulate) KQ_PIPE(0, true);
    else KQ_PIPE(0, false);
#undef KQ_PIPE
}

template <int WN, int WM, int TN, int TM, bool PING>
static void launch_pipe(const GemmParams& g, hipStream_t st) {
    const int64_t nkb = g.K / 32;
    if (nkb % 4 == 0 && nkb >= 16 && g.scales_aligned) launch_pipe_out<WN, WM, TN, TM, PING, true>(g, st);
    else launch_pipe_out<WN, WM, TN, TM, PING, false>(g, st);
}

hipError_t launch_mxfp4_gemm(const GemmParams& g, hipStream_t st) {
    switch (gemm_tile_of(g)) {
        case GemmTile::Thin32: launch_split<1, 1, 2, 4>(g, st); break;
        case GemmTile::Split32: launch_split<1, 1, 8, 4>(g, st); break;
        case GemmTile::Split32x64: launch_split<2, 1, 8, 3>(g, st); break;
        case GemmTile::Split64: launch_split<2, 2, 8, 2>(g, st); break;
        case GemmTile::Pipe128: launch_pipe<2, 2, 2, 2, false>(g, st); break;
        case GemmTile::Pipe256: launch_pipe<2, 4, 4, 2, true>(g, st); break;
    }
    return hipGetLastError();
}

}  // namespace kq
