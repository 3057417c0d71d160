// W4A4 linear layers: the MXFP4 product with what follows it in its epilogue,
//     out = residual + gate act(deq(A) deq(B)^T + bias),
// and the same product grouped by expert, rows gathered and weighted,
//     out[r] = row_scale[r] act(deq(A)[rows[r]] deq(B_e)^T + bias_e),
// where expert e has the rows offsets[e] .. offsets[e + 1] - 1.  Products are
// exact, sums and the epilogue are in 32 bits, out is rounded once.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kq_act.h"
#include "kq_gemm_tile.h"
#include "kq_linear.h"
#include "kq_place.h"

namespace kq {

// Lambdas over the parameters: one that is called keeps them in scratch memory.
#define KQ_INLINE __attribute__((always_inline))

typedef float f32x4m __attribute__((ext_vector_type(4)));

namespace {

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }

// V (a multiple of 4) values of a bf16 or fp32 array from element `at`, the first `n` of them; zeros past.
template <int V>
__device__ __forceinline__ void load_values(const void* p, int is16, int64_t at, int n, float (&v)[V]) {
    if (is16) {
        const uint16_t* const q = static_cast<const uint16_t*>(p) + at;
        if (n >= V) {
#pragma unroll
            for (int k = 0; k < V; k += 4) {
                const u32x2b w = *reinterpret_cast<const u32x2b*>(q + k);
                v[k] = __uint_as_float(w.x << 16);
                v[k + 1] = __uint_as_float(w.x & 0xffff0000u);
                v[k + 2] = __uint_as_float(w.y << 16);
                v[k + 3] = __uint_as_float(w.y & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = k < n ? bf16_value(q[k]) : 0.f;
        }
    } else {
        const float* const q = static_cast<const float*>(p) + at;
        if (n >= V) {
#pragma unroll
            for (int k = 0; k < V; k += 4) {
                const f32x4 w = *reinterpret_cast<const f32x4*>(q + k);
                v[k] = w.x;
                v[k + 1] = w.y;
                v[k + 2] = w.z;
                v[k + 3] = w.w;
            }
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = k < n ? q[k] : 0.f;
        }
    }
}

// *q = v; PAST: past the caches, which would not keep it.
template <bool PAST, class T>
__device__ __forceinline__ void put(T* q, T v) {
    if constexpr (PAST) __builtin_nontemporal_store(v, q);
    else *q = v;
}

// The first n of V values to a bf16 or fp32 array.
template <int V, bool PAST = false>
__device__ __forceinline__ void store_values(void* p, int is16, int64_t at, int n, const float (&v)[V]) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    if (is16) {
        uint16_t* const q = static_cast<uint16_t*>(p) + at;
        uint32_t w[V / 2];
#pragma unroll
        for (int k = 0; k < V / 2; ++k) w[k] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)v[2 * k], (__bf16)v[2 * k + 1]});
        if (n >= V) {
            if constexpr (V == 8) put<PAST>(reinterpret_cast<u32x4b*>(q), u32x4b{w[0], w[1], w[2], w[3]});
            else if constexpr (V == 4) put<PAST>(reinterpret_cast<u32x2b*>(q), u32x2b{w[0], w[1]});
            else *reinterpret_cast<u32b*>(q) = w[0];
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k < n) q[k] = (uint16_t)(w[k / 2] >> (16 * (k & 1)));
        }
    } else {
        float* const q = static_cast<float*>(p) + at;
        if (n >= V) {
            typedef float f32x2 __attribute__((ext_vector_type(2), aligned(4)));
            if constexpr (V == 2) *reinterpret_cast<f32x2*>(q) = f32x2{v[0], v[1]};
            else
#pragma unroll
                for (int k = 0; k < V; k += 4) put<PAST>(reinterpret_cast<f32x4*>(q + k), f32x4{v[k], v[k + 1], v[k + 2], v[k + 3]});
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k < n) q[k] = v[k];
        }
    }
}

// V sums of row m from column n (v; `have` columns of them inside N) to the output: the epilogue where
// everything is loaded as it is needed.
template <Act A, int V>
__device__ __forceinline__ void finish(const LinearParams& p, int64_t m, int64_t n, int have, float (&v)[V]) {
    if (p.bias) {
        float b[V];
        load_values<V>(p.bias, p.vec16, n, have, b);
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] += b[k];
    }
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = A == Act::Swiglu && (k & 1) ? v[k] : activate<A>(v[k]);
    const float rs = p.row_scale ? p.row_scale[m] : 1.0f;
    constexpr int VO = A == Act::Swiglu ? V / 2 : V;
    const int64_t c = A == Act::Swiglu ? n / 2 : n;
    const int nc = A == Act::Swiglu ? have / 2 : have;
    float o[VO];
#pragma unroll
    for (int k = 0; k < VO; ++k) o[k] = A == Act::Swiglu ? v[2 * k] * v[2 * k + 1] : v[k];
    if (p.row_scale) {
#pragma unroll
        for (int k = 0; k < VO; ++k) o[k] *= rs;
    }
    if constexpr (VO >= 4) {
        if (p.gate) {
            float g[VO];
            load_values<VO>(p.gate, p.vec16, m / p.gate_rows * p.gate_stride + c, nc, g);
#pragma unroll
            for (int k = 0; k < VO; ++k) o[k] *= g[k];
        }
        if (p.residual) {
            float r[VO];
            load_values<VO>(p.residual, p.out16, m * p.ldr + c, nc, r);
#pragma unroll
            for (int k = 0; k < VO; ++k) o[k] += r[k];
        }
    } else {
        auto at = [&](const void* q, int is16, int64_t i) {
            return is16 ? bf16_value(static_cast<const uint16_t*>(q)[i]) : static_cast<const float*>(q)[i];
        };
#pragma unroll
        for (int k = 0; k < VO; ++k) {
            if (k >= nc) break;
            if (p.gate) o[k] *= at(p.gate, p.vec16, m / p.gate_rows * p.gate_stride + c + k);
            if (p.residual) o[k] += at(p.residual, p.out16, m * p.ldr + c + k);
        }
    }
    store_values<VO>(p.out, p.out16, m * p.ldo + c, nc, o);
}

}  // namespace

// V values of a bf16 or fp32 array as they are stored (bf16: the first V / 2 words).
template <int V>
__device__ __forceinline__ void load_stored(const void* p, int is16, int64_t at, uint32_t (&w)[V]) {
    typedef uint32_t u32x4f __attribute__((ext_vector_type(4), aligned(4)));
    if (is16) {
        const uint16_t* const q = static_cast<const uint16_t*>(p) + at;
        if constexpr (V == 8) {
            const u32x4b v = *reinterpret_cast<const u32x4b*>(q);
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = v[k];
        } else {
            const u32x2b v = *reinterpret_cast<const u32x2b*>(q);
            w[0] = v.x;
            w[1] = v.y;
        }
    } else {
        const uint32_t* const q = static_cast<const uint32_t*>(p) + at;
#pragma unroll
        for (int k = 0; k < V; k += 4) {
            const u32x4f v = *reinterpret_cast<const u32x4f*>(q + k);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[k + e] = v[e];
        }
    }
}
template <int V>
__device__ __forceinline__ float stored_value(const uint32_t (&w)[V], int is16, int k) {
    return __uint_as_float(!is16 ? w[k] : k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16);
}

// The pipelined tile's sums to the output, through LDS in fp32 so that the output and the residual are
// accessed along their rows.  A thread keeps its eight columns: the bias is loaded once a pass, and the gate
// where the tile's rows are of one batch.  The residual's and the router's loads of a pass are issued before its
// stores (a wait for a load waits for every store issued before it too).
template <int WN, int WM, int TN, int TM, bool GROUPED>
__device__ __forceinline__ void finish_tile(const LinearParams& p, uint8_t* lds, int64_t nb0, int64_t mb0,
                                            const f32x16g (&acc)[TN][TM]) {
    typedef Tile<WN, WM, TN, TM> T;
    constexpr int NP = (T::BM * (T::BN * 4 + 16) <= (int)sizeof(typename T::Lds)) ? 1 : 2;
    constexpr int TP = TN / NP, RB = T::BN / NP * 4, RS = RB + 16;
    static_assert(T::BM * RS <= (int)sizeof(typename T::Lds), "a pass fits LDS");
    constexpr int V = 8, CPR = RB / (4 * V), STEP = 64 * T::WAVES / CPR, CH = T::BM / STEP;
    static_assert(32 * TP % V == 0 && 64 * T::WAVES % CPR == 0, "a thread keeps its columns, inside one wave's range");
    const int t = threadIdx.x;
    const int wave = t >> 6, lane = t & 63;
    const int r = lane & 31, h = lane >> 5, wn = wave / WM, wm = wave % WM;
    const int last = (int)min<int64_t>(T::BM, p.g.M - mb0) - 1;
    const int trow = t / CPR, cl = t % CPR * V, seg = cl / (32 * TP);
    const bool one_gate = !GROUPED && p.gate && mb0 / p.gate_rows == (mb0 + last) / p.gate_rows;
    auto one_pass = [&](auto which) KQ_INLINE {
        constexpr int pass = decltype(which)::value;
        const int64_t n = nb0 + seg * 32 * TN + 32 * pass * TP + (cl - seg * 32 * TP);
        const int have = (int)max<int64_t>(0, min<int64_t>(V, p.g.N - n));
        if (pass > 0) __syncthreads();
#pragma unroll
        for (int i = 0; i < TP; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                uint8_t* const dst = lds + (32 * (wm * TM + j) + r) * RS + (32 * (wn * TP + i) + 4 * h) * 4;
                const f32x16g& c = acc[pass * TP + i][j];
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<float4*>(dst + 32 * q) = make_float4(c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]);
            }
        __builtin_amdgcn_sched_barrier(0);  // the pass's accumulators are free for what is loaded
        const uint8_t* const from = lds + trow * RS + 4 * cl;
        with_act(p.act, [&](auto act) KQ_INLINE {
            constexpr Act A = decltype(act)::value;
            constexpr int VO = A == Act::Swiglu ? V / 2 : V;
            const int64_t c = A == Act::Swiglu ? n / 2 : n;
            float bias[V], gate[VO], scale[GROUPED ? CH : 1];
            uint32_t res[GROUPED ? 1 : CH][VO];
#pragma unroll
            for (int k = 0; k < V; ++k) bias[k] = 0.f;
            if (have == V) {
                if (p.bias) load_values<V>(p.bias, p.vec16, n, V, bias);
                if (GROUPED) {
                    if (p.row_scale) {
#pragma unroll
                        for (int k = 0; k < CH; ++k) scale[GROUPED ? k : 0] = p.row_scale[mb0 + min(trow + k * STEP, last)];
                    }
                } else {
                    if (one_gate) load_values<VO>(p.gate, p.vec16, mb0 / p.gate_rows * p.gate_stride + c, VO, gate);
                    if (p.residual) {  // rows past M load the last one again
#pragma unroll
                        for (int k = 0; k < CH; ++k)
                            load_stored<VO>(p.residual, p.out16, (mb0 + min(trow + k * STEP, last)) * p.ldr + c, res[GROUPED ? 0 : k]);
                    }
                }
            }
            __syncthreads();
            if (have < V) {
                if (have > 0)
                    for (int k = 0; k < CH && trow + k * STEP <= last; ++k) {
                        float v[V];
#pragma unroll
                        for (int e = 0; e < V; ++e) v[e] = reinterpret_cast<const float*>(from + k * STEP * RS)[e];
                        finish<A, V>(p, mb0 + trow + k * STEP, n, have, v);
                    }
                return;
            }
            auto rows = [&](auto past) KQ_INLINE {
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    if (trow + k * STEP > last) break;
                    const int64_t m = mb0 + trow + k * STEP;
                    const float4 a = *reinterpret_cast<const float4*>(from + k * STEP * RS);
                    const float4 b = *reinterpret_cast<const float4*>(from + k * STEP * RS + 16);
                    const float v[V] = {a.x + bias[0], a.y + bias[1], a.z + bias[2], a.w + bias[3],
                                        b.x + bias[4], b.y + bias[5], b.z + bias[6], b.w + bias[7]};
                    float o[VO];
#pragma unroll
                    for (int e = 0; e < VO; ++e) o[e] = A == Act::Swiglu ? activate<A>(v[2 * e]) * v[2 * e + 1] : activate<A>(v[e]);
                    if (GROUPED) {
                        if (p.row_scale) {
#pragma unroll
                            for (int e = 0; e < VO; ++e) o[e] *= scale[GROUPED ? k : 0];
                        }
                    } else {
                        if (p.gate) {
                            if (!one_gate) load_values<VO>(p.gate, p.vec16, m / p.gate_rows * p.gate_stride + c, VO, gate);
#pragma unroll
                            for (int e = 0; e < VO; ++e) o[e] *= gate[e];
                        }
                        if (p.residual) {
#pragma unroll
                            for (int e = 0; e < VO; ++e) o[e] += stored_value<VO>(res[GROUPED ? 0 : k], p.out16, e);
                        }
                    }
                    store_values<VO, decltype(past)::value>(p.out, p.out16, m * p.ldo + c, VO, o);
                }
            };
            if (p.stream_out) rows(std::true_type{});
            else rows(std::false_type{});
        });
    };
    one_pass(std::integral_constant<int, 0>{});
    if constexpr (NP > 1) one_pass(std::integral_constant<int, 1>{});
}

template <int WN, int WM, int TN, int TM, bool PING, bool DMA_SCALES, bool GROUPED, bool GATHER>
__global__ __launch_bounds__(64 * WN * WM) void mxfp4_linear_pipe_kernel(LinearParams p) {
    typedef Tile<WN, WM, TN, TM> T;
    __shared__ typename T::Lds lds;
    int64_t nb0, mb0;
    if (!place<GROUPED>(p, T::BN, T::BM, nb0, mb0)) return;
    f32x16g acc[TN][TM];
    gemm_tile<WN, WM, TN, TM, PING, DMA_SCALES, GATHER>(p.g, lds, nb0, mb0, acc);
    finish_tile<WN, WM, TN, TM, GROUPED>(p, reinterpret_cast<uint8_t*>(&lds), nb0, mb0, acc);
}

// Few tiles of more than a few rows: W waves share a tile and split K.
template <int TN, int TM, int W, int D, bool GROUPED, bool GATHER>
__global__ __launch_bounds__(64 * W) void mxfp4_linear_split_kernel(LinearParams p) {
    constexpr int BN = 32 * TN, BM = 32 * TM, RS = BN + 4;
    __shared__ float sums[W * BM * RS];
    int64_t nb0, mb0;
    if (!place<GROUPED>(p, BN, BM, nb0, mb0)) return;
    const int active = split_tile<TN, TM, W, D, GATHER>(p.g, sums, nb0, mb0);
    with_act(p.act, [&](auto act) KQ_INLINE {
        for (int k = threadIdx.x; k < BM * BN / 4; k += 64 * W) {
            const int row = k / (BN / 4), col = 4 * (k % (BN / 4));
            const int64_t m = mb0 + row, n = nb0 + col;
            if (m >= p.g.M || n >= p.g.N) continue;
            float4 s = *reinterpret_cast<const float4*>(sums + row * RS + col);
            for (int w = 1; w < active; ++w) {
                const float4 o = *reinterpret_cast<const float4*>(sums + (w * BM + row) * RS + col);
                s = make_float4(s.x + o.x, s.y + o.y, s.z + o.z, s.w + o.w);
            }
            float v[4] = {s.x, s.y, s.z, s.w};
            finish<decltype(act)::value, 4>(p, m, n, (int)min<int64_t>(4, p.g.N - n), v);
        }
    });
}

// A few rows (a decoding step): the weight is read once and bounds the call (64 experts of 2048 x 2816, a row each,
// 196 MB: 43 us, 4.5 TB/s; one row through 3072 x 12288, 20 MB: 7.2 us, of which an empty launch is 3).  A tile is 16 TM rows of A
// by 16 of B; v_mfma_scale_f32_16x16x128_f8f6f4 takes lane l's 16 code bytes as row l % 16, block l / 16
// of the 128-wide K step, so fragments are plain loads.  WN waves have a tile each, next to each other
// along N, and WK waves split each tile's K, in units of 256 (whole 128-byte lines of B), D units in flight;
// their sums meet in LDS in wave order.
template <int TM, int WN, int WK, int D, bool GROUPED, bool GATHER>
__global__ __launch_bounds__(64 * WN * WK) void mxfp4_linear_rows_kernel(LinearParams p) {
    constexpr int BM = 16 * TM, BN = 16 * WN, RS = 20;  // LDS row in floats
    __shared__ float sums[WN * WK * BM * RS];
    int64_t nb0, mb0;
    if (!place<GROUPED>(p, BN, BM, nb0, mb0)) return;
    const GemmParams& g = p.g;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wn = wave / WK, wk = wave % WK, r = lane & 15, b = lane >> 4;
    const int64_t nkb = g.K / 32, row_bytes = g.K / 2, units = (nkb + 7) / 8;
    const int64_t nrow = min(nb0 + 16 * wn + r, g.N - 1);  // rows past N or M read the last row
    const uint8_t *cw = g.b_codes + nrow * row_bytes, *sw = g.b_scales + nrow * nkb, *cx[TM], *sx[TM];
#pragma unroll
    for (int j = 0; j < TM; ++j) {
        int64_t m = min(mb0 + 16 * j + r, g.M - 1);
        if (GATHER) m = gathered(g, m);
        cx[j] = g.a_codes + m * row_bytes;
        sx[j] = g.a_scales + m * nkb;
    }
    struct Unit {
        uint4 w[2], x[2][TM];
        uint2 sw, sx[TM];  // the row's eight scales
    };
    auto scales = [&](const uint8_t* q, int64_t u) {
        typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(1)));
        if (8 * u + 8 <= nkb) {
            const u32x2u v = *reinterpret_cast<const u32x2u*>(q + 8 * u);
            return make_uint2(v.x, v.y);
        }
        // the last unit of a K that ends inside it: this lane's two blocks (the last one's for those past K)
        const int64_t k = 8 * u + b;
        return make_uint2((uint32_t)q[min(k, nkb - 1)] << (8 * b), (uint32_t)q[min(k + 4, nkb - 1)] << (8 * b));
    };
    auto load = [&](int64_t u, Unit& f) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int64_t k = min(8 * u + 4 * s + b, nkb - 1);  // blocks past K read the last one; masked below
            f.w[s] = *reinterpret_cast<const uint4*>(cw + 16 * k);
#pragma unroll
            for (int j = 0; j < TM; ++j) f.x[s][j] = *reinterpret_cast<const uint4*>(cx[j] + 16 * k);
        }
        f.sw = scales(sw, u);
#pragma unroll
        for (int j = 0; j < TM; ++j) f.sx[j] = scales(sx[j], u);
    };
    f32x4m acc[TM];
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[j] = f32x4m{};
    auto multiply = [&](int64_t u, Unit& f) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            uint32_t w = (s ? f.sw.y : f.sw.x) >> (8 * b);
            const bool past = 8 * u + 4 * s + b >= nkb;  // zero codes, scale 1
            if (past) {
                f.w[s] = make_uint4(0u, 0u, 0u, 0u);
                w = 127u;
            }
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                const uint32_t x = past ? 127u : (s ? f.sx[j].y : f.sx[j].x) >> (8 * b);
                acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(Frag{f.w[s], 0u}), operand(Frag{f.x[s][j], 0u}),
                                                                          acc[j], 4, 4, 0, (int)w, 0, (int)x);
            }
        }
    };
    Unit f[D];
#pragma unroll
    for (int i = 0; i < D; ++i)
        if (wk + i * WK < units) load(wk + i * WK, f[i]);
    for (int64_t u = wk; u < units; u += D * WK) {
#pragma unroll
        for (int i = 0; i < D; ++i) {
            const int64_t v = u + i * WK;
            if (v < units) {
                multiply(v, f[i]);
                if (v + D * WK < units) load(v + D * WK, f[i]);
            }
        }
    }
    // acc[j][e]: row 16 j + r of A, row 4 b + e of B
#pragma unroll
    for (int j = 0; j < TM; ++j)
        *reinterpret_cast<float4*>(sums + ((wn * WK + wk) * BM + 16 * j + r) * RS + 4 * b) =
            make_float4(acc[j][0], acc[j][1], acc[j][2], acc[j][3]);
    __syncthreads();
    with_act(p.act, [&](auto act) KQ_INLINE {
        for (int k = threadIdx.x; k < WN * BM * 4; k += 64 * WN * WK) {
            const int c = k % (4 * WN), row = k / (4 * WN);
            const int64_t m = mb0 + row, n = nb0 + 4 * c;
            if (m >= g.M || n >= g.N) continue;
            const float* const from = sums + (c / 4 * WK * BM + row) * RS + 4 * (c % 4);
            float4 s = *reinterpret_cast<const float4*>(from);
#pragma unroll
            for (int w = 1; w < WK; ++w) {
                const float4 o = *reinterpret_cast<const float4*>(from + w * BM * RS);
                s = make_float4(s.x + o.x, s.y + o.y, s.z + o.z, s.w + o.w);
            }
            float v[4] = {s.x, s.y, s.z, s.w};
            finish<decltype(act)::value, 4>(p, m, n, (int)min<int64_t>(4, g.N - n), v);
        }
    });
}

constexpr int64_t kPipeMaxK = int64_t(1) << 24;  // 32-bit offsets within a tile

// Row tiles that a call can need.
static int64_t row_tiles(const LinearParams& p, int64_t bm) {
    return p.offsets ? group_tiles(p.g.M, p.experts, bm) : (p.g.M + bm - 1) / bm;
}

// K of a tile of a few rows is split over as many waves as it takes to have about this many, 22 on a CU.
constexpr int64_t kRowsWaves = 22 * 256;
// Tiles of bm rows that have work: a group of a few rows is one.
static int64_t rows_tiles(const LinearParams& p, int64_t bm) {
    return (p.g.N + 15) / 16 * (p.offsets ? std::min(p.experts, p.g.M) : (p.g.M + bm - 1) / bm);
}

// Tile of a call.  Measured, us (bf16 out, weights not in the caches).
// A few rows, K x N 3072 x 12288 / 12288 x 3072 / 1152 x 4608: tiles of 16 (32) rows and what splits K otherwise (64 x 64,
// 32 x 32, 32 x 32): 1 row 7.2, 9.0, 4.2 and 10.6, 14.8, 4.0; 16 rows 9.0, 12.5, 4.5 and 11.5, 20.5, 4.2; 32 rows
// 12.0, 16.6, 4.9 and 12.5, 25.9, 4.4; 64 rows 22.5, 26.2, 6.8 (tiles of 64 rows, not kept) and 15.3, 23.9, 6.1.
// Waves that split K, 8, 4, 2, 1: 1 row 8.2, 7.2, 8.8, 13.0; 9.0, 11.8, 20.1, 47.0; 8 of 64 experts of 2048 x 2816, a row
// each 13.5, 9.6, 9.0, 12.2; all 64 93, 57.1, 45.8, 43.3; 8 experts of 2240 x 5600, 2 rows each -, 17.6, 17.2, 17.4.
// Workgroups of 8 waves where these have 4: 1 row 8.1 for 7.2; 8 tokens with 8 of 64 experts each 28.8 for 27.6.
// Grouped, tiles of 16 rows and 128 x 128: 64 experts of 2048 x 2816, 1, 2, 4, 8 rows an expert 43.3, 44.6, 47.1, 51.0
// and 51.2, 48.0, 49.3, 50.8 (tiles that split K: 66.6 at 1 row); 8 experts of 2240 x 5600, 1, 2, 4, 8, 16 rows
// 17.2, 17.2, 17.5, 17.8, 20.0 and 21.9, 21.9, 22.1, 22.2, 22.7: the rule's 2 and 8 rows are below where the two meet.
// More rows: as mxfp4_gemm's tiles; 128 x 128 and 256 x 256, grouped 32 experts 12004 x 1152 x 2240 fp32 61, 76,
// 16 experts 16384 x 2240 x 5600 224, 203.
enum class LinearTile { Rows16, Rows32, Split32, Split64, Pipe128, Pipe256 };

static LinearTile linear_tile_of(const LinearParams& p) {
    const GemmParams& g = p.g;
    auto tiles = [&](int64_t tm, int64_t tn) { return row_tiles(p, tm) * ((g.N + tn - 1) / tn); };
    // gathered pipelined tiles have 32-bit offsets into all of A
    const bool pipe = g.K <= kPipeMaxK && (!g.rows || g.a_rows <= (int64_t(1) << 32) / (g.K / 2));
    if (p.offsets) {
        if (g.M <= p.experts * (rows_tiles(p, 16) <= kRowsWaves ? 8 : 2)) return LinearTile::Rows16;
    } else {
        if (g.M <= 16) return LinearTile::Rows16;
        if (g.M <= 32 && g.K > 4096) return LinearTile::Rows32;
    }
    if (tiles(32, 32) <= 256) return LinearTile::Split32;
    if (tiles(64, 64) <= 256 || !pipe) return LinearTile::Split64;
    const int64_t rounds128 = (tiles(128, 128) + 511) / 512, rounds256 = (tiles(256, 256) + 255) / 256;
    if (g.K <= 1536 && rounds128 < 2 * rounds256) return LinearTile::Pipe128;
    return g.K <= 128 || rounds128 <= rounds256 ? LinearTile::Pipe128 : LinearTile::Pipe256;
}

// Calls f(std::integral_constant<bool, GROUPED>, std::integral_constant<bool, GATHER>).
template <class F>
static void by_group(const LinearParams& p, F f) {
    if (!p.offsets) f(std::false_type{}, std::false_type{});
    else if (!p.g.rows) f(std::true_type{}, std::false_type{});
    else f(std::true_type{}, std::true_type{});
}

// Whether a launch holds that many workgroups: a grid's threads are counted in 32 bits, and past them HIP starts fewer
// workgroups, without an error.
static bool one_launch(int64_t groups, int64_t threads) { return groups <= int64_t(UINT32_MAX) / threads; }

template <int TM, int WN, int WK, int D>
static hipError_t launch_rows(const LinearParams& p, hipStream_t st) {
    const int64_t groups = (p.g.N + 16 * WN - 1) / (16 * WN) * row_tiles(p, 16 * TM);
    if (!one_launch(groups, 64 * WN * WK)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)groups);
    by_group(p, [&](auto grouped, auto gather) {
        hipLaunchKernelGGL((mxfp4_linear_rows_kernel<TM, WN, WK, D, decltype(grouped)::value, decltype(gather)::value>), grid,
                           dim3(64 * WN * WK), 0, st, p);
    });
    return hipGetLastError();
}

template <int TM, int D>
static hipError_t launch_rows_by_waves(const LinearParams& p, hipStream_t st) {
    const int64_t split = std::min(kRowsWaves / rows_tiles(p, 16 * TM), (p.g.K + 255) / 256);
    if (split >= 8) return launch_rows<TM, 1, 8, D>(p, st);
    if (split >= 4) return launch_rows<TM, 1, 4, D>(p, st);
    if (split >= 2) return launch_rows<TM, 2, 2, D>(p, st);
    return launch_rows<TM, 4, 1, D>(p, st);
}

template <int TN, int TM, int W, int D>
static hipError_t launch_split(const LinearParams& p, hipStream_t st) {
    const int64_t groups = (p.g.N + 32 * TN - 1) / (32 * TN) * row_tiles(p, 32 * TM);
    if (!one_launch(groups, 64 * W)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)groups);
    by_group(p, [&](auto grouped, auto gather) {
        hipLaunchKernelGGL((mxfp4_linear_split_kernel<TN, TM, W, D, decltype(grouped)::value, decltype(gather)::value>), grid,
                           dim3(64 * W), 0, st, p);
    });
    return hipGetLastError();
}

template <int WN, int WM, int TN, int TM, bool PING>
static hipError_t launch_pipe(const LinearParams& p, hipStream_t st) {
    typedef Tile<WN, WM, TN, TM> T;
    const int64_t groups = (p.g.N + T::BN - 1) / T::BN * row_tiles(p, T::BM);
    if (!one_launch(groups, 64 * T::WAVES)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)groups);
    const int64_t nkb = p.g.K / 32;
    const bool dma = nkb % 4 == 0 && nkb >= 16 && p.g.scales_aligned;
    by_group(p, [&](auto grouped, auto gather) {
        constexpr bool GR = decltype(grouped)::value, GA = decltype(gather)::value;
        if (dma) hipLaunchKernelGGL((mxfp4_linear_pipe_kernel<WN, WM, TN, TM, PING, true, GR, GA>), grid, dim3(64 * T::WAVES), 0, st, p);
        else hipLaunchKernelGGL((mxfp4_linear_pipe_kernel<WN, WM, TN, TM, PING, false, GR, GA>), grid, dim3(64 * T::WAVES), 0, st, p);
    });
    return hipGetLastError();
}

int64_t mxfp4_grouped_workgroups(const LinearParams& p) { return (p.g.N + 15) / 16 * row_tiles(p, 16); }

// Bytes that a call reads and writes.
static int64_t touched(const LinearParams& p) {
    const int64_t cols = p.act == Act::Swiglu ? p.g.N / 2 : p.g.N, out = p.g.M * cols * (p.out16 ? 2 : 4);
    const int64_t weights = p.offsets ? std::min(p.experts, p.g.M) : 1;
    return (std::min(p.g.rows ? p.g.a_rows : p.g.M, p.g.M) + weights * p.g.N) * (p.g.K / 2) + (p.residual ? 2 : 1) * out;
}

hipError_t launch_mxfp4_linear(LinearParams p, hipStream_t st) {
    // Half of the 256 MB memory-side cache: past it an output that is kept there drives out what the next tiles
    // read.  us, kept and not: grouped 12004 x 1152 x 2240 fp32 with 32 experts (159 MB) 72, 52; 4608 x 3072 x 12288
    // (141 MB) 140, 132; 12004 x 1152 x 2240 fp32, one weight (115 MB), onto the same output each time 46, 54.
    p.stream_out = touched(p) > (int64_t(128) << 20);
    switch (linear_tile_of(p)) {
        case LinearTile::Rows16: return launch_rows_by_waves<1, 3>(p, st);
        case LinearTile::Rows32: return launch_rows_by_waves<2, 3>(p, st);
        case LinearTile::Split32: return launch_split<1, 1, 8, 4>(p, st);
        case LinearTile::Split64: return launch_split<2, 2, 8, 2>(p, st);
        case LinearTile::Pipe128: return launch_pipe<2, 2, 2, 2, false>(p, st);
        case LinearTile::Pipe256: break;
    }
    return launch_pipe<2, 4, 4, 2, true>(p, st);
}

}  // namespace kq
