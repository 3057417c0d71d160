// A paged cache of keys and values, quantized as it is written, and read back.
// A block of 32 values shares a scale 2^s, s = floor(log2 max|x|) - m, m = 2
// for E2M1 and 8 for E4M3 elements; values round to the nearest element, ties
// to even, and saturate.  A bf16 cache rounds values once.
//
// Four lanes of eight values hold a block; its maximum is two exchanges
// between them.  Bound by HBM: a value is read and written once.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "kq_mx.h"
#include "kq_serve.h"

namespace kq {

namespace {

constexpr int kCacheThreads = 256;

// Eight values of a row, at any alignment of their elements.
__device__ __forceinline__ void load8(const void* p, int is16, int64_t at, float (&v)[8]) {
    if (is16) {
        typedef uint32_t W __attribute__((ext_vector_type(4), aligned(2)));
        const W w = *reinterpret_cast<const W*>(static_cast<const uint16_t*>(p) + at);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k] = bf16_low(w[k]);
            v[2 * k + 1] = bf16_high(w[k]);
        }
    } else {
        typedef float W __attribute__((ext_vector_type(4), aligned(4)));
        const W a = *reinterpret_cast<const W*>(static_cast<const float*>(p) + at);
        const W b = *reinterpret_cast<const W*>(static_cast<const float*>(p) + at + 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[k] = a[k];
            v[4 + k] = b[k];
        }
    }
}

// The largest of four neighbouring lanes' values.
__device__ __forceinline__ float quad_max(float v) {
    v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0xb1, 0xf, 0xf, false)));  // lane ^ 1
    return fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x4e, 0xf, 0xf, false)));  // lane ^ 2
}

// How a call's eights of values are shared out: in order of token, half (keys, values), head and column; `in` counts those
// of a workgroup's tokens.  (In order of head first, whose codes and scales are whole lines of the cache, 32768 tokens of
// 8 x 128 in MXFP8 took 48 us to read for 38, 8191 18.4 to write for 17.0.)  Divisions are multiplications by 2^32 / n,
// rounded up: exact for `in` below 2048 by `each` up to 1024 (where a workgroup has several tokens), and below 2^21 by up
// to 32 columns of eight.
struct Shares {
    int tokens;      // of a workgroup
    int each, half;  // eights of a token, and of one of its halves
    uint32_t by_each, by_columns;
};
struct Eight {
    int token, head, column;
    bool value;
    __device__ __forceinline__ Eight(const Cache& c, const Shares& sh, int in) {
        token = sh.tokens > 1 ? (int)__umulhi((uint32_t)in, sh.by_each) : 0;
        const int r = in - token * sh.each;
        value = r >= sh.half;
        const int s = value ? r - sh.half : r;
        head = (int)__umulhi((uint32_t)s, sh.by_columns);
        column = 8 * (s - head * (c.d / 8));
    }
};

// The cache's row of a slot, -1 for one outside the cache.
__device__ __forceinline__ int64_t cache_row(const Cache& c, int64_t slot, int head) {
    if (slot < 0 || slot >= c.pages * c.page_size) return -1;
    return (((slot >> c.page_shift) * c.heads + head) << c.page_shift) + (slot & (c.page_size - 1));
}

// A thread's eights of a turn: their loads are in flight together.
constexpr int kAtOnce = 4;

template <CacheFormat F>
__global__ __launch_bounds__(kCacheThreads) void cache_write_kernel(CacheCopyParams p, Shares sh) {
    const Cache& c = p.c;
    const int64_t t0 = (int64_t)blockIdx.x * sh.tokens;
    const int n = (int)min((int64_t)sh.tokens, p.T - t0) * sh.each;  // a multiple of 8: a block's lanes stay together
    for (int i = blockIdx.y * kAtOnce * kCacheThreads + threadIdx.x; i < n; i += gridDim.y * kAtOnce * kCacheThreads) {
        float v[kAtOnce][8];
        int64_t slot[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (i + j * kCacheThreads >= n) break;
            const Eight e(c, sh, i + j * kCacheThreads);
            const int64_t token = t0 + e.token;
            slot[j] = p.slots[token];
            load8(e.value ? p.v : p.k, p.is16,
                  e.value ? token * p.v_token + e.head * p.v_head + e.column : token * p.k_token + e.head * p.k_head + e.column, v[j]);
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (i + j * kCacheThreads >= n) break;
            const Eight e(c, sh, i + j * kCacheThreads);
            const int64_t row = cache_row(c, slot[j], e.head);
            uint8_t* const codes = e.value ? c.v : c.k;
            if (F == CacheFormat::Bf16) {
                if (row < 0) continue;
                u32x4v w;
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = bf16_pair(v[j][2 * k], v[j][2 * k + 1]);
                *reinterpret_cast<u32x4v*>(codes + 2 * (row * c.d + e.column)) = w;
                continue;
            }
            float amax = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) amax = fmaxf(amax, fabsf(v[j][k]));
            amax = quad_max(amax);
            const uint32_t s = mx_byte<F == CacheFormat::Mxfp4 ? 2 : 8>(amax);
            if (row < 0) continue;
            if (F == CacheFormat::Mxfp4) *reinterpret_cast<uint32_t*>(codes + (row * c.d + e.column) / 2) = e2m1_codes(v[j], mx_scale(s));
            else *reinterpret_cast<u32x2v*>(codes + row * c.d + e.column) = e4m3_codes(v[j], mx_scale(s));
            if (e.column % 32 == 0) (e.value ? c.v_scales : c.k_scales)[row * (c.d / 32) + e.column / 32] = (uint8_t)s;
        }
    }
}

template <CacheFormat F>
__global__ __launch_bounds__(kCacheThreads) void cache_read_kernel(CacheCopyParams p, Shares sh) {
    constexpr int kWords = F == CacheFormat::Bf16 ? 4 : F == CacheFormat::Mxfp8 ? 2 : 1;
    const Cache& c = p.c;
    const int64_t t0 = (int64_t)blockIdx.x * sh.tokens;
    const int n = (int)min((int64_t)sh.tokens, p.T - t0) * sh.each;
    for (int i = blockIdx.y * kAtOnce * kCacheThreads + threadIdx.x; i < n; i += gridDim.y * kAtOnce * kCacheThreads) {
        int64_t slot[kAtOnce];
        uint32_t q[kAtOnce][kWords], s[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (i + j * kCacheThreads >= n) break;
            slot[j] = p.slots[t0 + Eight(c, sh, i + j * kCacheThreads).token];
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (i + j * kCacheThreads >= n) break;
            const Eight e(c, sh, i + j * kCacheThreads);
            const int64_t row = cache_row(c, slot[j], e.head), at = row < 0 ? 0 : row;
            const uint8_t* const codes = (e.value ? c.v : c.k) + (at * c.d + e.column) * kWords / 2;
            if constexpr (F == CacheFormat::Mxfp4) {
                q[j][0] = *reinterpret_cast<const uint32_t*>(codes);
            } else if constexpr (F == CacheFormat::Mxfp8) {
                const u32x2v w = *reinterpret_cast<const u32x2v*>(codes);
                q[j][0] = w[0];
                q[j][1] = w[1];
            } else {
                const u32x4v w = *reinterpret_cast<const u32x4v*>(codes);
#pragma unroll
                for (int k = 0; k < 4; ++k) q[j][k] = w[k];
            }
            s[j] = F == CacheFormat::Bf16 ? 0u : (e.value ? c.v_scales : c.k_scales)[at * (c.d / 32) + e.column / 32];
            slot[j] = row;
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (i + j * kCacheThreads >= n) break;
            const Eight e(c, sh, i + j * kCacheThreads);
            u32x4v w;  // as bf16, which holds every value of these formats
            const float sc = mx_scale(s[j]);
            if constexpr (F == CacheFormat::Bf16) w = u32x4v{q[j][0], q[j][1], q[j][2], q[j][3]};
            else if constexpr (F == CacheFormat::Mxfp4) w = u32x4v{e2m1_pair<0>(q[j][0], sc), e2m1_pair<1>(q[j][0], sc), e2m1_pair<2>(q[j][0], sc), e2m1_pair<3>(q[j][0], sc)};
            else w = u32x4v{e4m3_pair<0>(q[j][0], sc), e4m3_pair<1>(q[j][0], sc), e4m3_pair<0>(q[j][1], sc), e4m3_pair<1>(q[j][1], sc)};
            if (slot[j] < 0) w = u32x4v{0u, 0u, 0u, 0u};
            void* const base = e.value ? p.v : p.k;
            const int64_t at = ((t0 + e.token) * c.heads + e.head) * c.d + e.column;
            if (p.is16) {
                *reinterpret_cast<u32x4v*>(static_cast<uint16_t*>(base) + at) = w;
            } else {
                typedef float f32x4 __attribute__((ext_vector_type(4)));
                f32x4* const out = reinterpret_cast<f32x4*>(static_cast<float*>(base) + at);
                out[0] = f32x4{bf16_low(w[0]), bf16_high(w[0]), bf16_low(w[1]), bf16_high(w[1])};
                out[1] = f32x4{bf16_low(w[2]), bf16_high(w[2]), bf16_low(w[3]), bf16_high(w[3])};
            }
        }
    }
}

// Tokens of a workgroup, and workgroups that share them.  A small call has fewer tokens a workgroup.
dim3 cache_grid(const CacheCopyParams& p, Shares* sh) {
    const int64_t columns = p.c.d / 8, half = p.c.heads * columns, each = 2 * half;
    const int64_t turn = kAtOnce * kCacheThreads;
    sh->each = (int)each;
    sh->half = (int)half;
    sh->by_each = (uint32_t)((0x100000000ull + each - 1) / each);
    sh->by_columns = (uint32_t)((0x100000000ull + columns - 1) / columns);
    int64_t tokens = std::max<int64_t>(1, turn / each);
    while (tokens > 1 && (p.T + tokens - 1) / tokens < 512) tokens /= 2;
    sh->tokens = (int)tokens;
    const int64_t share = std::min<int64_t>(65535, (tokens * each + turn - 1) / turn);
    return dim3((unsigned)((p.T + tokens - 1) / tokens), (unsigned)share);
}

}  // namespace

hipError_t launch_cache_write(const CacheCopyParams& p, hipStream_t st) {
    Shares sh;
    const dim3 grid = cache_grid(p, &sh);
    switch (p.c.format) {
        case CacheFormat::Bf16: cache_write_kernel<CacheFormat::Bf16><<<grid, kCacheThreads, 0, st>>>(p, sh); break;
        case CacheFormat::Mxfp8: cache_write_kernel<CacheFormat::Mxfp8><<<grid, kCacheThreads, 0, st>>>(p, sh); break;
        case CacheFormat::Mxfp4: cache_write_kernel<CacheFormat::Mxfp4><<<grid, kCacheThreads, 0, st>>>(p, sh); break;
    }
    return hipGetLastError();
}

hipError_t launch_cache_read(const CacheCopyParams& p, hipStream_t st) {
    Shares sh;
    const dim3 grid = cache_grid(p, &sh);
    switch (p.c.format) {
        case CacheFormat::Bf16: cache_read_kernel<CacheFormat::Bf16><<<grid, kCacheThreads, 0, st>>>(p, sh); break;
        case CacheFormat::Mxfp8: cache_read_kernel<CacheFormat::Mxfp8><<<grid, kCacheThreads, 0, st>>>(p, sh); break;
        case CacheFormat::Mxfp4: cache_read_kernel<CacheFormat::Mxfp4><<<grid, kCacheThreads, 0, st>>>(p, sh); break;
    }
    return hipGetLastError();
}

}  // namespace kq
