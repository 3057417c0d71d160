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

// Where an eight of a call's values is: its token, head, column and half of the cache.
struct Eight {
    int64_t token;
    int head, column;
    bool value;
    // Eights are in order of token, half, head and column; `in` counts those of `tokens` tokens from t0 on.
    __device__ __forceinline__ Eight(const Cache& c, int64_t t0, int in) {
        const int columns = c.d / 8, half = c.heads * columns;
        const int t = in / (2 * half), r = in - t * 2 * half;
        token = t0 + t;
        value = r >= half;
        const int s = value ? r - half : r;
        head = s / columns;
        column = 8 * (s - head * columns);
    }
};

// The cache's row of a slot, -1 for one outside the cache.
__device__ __forceinline__ int64_t cache_row(const Cache& c, int64_t slot, int head) {
    if (slot < 0 || slot >= c.pages * c.page_size) return -1;
    return (((slot >> c.page_shift) * c.heads + head) << c.page_shift) + (slot & (c.page_size - 1));
}

template <CacheFormat F>
__global__ __launch_bounds__(kCacheThreads) void cache_write_kernel(CacheCopyParams p, int tokens) {
    const Cache& c = p.c;
    const int64_t t0 = (int64_t)blockIdx.x * tokens;
    const int n = (int)min((int64_t)tokens, p.T - t0) * 2 * c.heads * (c.d / 8);  // a multiple of 8: a block's lanes stay together
    for (int i = blockIdx.y * kCacheThreads + threadIdx.x; i < n; i += gridDim.y * kCacheThreads) {
        const Eight e(c, t0, i);
        float v[8];
        load8(e.value ? p.v : p.k, p.is16,
              e.value ? e.token * p.v_token + e.head * p.v_head + e.column : e.token * p.k_token + e.head * p.k_head + e.column, v);
        const int64_t row = cache_row(c, p.slots[e.token], e.head);
        if (F == CacheFormat::Bf16) {
            if (row < 0) continue;
            u32x4v w;
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = bf16_pair(v[2 * k], v[2 * k + 1]);
            *reinterpret_cast<u32x4v*>((e.value ? c.v : c.k) + 2 * (row * c.d + e.column)) = w;
            continue;
        }
        float amax = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) amax = fmaxf(amax, fabsf(v[k]));
        amax = quad_max(amax);
        const uint32_t s = mx_byte<F == CacheFormat::Mxfp4 ? 2 : 8>(amax);
        if (row < 0) continue;
        uint8_t* const codes = e.value ? c.v : c.k;
        if (F == CacheFormat::Mxfp4) *reinterpret_cast<uint32_t*>(codes + (row * c.d + e.column) / 2) = e2m1_codes(v, mx_scale(s));
        else *reinterpret_cast<u32x2v*>(codes + row * c.d + e.column) = e4m3_codes(v, mx_scale(s));
        if (e.column % 32 == 0) (e.value ? c.v_scales : c.k_scales)[row * (c.d / 32) + e.column / 32] = (uint8_t)s;
    }
}

template <CacheFormat F>
__global__ __launch_bounds__(kCacheThreads) void cache_read_kernel(CacheCopyParams p, int tokens) {
    const Cache& c = p.c;
    const int64_t t0 = (int64_t)blockIdx.x * tokens;
    const int n = (int)min((int64_t)tokens, p.T - t0) * 2 * c.heads * (c.d / 8);
    for (int i = blockIdx.y * kCacheThreads + threadIdx.x; i < n; i += gridDim.y * kCacheThreads) {
        const Eight e(c, t0, i);
        const int64_t row = cache_row(c, p.slots[e.token], e.head);
        u32x4v w = {0u, 0u, 0u, 0u};  // as bf16, which holds every value of these formats
        if (row >= 0) {
            const uint8_t* const codes = e.value ? c.v : c.k;
            if (F == CacheFormat::Bf16) {
                w = *reinterpret_cast<const u32x4v*>(codes + 2 * (row * c.d + e.column));
            } else {
                const float s = mx_scale((e.value ? c.v_scales : c.k_scales)[row * (c.d / 32) + e.column / 32]);
                if (F == CacheFormat::Mxfp4) {
                    const uint32_t q = *reinterpret_cast<const uint32_t*>(codes + (row * c.d + e.column) / 2);
                    w = u32x4v{e2m1_pair<0>(q, s), e2m1_pair<1>(q, s), e2m1_pair<2>(q, s), e2m1_pair<3>(q, s)};
                } else {
                    const u32x2v q = *reinterpret_cast<const u32x2v*>(codes + row * c.d + e.column);
                    w = u32x4v{e4m3_pair<0>(q[0], s), e4m3_pair<1>(q[0], s), e4m3_pair<0>(q[1], s), e4m3_pair<1>(q[1], s)};
                }
            }
        }
        void* const base = e.value ? p.v : p.k;
        const int64_t at = (e.token * c.heads + e.head) * c.d + e.column;
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

// Tokens of a workgroup, and workgroups that share them.
dim3 cache_grid(const CacheCopyParams& p, int* tokens) {
    const int64_t each = 2 * p.c.heads * (p.c.d / 8);
    *tokens = (int)std::max<int64_t>(1, 4 * kCacheThreads / each);
    const int64_t share = std::min<int64_t>(65535, std::max<int64_t>(1, each / (4 * kCacheThreads)));
    return dim3((unsigned)((p.T + *tokens - 1) / *tokens), (unsigned)share);
}

}  // namespace

hipError_t launch_cache_write(const CacheCopyParams& p, hipStream_t st) {
    int tokens;
    const dim3 grid = cache_grid(p, &tokens);
    switch (p.c.format) {
        case CacheFormat::Bf16: cache_write_kernel<CacheFormat::Bf16><<<grid, kCacheThreads, 0, st>>>(p, tokens); break;
        case CacheFormat::Mxfp8: cache_write_kernel<CacheFormat::Mxfp8><<<grid, kCacheThreads, 0, st>>>(p, tokens); break;
        case CacheFormat::Mxfp4: cache_write_kernel<CacheFormat::Mxfp4><<<grid, kCacheThreads, 0, st>>>(p, tokens); break;
    }
    return hipGetLastError();
}

hipError_t launch_cache_read(const CacheCopyParams& p, hipStream_t st) {
    int tokens;
    const dim3 grid = cache_grid(p, &tokens);
    switch (p.c.format) {
        case CacheFormat::Bf16: cache_read_kernel<CacheFormat::Bf16><<<grid, kCacheThreads, 0, st>>>(p, tokens); break;
        case CacheFormat::Mxfp8: cache_read_kernel<CacheFormat::Mxfp8><<<grid, kCacheThreads, 0, st>>>(p, tokens); break;
        case CacheFormat::Mxfp4: cache_read_kernel<CacheFormat::Mxfp4><<<grid, kCacheThreads, 0, st>>>(p, tokens); break;
    }
    return hipGetLastError();
}

}  // namespace kq
