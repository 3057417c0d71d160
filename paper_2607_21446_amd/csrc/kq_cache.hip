// A paged cache of keys and values, quantized as it is written, and read back.
// A block of 32 values shares a scale 2^s, s = floor(log2 max|x|) - m, m = 2
// for E2M1 and 8 for E4M3 elements; values round to the nearest element, ties
// to even, and saturate.  A bf16 cache rounds values once.
//
// Four lanes of eight values hold a block; its maximum is two exchanges
// between them.  Bound by HBM, a value is read and written once: 32768 tokens
// of 8 x 128 are read from MXFP8 in 34.4 us (203 MB, 5.9 TB/s), 8191 written in
// 12.9 (51 MB).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "kq_mx.h"
#include "kq_serve.h"

namespace kq {

namespace {

constexpr int kCacheThreads = 256;

// Eight values of a row, at any alignment of their elements.
template <bool B16>
__device__ __forceinline__ void load8(const void* p, uint64_t at, float (&v)[8]) {
    if constexpr (B16) {
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

// How a call's eights of values are shared out: a workgroup takes keys or values (in turn: their addresses and strides are
// uniform) of some tokens, in order of token, head and column; `in` counts its eights.  Divisions are multiplications by
// 2^32 / n, rounded up: exact for `in` below 2048 by `each` up to 1024 (where a workgroup has several tokens), and below 2^21
// by up to 32 columns of eight.  The other multiplications are of 24 bits where their factors are (whole ones of 32 bits take
// four times as long).  Index arithmetic in 64 bits with keys and values in one workgroup kept the vector units busy for 0.8
// of a write and 0.9 of a read: 17.0 and 38.4 us for the calls above.  In order of head first, whose codes and scales are
// whole lines of the cache, they took 18.4 and 48.  With all keys before the values, both calls on data that no cache holds
// take 55.5 us instead of 52.8.
struct Shares {
    int tokens;     // of a workgroup
    uint32_t each;  // eights of a token
    uint32_t by_each, by_columns;
};
struct Eight {
    uint32_t token, head, column;
    __device__ __forceinline__ Eight(const Cache& c, const Shares& sh, uint32_t in) {
        token = sh.tokens > 1 ? __umulhi(in, sh.by_each) : 0u;
        const uint32_t s = in - __umul24(token, sh.each);
        head = __umulhi(s, sh.by_columns);
        column = 8 * (s - __umul24(head, (uint32_t)c.d / 8));
    }
};

// Where a slot's row of a head is: its first block of 32 among the cache's.
struct CacheRow {
    bool in;  // the cache holds the slot
    uint64_t block;
    __device__ __forceinline__ CacheRow(const Cache& c, int64_t slot, uint32_t head) {
        in = (uint64_t)slot < (uint64_t)(c.pages * c.page_size);
        const uint32_t page = in ? (uint32_t)(slot >> c.page_shift) : 0u, token = (uint32_t)slot & (uint32_t)(c.page_size - 1);
        const uint64_t row = (((uint64_t)page * (uint32_t)c.heads + head) << c.page_shift) + token;
        block = row * (uint32_t)(c.d / 32);
    }
};

// A thread's eights of a turn: their loads are in flight together.
constexpr int kAtOnce = 4;

template <CacheFormat F>
constexpr int kEightBytes = F == CacheFormat::Bf16 ? 16 : F == CacheFormat::Mxfp8 ? 8 : 4;

template <CacheFormat F, bool B16>
__global__ __launch_bounds__(kCacheThreads) void cache_write_kernel(CacheCopyParams p, Shares sh) {
    const Cache& c = p.c;
    const int64_t t0 = (int64_t)(blockIdx.x >> 1) * sh.tokens;
    const uint32_t n = (uint32_t)min((int64_t)sh.tokens, p.T - t0) * sh.each;  // a multiple of 4: a block's lanes stay together
    const bool value = blockIdx.x & 1;
    const int64_t by_token = value ? p.v_token : p.k_token, by_head = value ? p.v_head : p.k_head;
    const uint8_t* const from = static_cast<const uint8_t*>(value ? p.v : p.k) + t0 * by_token * (B16 ? 2 : 4);
    uint8_t *const to = value ? c.v : c.k, *const scales = value ? c.v_scales : c.k_scales;
    for (uint32_t i = blockIdx.y * kAtOnce * kCacheThreads + threadIdx.x; i < n; i += gridDim.y * kAtOnce * kCacheThreads) {
        float v[kAtOnce][8];
        int64_t slot[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (i + j * kCacheThreads >= n) break;
            const Eight e(c, sh, i + j * kCacheThreads);
            slot[j] = p.slots[t0 + e.token];
            load8<B16>(from, e.token * (uint64_t)by_token + e.head * (uint64_t)by_head + e.column, v[j]);
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (i + j * kCacheThreads >= n) break;
            const Eight e(c, sh, i + j * kCacheThreads);
            const CacheRow row(c, slot[j], e.head);
            uint8_t* const codes = to + (row.block * 4 + e.column / 8) * kEightBytes<F>;
            if constexpr (F == CacheFormat::Bf16) {
                if (!row.in) continue;
                u32x4v w;
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = bf16_pair(v[j][2 * k], v[j][2 * k + 1]);
                *reinterpret_cast<u32x4v*>(codes) = w;
            } else {
                float amax = 0.f;
#pragma unroll
                for (int k = 0; k < 8; ++k) amax = fmaxf(amax, fabsf(v[j][k]));
                amax = quad_max(amax);
                const uint32_t s = mx_byte<F == CacheFormat::Mxfp4 ? 2 : 8>(amax);
                if (!row.in) continue;
                if constexpr (F == CacheFormat::Mxfp4) *reinterpret_cast<uint32_t*>(codes) = e2m1_codes(v[j], mx_scale(s));
                else *reinterpret_cast<u32x2v*>(codes) = e4m3_codes(v[j], mx_scale(s));
                if (e.column % 32 == 0) scales[row.block + e.column / 32] = (uint8_t)s;
            }
        }
    }
}

template <CacheFormat F, bool B16>
__global__ __launch_bounds__(kCacheThreads) void cache_read_kernel(CacheCopyParams p, Shares sh) {
    constexpr int kWords = kEightBytes<F> / 4;
    const Cache& c = p.c;
    const int64_t t0 = (int64_t)(blockIdx.x >> 1) * sh.tokens;
    const uint32_t n = (uint32_t)min((int64_t)sh.tokens, p.T - t0) * sh.each;
    const bool value = blockIdx.x & 1;
    const uint8_t *const from = value ? c.v : c.k, *const scales = value ? c.v_scales : c.k_scales;
    uint8_t* const to = static_cast<uint8_t*>(value ? p.v : p.k) + t0 * sh.each * (B16 ? 16 : 32);
    for (uint32_t i = blockIdx.y * kAtOnce * kCacheThreads + threadIdx.x; i < n; i += gridDim.y * kAtOnce * kCacheThreads) {
        int64_t slot[kAtOnce];
        bool in[kAtOnce];
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
            const CacheRow row(c, slot[j], e.head);
            in[j] = row.in;
            const uint8_t* const codes = from + (row.block * 4 + e.column / 8) * kEightBytes<F>;
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
            if constexpr (F != CacheFormat::Bf16) s[j] = scales[row.block + e.column / 32];
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (i + j * kCacheThreads >= n) break;
            u32x4v w;  // as bf16, which holds every value of these formats
            if constexpr (F == CacheFormat::Bf16) {
                w = u32x4v{q[j][0], q[j][1], q[j][2], q[j][3]};
            } else {
                const float sc = mx_scale(s[j]);
                if constexpr (F == CacheFormat::Mxfp4) w = u32x4v{e2m1_pair<0>(q[j][0], sc), e2m1_pair<1>(q[j][0], sc), e2m1_pair<2>(q[j][0], sc), e2m1_pair<3>(q[j][0], sc)};
                else w = u32x4v{e4m3_pair<0>(q[j][0], sc), e4m3_pair<1>(q[j][0], sc), e4m3_pair<0>(q[j][1], sc), e4m3_pair<1>(q[j][1], sc)};
            }
            if (!in[j]) w = u32x4v{0u, 0u, 0u, 0u};
            uint8_t* const out = to + (i + j * kCacheThreads) * (B16 ? 16u : 32u);
            if constexpr (B16) {
                *reinterpret_cast<u32x4v*>(out) = w;
            } else {
                typedef float f32x4 __attribute__((ext_vector_type(4)));
                reinterpret_cast<f32x4*>(out)[0] = f32x4{bf16_low(w[0]), bf16_high(w[0]), bf16_low(w[1]), bf16_high(w[1])};
                reinterpret_cast<f32x4*>(out)[1] = f32x4{bf16_low(w[2]), bf16_high(w[2]), bf16_low(w[3]), bf16_high(w[3])};
            }
        }
    }
}

// Tokens of a workgroup.  A small call has fewer.
Shares cache_shares(const CacheCopyParams& p) {
    const int64_t columns = p.c.d / 8, each = p.c.heads * columns;
    Shares sh;
    sh.each = (uint32_t)each;
    sh.by_each = (uint32_t)((0x100000000ull + each - 1) / each);
    sh.by_columns = (uint32_t)((0x100000000ull + columns - 1) / columns);
    int64_t tokens = std::max<int64_t>(1, kAtOnce * kCacheThreads / each);
    while (tokens > 1 && (p.T + tokens - 1) / tokens < 256) tokens /= 2;
    sh.tokens = (int)tokens;
    return sh;
}

// launch(params, shares, grid): workgroups for keys and values of as many tokens as a launch holds.
template <class F>
void cache_launches(const CacheCopyParams& p, F launch) {
    const Shares sh = cache_shares(p);
    const int64_t turn = kAtOnce * kCacheThreads, share = std::min<int64_t>(65535, ((int64_t)sh.tokens * sh.each + turn - 1) / turn);
    const int64_t size = p.is16 ? 2 : 4;
    in_launches(p.T, sh.tokens, 2 * kCacheThreads, [&](int64_t from, int64_t n) {
        CacheCopyParams l = p;
        l.T = n;
        l.slots = p.slots + from;
        l.k = static_cast<uint8_t*>(p.k) + from * p.k_token * size;
        l.v = static_cast<uint8_t*>(p.v) + from * p.v_token * size;
        launch(l, sh, dim3((unsigned)(2 * ((n + sh.tokens - 1) / sh.tokens)), (unsigned)share));
    });
}

template <CacheFormat F>
void launch_write_of(const CacheCopyParams& p, hipStream_t st) {
    cache_launches(p, [&](const CacheCopyParams& l, const Shares& sh, dim3 grid) {
        if (l.is16) cache_write_kernel<F, true><<<grid, kCacheThreads, 0, st>>>(l, sh);
        else cache_write_kernel<F, false><<<grid, kCacheThreads, 0, st>>>(l, sh);
    });
}
template <CacheFormat F>
void launch_read_of(const CacheCopyParams& p, hipStream_t st) {
    cache_launches(p, [&](const CacheCopyParams& l, const Shares& sh, dim3 grid) {
        if (l.is16) cache_read_kernel<F, true><<<grid, kCacheThreads, 0, st>>>(l, sh);
        else cache_read_kernel<F, false><<<grid, kCacheThreads, 0, st>>>(l, sh);
    });
}

}  // namespace

hipError_t launch_cache_write(const CacheCopyParams& p, hipStream_t st) {
    switch (p.c.format) {
        case CacheFormat::Bf16: launch_write_of<CacheFormat::Bf16>(p, st); break;
        case CacheFormat::Mxfp8: launch_write_of<CacheFormat::Mxfp8>(p, st); break;
        case CacheFormat::Mxfp4: launch_write_of<CacheFormat::Mxfp4>(p, st); break;
    }
    return hipGetLastError();
}

hipError_t launch_cache_read(const CacheCopyParams& p, hipStream_t st) {
    switch (p.c.format) {
        case CacheFormat::Bf16: launch_read_of<CacheFormat::Bf16>(p, st); break;
        case CacheFormat::Mxfp8: launch_read_of<CacheFormat::Mxfp8>(p, st); break;
        case CacheFormat::Mxfp4: launch_read_of<CacheFormat::Mxfp4>(p, st); break;
    }
    return hipGetLastError();
}

}  // namespace kq
