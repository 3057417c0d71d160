// Internal interface of the operators of a generation step to the C-ABI layer: rotary positions (kq_rope.hip), the
// paged cache (kq_cache.hip), attention over it (kq_attn.hip) and W4A16 linear layers (kq_matvec.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kq_linear.h"

namespace kq {

// Sizes already validated by the caller, in every struct here.

// A grid's threads along a dimension are counted in 32 bits; past them HIP starts fewer workgroups, without an error.  So n
// items, `each` of them to `threads` threads, go in as many launches as it takes: launch(first item, items).
template <class F>
void in_launches(int64_t n, int64_t each, int64_t threads, F launch) {
    const int64_t most = (int64_t(UINT32_MAX) / threads) * each;
    for (int64_t at = 0; at < n; at += most) launch(at, n - at < most ? n - at : most);
}

constexpr int kRopeMaxAxes = 4;
constexpr int64_t kRopeMaxColumns = 1024;

enum class Position { Int32 = 0, Int64 = 1, Fp32 = 2 };

struct RopeParams {
    const void* x;  // [T, H, D] at its strides, columns contiguous
    void* y;
    int64_t T;
    int H, D;
    int64_t x_token, x_head, y_token, y_head;  // strides in elements
    const void* positions;                     // [T, axes], row stride pos_stride
    int64_t pos_stride;
    Position pos_type;
    int axes;
    int end[kRopeMaxAxes];  // pairs up to and with an axis' section; the last one: of the rotated part
    double log2_theta;
    const double* freqs;  // [pairs] or null
    int halves;           // pairs (p, p + pairs), not (2p, 2p + 1)
    int is16;             // 1: bf16, 0: fp32
    int backward;
    int64_t heads;      // filled in by the launcher: heads of a workgroup,
    int tokens;         // and its tokens
};
hipError_t launch_rope(RopeParams p, hipStream_t st);

enum class CacheFormat { Bf16 = 0, Mxfp8 = 1, Mxfp4 = 2 };
constexpr int64_t kCacheMaxColumns = 256;

// Keys and values of pages of page_size tokens: [pages, heads, page_size, d] elements, and E8M0 scales of blocks of 32.
struct Cache {
    uint8_t* k;
    uint8_t* v;
    uint8_t* k_scales;
    uint8_t* v_scales;
    CacheFormat format;
    int64_t pages;
    int heads, page_size, d;  // page_size a power of two, d a multiple of 32
    int page_shift;           // log2 page_size
};

struct CacheCopyParams {
    Cache c;
    const int64_t* slots;  // [T]: page * page_size + token in the page; others: the token is left out
    int64_t T;
    void* k;  // write: [T, heads, d] at its strides; read: contiguous
    void* v;
    int64_t k_token, k_head, v_token, v_head;
    int is16;  // k and v: 1 bf16, 0 fp32
};
hipError_t launch_cache_write(const CacheCopyParams& p, hipStream_t st);
hipError_t launch_cache_read(const CacheCopyParams& p, hipStream_t st);

struct AttnParams {
    Cache c;
    const void* q;  // [B, heads * group, d] at its strides
    void* out;
    int64_t q_seq, q_head, out_seq, out_head;
    int64_t B;
    int group;                // query heads of a head of the cache
    const int32_t* table;     // [B, max_pages], row stride table_stride
    int64_t table_stride;
    int64_t max_tokens;       // max_pages * page_size, at most 2^31 - 1
    const int32_t* lengths;   // [B]
    int64_t window;           // the last so many tokens count; 0: all
    float scale;
    int is16;                 // q and out: 1 bf16, 0 fp32
    float* lse;               // [B, heads * group] or null
    uint8_t* workspace;       // attn_workspace bytes
    // filled in by the launcher: runs that a head's tiles are cut into, and the places of their pieces' results in the
    // workspace
    int runs;
    double inverse;  // 1 / runs
    int32_t* plan;   // [B, 2]: a sequence's first run, and how many it has pieces in
    float* stats;    // [run_slots, heads * group, 2]: maximum and sum
    float* partial;  // [run_slots, heads * group, d]
};
int64_t attn_workspace(int64_t B, int64_t heads, int64_t group, int64_t d);
hipError_t launch_attn(AttnParams p, hipStream_t st);

struct MatvecParams {
    const void* x;  // [M, K], row stride ldx
    int64_t ldx;
    int x16;  // 1: bf16, 0: fp32
    LinearParams l;  // weight, sizes, epilogue; no A
    float* partial;  // matvec_workspace bytes, or null: a form without
    int64_t columns;  // of its rows, filled in by the launcher
};
int64_t matvec_workspace(int64_t M, int64_t N, int64_t K, bool x16);  // 0: none is used
hipError_t launch_matvec(MatvecParams p, hipStream_t st);

}  // namespace kq
