// How attention over a cache (kq_attn.hip) cuts ragged sequences into parts of
// equal length, from lengths that are on the device only.
//
// Tokens count in tiles of 32.  All sequences' tiles T together are cut into
// parts of c = max(least, ceil(T / parts)) tiles, a sequence's last part
// shorter; an empty sequence has one part.  So there are at most
// parts + B parts, and at most 2 parts of them belong to sequences of several
// (a sequence of t > c tiles has ceil(t / c) < 2 t / c): the grid and the
// places for their results are sized by that, whatever the lengths are.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kq {

namespace {

constexpr int kTileTokens = 32;
constexpr int kLeastTiles = 4;  // of a part: a tile for each of a workgroup's waves

// The tokens of a sequence that count: first .. end - 1; tiles start at multiples of 32.
struct Span {
    int first, end;
    __host__ __device__ __forceinline__ Span(int length, int64_t max_tokens, int64_t window) {
        const int64_t n = length < 0 ? 0 : length < max_tokens ? length : max_tokens;
        end = (int)n;
        first = window > 0 && window < n ? (int)(n - window) : 0;
    }
    __host__ __device__ __forceinline__ int first_tile() const { return first / kTileTokens; }
    __host__ __device__ __forceinline__ int tiles() const {
        return end > first ? (end - 1) / kTileTokens + 1 - first_tile() : 0;
    }
};

// Tiles of a part, at least total / parts; `inverse` is 1 / parts.  No sequence has 2^26 tiles.
__host__ __device__ __forceinline__ int part_tiles(uint64_t total, double inverse) {
    const double c = (double)total * inverse * (1.0 + 0x1p-50);  // (total < 2^46: the product's errors are below that factor's)
    const int n = c < 0x1p26 ? (int)c + ((double)(int)c < c) : 1 << 26;
    return n > kLeastTiles ? n : kLeastTiles;
}
__host__ __device__ __forceinline__ int part_count(int tiles, int c) {
    return tiles <= c ? 1 : (int)((uint32_t)(tiles + c - 1) / (uint32_t)c);
}
// Places for the results of parts.
__host__ __device__ __forceinline__ int64_t part_slots(int64_t parts, int64_t B) {
    return 2 * parts < parts + B ? 2 * parts : parts + B;
}

// Which of a sequence's pages holds token `token`; tokens from `end` (at least 1) on are looked up in the last one.
__host__ __device__ __forceinline__ int page_index(int token, int end, int page_shift) {
    const int at = token >> page_shift, last = (end - 1) >> page_shift;
    return at < last ? at : last;
}
// The page of a table's entry: the nearest one of the cache.
__host__ __device__ __forceinline__ int64_t page_of(int32_t entry, int64_t pages) {
    return entry < 0 ? 0 : entry < pages ? entry : pages - 1;
}

// A workgroup's part; b < 0: none.
struct Part {
    int b, index, count;  // sequence, number in it and how many it has
    int slot;             // place of the sequence's first result, if it has several parts
    int first, end;       // its tokens that count
    int tile, tiles;      // its tiles from `tile` on, tile 0 starting at token 0
};

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_sum(uint32_t v) {
    return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
// The sum of the lanes up to and with each.
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
    v = dpp_sum<0x111, 0xf>(v);  // row_shr 1, 2, 4, 8: sums up to the lane in its row of 16
    v = dpp_sum<0x112, 0xf>(v);
    v = dpp_sum<0x114, 0xf>(v);
    v = dpp_sum<0x118, 0xf>(v);
    v = dpp_sum<0x142, 0xa>(v);  // rows 0 and 2 onto 1 and 3, then 1 onto 2 and 3
    return dpp_sum<0x143, 0xc>(v);
}
__device__ __forceinline__ int lane_value(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

// Part `x` of the call, found by each of a workgroup's waves: two passes over the lengths, 64 at a time (their tiles
// together are below 2^32); one where there are no more than 64.
__device__ __forceinline__ Part find_part(const int32_t* lengths, int B, int64_t max_tokens, int64_t window, double inverse, int x) {
    const int lane = threadIdx.x & 63;
    auto span = [&](int b) __attribute__((always_inline)) { return Span(b < B ? lengths[b] : 0, max_tokens, window); };
    Span s = span(lane);
    uint64_t total = 0;
    for (int b0 = 0;;) {
        total += (uint32_t)lane_value((int)wave_scan((uint32_t)s.tiles()), 63);
        b0 += 64;
        if (b0 >= B) break;
        s = span(b0 + lane);
    }
    const int c = part_tiles(total, inverse);
    Part p{-1, 0, 0, 0, 0, 0, 0, 0};
    int before = 0, slot = 0;
    if (B > 64) s = span(lane);
    for (int b0 = 0; b0 < B;) {
        const int tiles = s.tiles(), n = b0 + lane < B ? part_count(tiles, c) : 0;
        const int upto = (int)wave_scan((uint32_t)n), several = (int)wave_scan(n > 1 ? (uint32_t)n : 0u);
        const uint64_t here = __ballot(before + upto > x);
        if (here) {
            const int at = __ffsll((unsigned long long)here) - 1;
            p.b = b0 + at;
            p.count = lane_value(n, at);
            p.index = x - (before + lane_value(upto, at) - p.count);
            p.slot = slot + lane_value(several, at) - (p.count > 1 ? p.count : 0);
            p.first = lane_value(s.first, at);
            p.end = lane_value(s.end, at);
            const int done = p.index * c, left = lane_value(tiles, at) - done;
            p.tile = p.first / kTileTokens + done;
            p.tiles = left < c ? left : c;
            return p;
        }
        before += lane_value(upto, 63);
        slot += lane_value(several, 63);
        b0 += 64;
        s = span(b0 + lane);
    }
    return p;
}

}  // namespace

}  // namespace kq
