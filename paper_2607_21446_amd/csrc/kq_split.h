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

__host__ __device__ __forceinline__ int64_t part_tiles(int64_t total, int parts) {
    const int64_t c = (total + parts - 1) / parts;
    return c > kLeastTiles ? c : kLeastTiles;
}
__host__ __device__ __forceinline__ int part_count(int tiles, int64_t c) {
    return tiles <= c ? 1 : (int)((tiles + c - 1) / c);
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

// Part `x` of the call, found by each of a workgroup's waves: two passes over the lengths, 64 at a time.
__device__ __forceinline__ Part find_part(const int32_t* lengths, int B, int64_t max_tokens, int64_t window, int parts, int x) {
    const int lane = threadIdx.x & 63;
    auto span = [&](int b) { return Span(b < B ? lengths[b] : 0, max_tokens, window); };
    int64_t total = 0;
    for (int b = lane; b < B; b += 64) total += span(b).tiles();
    for (int k = 1; k < 64; k <<= 1) total += __shfl_xor((long long)total, k);
    const int64_t c = part_tiles(total, parts);
    Part p{-1, 0, 0, 0, 0, 0, 0, 0};
    int before = 0, slot = 0;
    for (int b0 = 0; b0 < B; b0 += 64) {
        const Span s = span(b0 + lane);
        const int n = b0 + lane < B ? part_count(s.tiles(), c) : 0;
        int upto = n, several = n > 1 ? n : 0;
        for (int k = 1; k < 64; k <<= 1) {
            const int u = __shfl_up(upto, k), v = __shfl_up(several, k);
            upto += lane >= k ? u : 0;
            several += lane >= k ? v : 0;
        }
        const uint64_t here = __ballot(before + upto > x);
        if (here) {
            const int at = __ffsll((unsigned long long)here) - 1;
            p.b = b0 + at;
            p.count = __builtin_amdgcn_readlane(n, at);
            p.index = x - (before + __builtin_amdgcn_readlane(upto, at) - p.count);
            p.slot = slot + __builtin_amdgcn_readlane(several, at) - (p.count > 1 ? p.count : 0);
            p.first = __builtin_amdgcn_readlane(s.first, at);
            p.end = __builtin_amdgcn_readlane(s.end, at);
            const int64_t done = p.index * c, all = Span(p.end, max_tokens, window).tiles();
            p.tile = p.first / kTileTokens + (int)done;
            p.tiles = (int)(all - done < c ? all - done : c);
            return p;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
        slot += __builtin_amdgcn_readlane(several, 63);
    }
    return p;
}

}  // namespace

}  // namespace kq
