// How attention over a cache (kq_attn.hip) shares ragged sequences out to its
// workgroups, from lengths that are on the device only.
//
// Tokens count in tiles of 32, an empty sequence as one, and what a sequence
// costs beside them as kPieceTiles before its first.  All sequences' tiles in a
// row, T of them, are cut into runs of c = max(least, ceil(T / runs)), one for
// each workgroup of a head: all have the same work, whatever the lengths are.
// A run is pieces of sequences.  A sequence inside one run is
// done by its workgroup; one that is cut has pieces in runs x0 .. x1, whose
// results go to places 2 x0 + 1, 2 (x0 + 1), 2 (x0 + 2) ..: a run has at most
// one piece that begins inside its sequence (its first) and one that ends
// there (its last).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kq {

namespace {

constexpr int kTileTokens = 32;
constexpr int kLeastTiles = 4;   // of a run: a tile for each of a workgroup's waves (1000 tokens in bf16 took 8.4 us, with 8 9.0: p as two terms)

// What a piece costs beside its tiles (its first loads, which nothing overlaps, and its result), in tiles: 64 ragged
// sequences of up to 8192 tokens in MXFP4 took 70 us with 0, 59 with 4, 51 with 8, 50 with 12, 52 with 20 (with 12 now 47 and the join's 5).
constexpr int kPieceTiles = 12;

// The tokens of a sequence that count: first .. end - 1; tiles start at multiples of 32.
struct Span {
    int first, end;
    __host__ __device__ __forceinline__ Span(int length, int64_t max_tokens, int64_t window) {
        const int64_t n = length < 0 ? 0 : length < max_tokens ? length : max_tokens;
        end = (int)n;
        first = window > 0 && window < n ? (int)(n - window) : 0;
    }
    __host__ __device__ __forceinline__ int first_tile() const { return first / kTileTokens; }
    // An empty sequence has one, which holds no token that counts.
    __host__ __device__ __forceinline__ int tiles() const {
        return end > first ? (end - 1) / kTileTokens + 1 - first_tile() : 1;
    }
};

// Tiles of a run, at least total / runs; `inverse` is 1 / runs.  (2^20 sequences in one run: up to 2^47, in 64 bits
// throughout; a piece is of one sequence, and below 2^27.)
__host__ __device__ __forceinline__ int64_t run_tiles(uint64_t total, double inverse) {
    const double c = (double)total * inverse * (1.0 + 0x1p-50);  // (total < 2^47: the product's errors are below that factor's)
    const int64_t n = (int64_t)c + ((double)(int64_t)c < c);
    return n > kLeastTiles ? n : kLeastTiles;
}
// Places for the results of pieces.
__host__ __device__ __forceinline__ int64_t run_slots(int64_t runs) { return 2 * runs; }

// Which of a sequence's pages holds token `token`; tokens from `end` (at least 1) on are looked up in the last one.
__host__ __device__ __forceinline__ int page_index(int token, int end, int page_shift) {
    const int at = token >> page_shift, last = (end - 1) >> page_shift;
    return at < last ? at : last;
}
// The page of a table's entry: the nearest one of the cache.
__host__ __device__ __forceinline__ int64_t page_of(int32_t entry, int64_t pages) {
    return entry < 0 ? 0 : entry < pages ? entry : pages - 1;
}

// A workgroup's run: from tile `skip` - kPieceTiles of sequence b on, `tiles` in all (0: none).
struct Run {
    int b;
    int length;  // its tokens, as given
    int skip;
    int64_t tiles;
    int64_t each;  // of every run
};

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_sum(uint32_t v) {
    return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
// The sum of the lanes up to and with each, in 32 bits.
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
    v = dpp_sum<0x111, 0xf>(v);  // row_shr 1, 2, 4, 8: sums up to the lane in its row of 16
    v = dpp_sum<0x112, 0xf>(v);
    v = dpp_sum<0x114, 0xf>(v);
    v = dpp_sum<0x118, 0xf>(v);
    v = dpp_sum<0x142, 0xa>(v);  // rows 0 and 2 onto 1 and 3, then 1 onto 2 and 3
    return dpp_sum<0x143, 0xc>(v);
}
__device__ __forceinline__ int lane_value(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

// Run x, found by each of a workgroup's waves: two passes over the lengths, 64 at a time; one where there are no more than
// 64.  Their own tiles are added up in 32 bits, which hold those of 64 sequences at the limit of 2^31 - 64 tokens; what their
// pieces cost beside them is a multiple of the number of sequences, added in 64 bits.
static_assert(64 * (((int64_t(1) << 31) - 64) / kTileTokens) < int64_t(1) << 32, "64 sequences' tiles in 32 bits");
__device__ __forceinline__ Run find_run(const int32_t* lengths, int B, int64_t max_tokens, int64_t window, double inverse, int x) {
    const int lane = threadIdx.x & 63;
    int length = lane < B ? lengths[lane] : 0;
    auto tiles = [&](int b) __attribute__((always_inline)) { return b < B ? (uint32_t)Span(length, max_tokens, window).tiles() : 0u; };
    uint32_t n = tiles(lane), upto;
    uint64_t total = (uint64_t)kPieceTiles * (uint32_t)B;
    for (int b0 = 0;;) {
        upto = wave_scan(n);
        total += (uint32_t)lane_value((int)upto, 63);
        b0 += 64;
        if (b0 >= B) break;
        length = b0 + lane < B ? lengths[b0 + lane] : 0;
        n = tiles(b0 + lane);
    }
    Run r{0, 0, 0, 0, run_tiles(total, inverse)};
    const uint64_t from = (uint64_t)x * (uint64_t)r.each;
    if (from >= total) return r;
    uint64_t before = 0;
    for (int b0 = 0; b0 < B; b0 += 64) {
        if (B > 64) {
            length = b0 + lane < B ? lengths[b0 + lane] : 0;
            n = tiles(b0 + lane);
            upto = wave_scan(n);
        }
        // (lanes past the last sequence come after one that holds `from`)
        const uint64_t here = __ballot(before + upto + (uint32_t)(kPieceTiles * (lane + 1)) > from);
        if (here) {
            const int at = __ffsll((unsigned long long)here) - 1;
            r.b = b0 + at;
            r.length = lane_value(length, at);
            r.skip = (int)(from - before - (uint32_t)(lane_value((int)upto, at) - lane_value((int)n, at)) - (uint32_t)(kPieceTiles * at));
            r.tiles = (int64_t)(total - from) < r.each ? (int64_t)(total - from) : r.each;
            return r;
        }
        before += (uint32_t)lane_value((int)upto, 63) + (uint64_t)(64 * kPieceTiles);
    }
    return r;
}

}  // namespace

}  // namespace kq
