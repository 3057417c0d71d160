// Where a workgroup of a W4A4 linear layer (kq_linear.hip) works: its tile of C, and in a grouped
// call its expert.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kq_linear.h"

namespace kq {

namespace {

// Row tiles of bm rows that any valid offsets of a grouped call can need: every group may end inside one.
__host__ __device__ __forceinline__ int64_t group_tiles(int64_t rows, int64_t experts, int64_t bm) {
    return rows / bm + (experts < rows ? experts : rows);
}

// The lane's sum with another's, at most `most` (sums are at most that, which is below 2^31).
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_add(uint32_t v, uint32_t most) {
    return min(v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false), most);
}

// xcd_tile for fewer than 2^31 workgroups, which every launch here has: its divisions in 32 bits.
__device__ __forceinline__ void xcd_tile32(uint32_t gx, uint32_t gy, int64_t& tn, int64_t& tm) {
    const uint32_t T = gx * gy, i = blockIdx.x, k = i % 8, j = i / 8;
    const uint32_t L = k * (T / 8) + min(k, T % 8) + j;
    const uint32_t q = L / (4 * gx), r = L - q * 4 * gx, gm = min(gy - 4 * q, 4u);
    const uint32_t n = gm == 4 ? r / 4 : r / gm;
    tn = n;
    tm = 4 * q + (r - n * gm);
}

// Experts e0 .. e0 + 63 of a grouped call, one a lane: its rows, and the row tiles of bm rows up to and with it, from
// `before` on.  Offsets outside [0, M] or decreasing are taken as an empty or a shorter group.  Groups that then
// overlap may have more tiles than the launch, and than 32 bits hold: sums end at `most`, the launch's.
struct Groups {
    int first, end;
    uint32_t cum;
    __device__ __forceinline__ Groups(const LinearParams& p, int e0, int bm, uint32_t most, uint32_t before) {
        const int lane = threadIdx.x & 63, e = e0 + lane, M = (int)p.g.M;
        first = end = 0;
        if (e < p.experts) {
            const int a = p.offsets[e], b = p.offsets[e + 1];
            first = min(max(a, 0), M);
            end = min(max(b, first), M);
        }
        cum = min((uint32_t)((end - first) / bm + ((end - first) % bm != 0)), most);
        cum = dpp_add<0x111, 0xf>(cum, most);  // row_shr 1, 2, 4, 8: sums up to the lane in its row of 16
        cum = dpp_add<0x112, 0xf>(cum, most);
        cum = dpp_add<0x114, 0xf>(cum, most);
        cum = dpp_add<0x118, 0xf>(cum, most);
        cum = dpp_add<0x142, 0xa>(cum, most);  // rows 0 and 2 onto 1 and 3, then 1 onto 2 and 3
        cum = min(dpp_add<0x143, 0xc>(cum, most) + before, most);
    }
    __device__ __forceinline__ uint32_t total() const { return (uint32_t)__builtin_amdgcn_readlane((int)cum, 63); }
};

// The tile of workgroup blockIdx.x: its place in C, and p narrowed to its expert.  False: none is left
// (the host's grid is the most that any valid offsets can need).
template <bool GROUPED>
__device__ __forceinline__ bool place(LinearParams& p, int bn, int bm, int64_t& nb0, int64_t& mb0) {
    const uint32_t gx = (uint32_t)((p.g.N + bn - 1) / bn);
    int64_t tn, tm;
    if (!GROUPED) {
        xcd_tile32(gx, (uint32_t)((p.g.M + bm - 1) / bm), tn, tm);
        nb0 = tn * bn;
        mb0 = tm * bm;
        return true;
    }
    const uint32_t most = (uint32_t)group_tiles(p.g.M, p.experts, bm);  // gx most workgroups are launched
    int e0 = 0;
    uint32_t before = 0;
    Groups g(p, 0, bm, most, 0);
    uint32_t total = g.total();
    const bool more = p.experts > 64;
    for (int e = 64; e < p.experts; e += 64) total = Groups(p, e, bm, most, total).total();
    if (blockIdx.x >= gx * total) return false;
    xcd_tile32(gx, total, tn, tm);
    while (more && g.total() <= tm && e0 + 64 < p.experts) {
        before = g.total();
        e0 += 64;
        g = Groups(p, e0, bm, most, before);
    }
    const uint64_t past = __ballot(g.cum > (uint32_t)tm);
    if (!past) return false;
    // the sums up to the lane before are at most tm, so that the tile is one of this lane's
    const int l = __builtin_ctzll(past), e = e0 + l;
    const int first = __builtin_amdgcn_readlane(g.first, l), end = __builtin_amdgcn_readlane(g.end, l);
    const uint32_t tile = (uint32_t)tm - (l ? (uint32_t)__builtin_amdgcn_readlane((int)g.cum, l - 1) : before);
    nb0 = tn * bn;
    mb0 = first + (int64_t)tile * bm;
    p.g.M = end;
    p.g.b_codes += e * p.g.N * (p.g.K / 2);
    p.g.b_scales += e * p.g.N * (p.g.K / 32);
    if (p.bias) p.bias = static_cast<const uint8_t*>(p.bias) + e * p.g.N * (p.vec16 ? 2 : 4);
    return true;
}

}  // namespace

}  // namespace kq
