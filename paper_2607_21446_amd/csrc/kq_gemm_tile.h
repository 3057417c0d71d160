// Tiles of the W4A4 products (kq_gemm.hip, kq_linear.hip): both operands in the
// MXFP4 layout the quantizer writes, codes [rows, K/2] and E8M0 scales [rows, K/32].
// The pipelined tile leaves its sums in accumulators, the split tile in LDS.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kq_kernels.h"
#include "kq_lds.h"

namespace kq {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16g __attribute__((ext_vector_type(16)));

namespace {

// One lane's share of a K step: the 16 code bytes of one block (as the low
// half of the 8-dword operand; E2M1 uses 4 dwords) and its scale byte.
struct Frag {
    uint4 codes;
    uint32_t scale;
};

__device__ __forceinline__ i32x8 operand(const Frag& f) {
    i32x8 v = {(int)f.codes.x, (int)f.codes.y, (int)f.codes.z, (int)f.codes.w, 0, 0, 0, 0};
    return v;
}

// C, the bias and the 16-bit C are accessed in whole vectors at any alignment of their
// elements (global memory takes such accesses, and the rows of an odd ldc start anywhere).
// With vectors only where all rows were 16-byte aligned and single elements elsewhere,
// us: 4608 x 3001 x 3072 bf16 54.9 with the quantizer, 40.0 now; 4608 x 3004 x 1152 38.8
// and 23.5 (3072 columns: 23.1); 4096 x 3001 x 1152 fp32 37.5 and 26.7.
typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32b __attribute__((aligned(2)));
typedef uint32_t u32x2b __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4b __attribute__((ext_vector_type(4), aligned(2)));

// A value that is the same in all lanes, in scalar registers: the compiler's own choice may be vector ones, which
// the loads into LDS do not take as their base.
template <class T>
__device__ __forceinline__ T scalar(T v) {
    static_assert(sizeof(T) == 8, "two registers");
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u), hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
    return __builtin_bit_cast(T, ((uint64_t)hi << 32) | lo);
}

// The row of a_codes that row m of X is (any index is kept inside the array).
__device__ __forceinline__ int64_t gathered(const GemmParams& g, int64_t m) {
    return min(max((int64_t)g.rows[m], (int64_t)0), g.a_rows - 1);
}

}  // namespace

// ------------------------------------------------------------------ pipelined kernels
// K advances 128 (four 32-blocks) per stage.  Codes and scales go from global
// memory straight into LDS (global_load_lds: lane l's 16 bytes land at the
// wave-uniform LDS address + 16 l), three stages ahead, so there is no register
// staging and no ds_write (scale rows that no such load can take: see DMA_SCALES).
constexpr int kStages = 4;  // LDS stage buffers: one in use, three in flight

// Until at most 4 * later code loads of this wave are outstanding.
__device__ __forceinline__ void wait_stage(int later) {
    if (later >= 2) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    else if (later == 1) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// LDS slot of block b of tile row q: 4 q + (b ^ ((q >> 2) & 3)).  A DMA
// instruction fills 64 consecutive slots (16 rows), so lane l reads row
// 16 i + l / 4, block (l % 4) ^ (((l / 4) >> 2) & 3): each instruction reads
// 16 contiguous 64-byte row segments, and a fragment read (32 rows, one
// block) spreads over all LDS banks.
__device__ __forceinline__ int pipe_slot(int q, int b) { return 4 * q + (b ^ ((q >> 2) & 3)); }

// Workgroup tile of BN (N) x BM (M): WN x WM waves of TN x TM instruction tiles
// of 32 x 32.  Every wave issues four code loads (16 rows x 64 bytes each) per
// stage and one scale load (64 rows x 16 bytes) per four stages.
template <int WN, int WM, int TN, int TM>
struct Tile {
    static constexpr int BN = 32 * WN * TN, BM = 32 * WM * TM, ROWS = BN + BM, WAVES = WN * WM;
    static_assert(ROWS == 64 * WAVES, "four code loads and one scale load per wave");
    // rows 0 .. BN-1 are W rows, BN .. ROWS-1 X rows, in every array
    struct Lds {
        uint4 codes[kStages][4 * ROWS];  // slot pipe_slot(row, block of the stage)
        uint4 scales[2][ROWS];           // [chunk parity][row]: the 16 scales of four stages
    };
};

// The 16 (or the last nvalid) scale bytes at p, any alignment.  Fewer than 16 come as
// up to four loads of 8, 4, 2 and 1 bytes that are all in flight before the first is
// waited for.  Byte by byte each load was waited for by itself, up to 15 memory latencies
// in a row; calls of K 320, 480, 1120 and 2240 took 3, 4, 0.6 and 1.3 % longer so.
__device__ __forceinline__ uint4 load_scales16(const uint8_t* p, int nvalid) {
    typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(1)));
    typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(1)));
    typedef uint32_t u32u __attribute__((aligned(1)));
    typedef uint16_t u16u __attribute__((aligned(1)));
    if (nvalid >= 16) {
        const u32x4u v = *reinterpret_cast<const u32x4u*>(p);
        return make_uint4(v.x, v.y, v.z, v.w);
    }
    u32x2u e = {0u, 0u};
    uint32_t q = 0u, d = 0u, b = 0u;
    if (nvalid & 8) e = *reinterpret_cast<const u32x2u*>(p);
    if (nvalid & 4) q = *reinterpret_cast<const u32u*>(p + (nvalid & 8));
    if (nvalid & 2) d = *reinterpret_cast<const u16u*>(p + (nvalid & 12));
    if (nvalid & 1) b = p[nvalid & 14];
    // the dword that the last 3 bytes begin
    const uint32_t tail = d | (b << (8 * (nvalid & 2)));
    uint32_t w[4] = {e.x, e.y, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i == (nvalid & 8) / 4) w[i] |= q;
        if (i == (nvalid & 12) / 4) w[i] |= tail;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// C tile [nb0, nb0 + BN) x [mb0, mb0 + BM).  Rows past N or M read row N-1 or
// M-1 (their products land in C rows or columns that are never stored).
//
// PING (eight waves, two per SIMD): waves 4-7 run half a stage behind waves
// 0-3, held apart by one extra barrier at the start, so that on every SIMD one
// wave reads its fragments from LDS and issues loads while the other runs its
// matrix-core instructions; with both in step the LDS reads (about 770 cycles a
// stage at 128 bytes a cycle) and the matrix cores (1024 cycles) add up.
// In phase 2k waves 0-3 read stage k and issue stage k + 3, and compute it in
// phase 2k + 1; waves 4-7 do so in phases 2k + 1 and 2k + 2.  Stage k + 3
// overwrites the buffer of stage k - 1, last read in phase 2k - 1, whose reads
// have returned before that phase's barrier.  Every wave has waited for its
// loads of stage k before the barrier that ends phase 2k - 1.
//
// Per stage (K 12288 less K 3072, 216 tiles, C stores left out): 0.91 us, of which
// 0.59 is what the matrix cores take at the clock they hold; 0.75 without the
// loads, 0.69 without the matrix instructions.  Both groups in step, with three
// buffers: 1.15 us.
//
// DMA_SCALES: a scale row has a multiple of 4 bytes, at least 16, and starts
// at a multiple of 4: the 16 scales of four stages come by a DMA load per row.
// The last such load of the last row would pass the end of the array, so it
// ends there instead and is read at an offset.  Otherwise each thread loads
// its row's 16 bytes into registers (byte-exact) and parks them in LDS two
// stages later; the compiler waits for them with vmcnt(0), which drains the stages in
// flight once per four stages (the other path never does).
//
// GATHER: row r of X is row g.rows[r] of a_codes and a_scales (32-bit offsets of the whole
// array); the last chunk's scales of every such row are loaded early.
template <int WN, int WM, int TN, int TM, bool PING, bool DMA_SCALES, bool GATHER = false>
__device__ __forceinline__ void gemm_tile(const GemmParams& g, typename Tile<WN, WM, TN, TM>::Lds& lds, int64_t nb0,
                                          int64_t mb0, f32x16g (&acc)[TN][TM]) {
    typedef Tile<WN, WM, TN, TM> T;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int r = lane & 31, h = lane >> 5, wn = wave / WM, wm = wave % WM;
    const int64_t row_bytes = g.K / 2, nkb = g.K / 32;
    const int nst = (int)((nkb + 3) / 4), tb = (int)(nkb & 3);  // tb: blocks of a partial last stage
    const int nch = (int)((nkb + 15) / 16);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)&lds;
    constexpr uint32_t kStageBytes = 64u * T::ROWS;
    constexpr uint32_t kScales0 = kStages * kStageBytes, kChunkBytes = 16u * T::ROWS;

    // this wave's code rows 64 wave .. 64 wave + 63 (all W or all X), its scale rows the same
    const bool isw = 64 * wave < T::BN;
    const int rel0 = 64 * wave - (isw ? 0 : T::BN);
    const int64_t row0 = (isw ? nb0 : mb0) + rel0, rows = isw ? g.N : g.M;
    const int last = (int)min<int64_t>(63, max<int64_t>(0, rows - 1 - row0));  // last row of the 64 to read
    const bool gather = GATHER && !isw;
    const int64_t rowc = min(row0, rows - 1), row1 = gather ? 0 : rowc;
    const uint8_t* const cbase = scalar((isw ? g.b_codes : g.a_codes) + row1 * row_bytes);
    const uint8_t* const sbase = scalar((isw ? g.b_scales : g.a_scales) + row1 * nkb);
    const int q = lane >> 2, blk = (lane & 3) ^ ((q >> 2) & 3);
    auto offset = [&](int i) { return gather ? (uint32_t)gathered(g, rowc + min(i, last)) : (uint32_t)min(i, last); };
    uint32_t voff[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) voff[i] = offset(16 * i + q) * (uint32_t)row_bytes + 16u * blk;
    const uint32_t soff = offset(lane) * (uint32_t)nkb;
    const uint32_t dst0 = lds0 + 4096u * wave, sdst0 = lds0 + kScales0 + 1024u * wave;

    auto issue_codes = [&](int st, int buf) {
        const uint8_t* const base = cbase + 64 * (int64_t)st;
        // blocks past K (a partial last stage) read its last block; they are masked below
        const uint32_t back = (tb && st == nst - 1 && blk >= tb) ? 16u * (blk - tb + 1) : 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) lds_dma16(dst0 + buf * kStageBytes + 1024u * i, voff[i] - back, base);
    };
    // distance by which the last chunk's load of the matrix's last row ends early
    // (the chunk's offset is added first: a row's own offset may be smaller than it)
    const uint32_t early = DMA_SCALES ? (uint32_t)(-nkb & 15) : 0u;
    auto issue_scales = [&](int ch) {
        const bool back = early && ch == nch - 1 && (gather || row0 + min(lane, last) >= rows - 1);
        lds_dma16(sdst0 + (ch & 1) * kChunkBytes, soff + 16u * ch - (back ? early : 0u), sbase);
    };
    uint4 parked = make_uint4(0u, 0u, 0u, 0u);
    auto fetch_scales = [&](int ch) {
        parked = load_scales16(sbase + soff + 16 * (int64_t)ch, (int)min<int64_t>(16, nkb - 16 * (int64_t)ch));
    };
    auto park_scales = [&](int ch) { lds.scales[ch & 1][threadIdx.x] = parked; };

    // fragment and scale addresses of this lane
    const uint32_t psel = h ? 0x0c0c0301u : 0x0c0c0200u;
    const int wrow = wn * 32 * TN + r, xrow = T::BN + wm * 32 * TM + r;
    const uint4* const sc0 = lds.scales[0];
    uint32_t late = 0;  // bit i (W) or 8 + j (X): this lane's row is the matrix's last
    if (DMA_SCALES && early) {
#pragma unroll
        for (int i = 0; i < TN; ++i) late |= (nb0 + wrow + 32 * i >= g.N - 1 ? 1u : 0u) << i;
#pragma unroll
        for (int j = 0; j < TM; ++j) late |= (GATHER || mb0 + xrow - T::BN + 32 * j >= g.M - 1 ? 1u : 0u) << (8 + j);
    }
    struct Frags {
        uint4 w[2][TN], x[2][TM];
        uint32_t sw[TN], sx[TM];
    };
    auto read_frags = [&](int st, int buf, int j4, Frags& f) {
        const uint4* const cb = lds.codes[buf];
        const int ch = st >> 2;
        const uint32_t* const sp = reinterpret_cast<const uint32_t*>(sc0 + (ch & 1) * T::ROWS) + j4;
        if (DMA_SCALES && early && ch == nch - 1) {
            const uint32_t e = early / 4;
#pragma unroll
            for (int i = 0; i < TN; ++i) f.sw[i] = sp[4 * (wrow + 32 * i) + ((late >> i) & 1u) * e];
#pragma unroll
            for (int j = 0; j < TM; ++j) f.sx[j] = sp[4 * (xrow + 32 * j) + ((late >> (8 + j)) & 1u) * e];
        } else {
#pragma unroll
            for (int i = 0; i < TN; ++i) f.sw[i] = sp[4 * (wrow + 32 * i)];
#pragma unroll
            for (int j = 0; j < TM; ++j) f.sx[j] = sp[4 * (xrow + 32 * j)];
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int i = 0; i < TN; ++i) f.w[s][i] = cb[pipe_slot(wrow + 32 * i, 2 * s + h)];
#pragma unroll
            for (int j = 0; j < TM; ++j) f.x[s][j] = cb[pipe_slot(xrow + 32 * j, 2 * s + h)];
        }
    };
    // scales to the byte order of the instruction's selectors; blocks past K: zero codes, scale 1
    auto finish_frags = [&](int st, Frags& f) {
#pragma unroll
        for (int i = 0; i < TN; ++i) f.sw[i] = __builtin_amdgcn_perm(0u, f.sw[i], psel);
#pragma unroll
        for (int j = 0; j < TM; ++j) f.sx[j] = __builtin_amdgcn_perm(0u, f.sx[j], psel);
        if (tb && st == nst - 1) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const bool past = 2 * s + h >= tb;
                const uint32_t keep = past ? 0u : ~0u;
                const uint32_t one = past ? 127u << (8 * s) : 0u, smask = past ? ~(255u << (8 * s)) : ~0u;
#pragma unroll
                for (int i = 0; i < TN; ++i) {
                    f.w[s][i] = make_uint4(f.w[s][i].x & keep, f.w[s][i].y & keep, f.w[s][i].z & keep, f.w[s][i].w & keep);
                    f.sw[i] = (f.sw[i] & smask) | one;
                }
#pragma unroll
                for (int j = 0; j < TM; ++j) {
                    f.x[s][j] = make_uint4(f.x[s][j].x & keep, f.x[s][j].y & keep, f.x[s][j].z & keep, f.x[s][j].w & keep);
                    f.sx[j] = (f.sx[j] & smask) | one;
                }
            }
        }
    };
    auto products = [&](const Frags& f) {
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(Frag{f.w[0][i], 0u}),
                                                                             operand(Frag{f.x[0][j], 0u}), acc[i][j], 4, 4,
                                                                             0, (int)f.sw[i], 0, (int)f.sx[j]);
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(Frag{f.w[1][i], 0u}),
                                                                             operand(Frag{f.x[1][j], 0u}), acc[i][j], 4, 4,
                                                                             1, (int)f.sw[i], 1, (int)f.sx[j]);
    };

#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = f32x16g{};
    if (DMA_SCALES) issue_scales(0);
    else fetch_scales(0);
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s)
        if (s < nst) issue_codes(s, s);
    if (!DMA_SCALES) {
        park_scales(0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    const bool behind = PING && wave >= T::WAVES / 2;

    // stage st in buffer J = st % 4
    auto stage = [&](int st, auto Jc) {
        constexpr int J = decltype(Jc)::value;
        Frags f;
        read_frags(st, J, J, f);
        if (DMA_SCALES) {
            if (J == 0 && (st >> 2) + 1 < nch) issue_scales((st >> 2) + 1);
        } else {
            if (J == 2 && (st >> 2) + 1 < nch) park_scales((st >> 2) + 1);
            if (J == 0 && (st >> 2) + 1 < nch) fetch_scales((st >> 2) + 1);
        }
        if (st + 3 < nst) issue_codes(st + 3, (J + 3) & 3);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        finish_frags(st, f);
        if (PING) {
            if (behind) wait_stage(nst - 2 - st);
            stage_barrier();
            products(f);
            if (!behind) wait_stage(nst - 2 - st);
            stage_barrier();
        } else {
            products(f);
            wait_stage(nst - 2 - st);
            stage_barrier();
        }
    };
    wait_stage(nst - 1);
    stage_barrier();
    if (behind) stage_barrier();
    for (int st = 0; st < nst; st += 4) {
        stage(st, std::integral_constant<int, 0>{});
        if (st + 1 < nst) stage(st + 1, std::integral_constant<int, 1>{});
        if (st + 2 < nst) stage(st + 2, std::integral_constant<int, 2>{});
        if (st + 3 < nst) stage(st + 3, std::integral_constant<int, 3>{});
    }
    if (PING && !behind) stage_barrier();
}

// Tile of workgroup blockIdx.x of gx x gy tiles.  Workgroups
// are dealt to the 8 XCDs round-robin by linear id, so XCD k runs ids
// k, k + 8, ...; those get consecutive logical ids (a bijection for any
// count), and logical ids walk the tiles in groups of 4 M rows (N fastest
// within a group, M fastest within a column), so each XCD's L2 sees a compact
// block of about 4 x (T / 32) tiles instead of every M row.
__device__ __forceinline__ void xcd_tile(int64_t gx, int64_t gy, int64_t& tn, int64_t& tm) {
    const int64_t T = gx * gy;
    const int64_t i = blockIdx.x;
    const int64_t k = i % 8, j = i / 8;
    const int64_t L = k * (T / 8) + (k < T % 8 ? k : T % 8) + j;
    constexpr int64_t GM = 4;
    const int64_t gsize = GM * gx;
    const int64_t first_m = (L / gsize) * GM;
    const int64_t gm = gy - first_m < GM ? gy - first_m : GM;
    tm = first_m + (L % gsize) % gm;
    tn = (L % gsize) / gm;
}

// Few tiles: W waves share one tile of 32 TM (M) x 32 TN (N), each taking every W-th
// 128-wide chunk of K with fragments straight from global memory (D chunks in flight),
// and their sums meet in LDS in wave order.  With fewer tiles than CUs the pipelined
// kernels walk K alone, a memory latency or more per few stages; here K is as wide as
// the workgroup.
// Returns how many waves had a share; wave w's sums are sums[(w BM + row) RS + column].
template <int TN, int TM, int W, int D, bool GATHER = false>
__device__ __forceinline__ int split_tile(const GemmParams& g, float* sums, int64_t nb0, int64_t mb0) {
    constexpr int BM = 32 * TM, RS = 32 * TN + 4;  // LDS row in floats
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63;
    const int r = lane & 31, h = lane >> 5;
    const int64_t nkb = g.K / 32, row_bytes = g.K / 2;
    const int nch = (int)((nkb + 3) / 4), tb = (int)(nkb & 3);
    // rows past N or M read the last row (their sums are never stored)
    const uint8_t *cw[TN], *cx[TM], *sw[TN], *sx[TM];
#pragma unroll
    for (int i = 0; i < TN; ++i) {
        const int64_t n = min(nb0 + 32 * i + r, g.N - 1);
        cw[i] = g.b_codes + n * row_bytes;
        sw[i] = g.b_scales + n * nkb;
    }
#pragma unroll
    for (int j = 0; j < TM; ++j) {
        int64_t m = min(mb0 + 32 * j + r, g.M - 1);
        if (GATHER) m = gathered(g, m);
        cx[j] = g.a_codes + m * row_bytes;
        sx[j] = g.a_scales + m * nkb;
    }
    struct Chunk {
        uint4 w[2][TN], x[2][TM];
        uint32_t sw[TN], sx[TM];
    };
    auto scales4 = [&](const uint8_t* p, int valid) {
        typedef uint32_t u32u __attribute__((aligned(1)));
        if (valid >= 4) return *reinterpret_cast<const u32u*>(p);
        uint32_t v = p[0];
        if (valid > 1) v |= (uint32_t)p[1] << 8;
        if (valid > 2) v |= (uint32_t)p[2] << 16;
        return v;
    };
    auto load = [&](int c, Chunk& f) {
        const int valid = (tb && c == nch - 1) ? tb : 4;  // blocks of the chunk; those past K read its last block
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int64_t at = 16 * (4 * (int64_t)c + min(2 * s + h, valid - 1));
#pragma unroll
            for (int i = 0; i < TN; ++i) f.w[s][i] = *reinterpret_cast<const uint4*>(cw[i] + at);
#pragma unroll
            for (int j = 0; j < TM; ++j) f.x[s][j] = *reinterpret_cast<const uint4*>(cx[j] + at);
        }
#pragma unroll
        for (int i = 0; i < TN; ++i) f.sw[i] = scales4(sw[i] + 4 * (int64_t)c, valid);
#pragma unroll
        for (int j = 0; j < TM; ++j) f.sx[j] = scales4(sx[j] + 4 * (int64_t)c, valid);
    };
    const uint32_t psel = h ? 0x0c0c0301u : 0x0c0c0200u;
    f32x16g acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = f32x16g{};
    auto multiply = [&](int c, Chunk& f) {
#pragma unroll
        for (int i = 0; i < TN; ++i) f.sw[i] = __builtin_amdgcn_perm(0u, f.sw[i], psel);
#pragma unroll
        for (int j = 0; j < TM; ++j) f.sx[j] = __builtin_amdgcn_perm(0u, f.sx[j], psel);
        if (tb && c == nch - 1) {  // blocks past K: zero codes, scale 1
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const bool past = 2 * s + h >= tb;
                const uint32_t keep = past ? 0u : ~0u, one = past ? 127u << (8 * s) : 0u, sm = past ? ~(255u << (8 * s)) : ~0u;
#pragma unroll
                for (int i = 0; i < TN; ++i) {
                    f.w[s][i] = make_uint4(f.w[s][i].x & keep, f.w[s][i].y & keep, f.w[s][i].z & keep, f.w[s][i].w & keep);
                    f.sw[i] = (f.sw[i] & sm) | one;
                }
#pragma unroll
                for (int j = 0; j < TM; ++j) f.sx[j] = (f.sx[j] & sm) | one;
            }
        }
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(Frag{f.w[0][i], 0u}),
                                                                             operand(Frag{f.x[0][j], 0u}), acc[i][j], 4, 4,
                                                                             0, (int)f.sw[i], 0, (int)f.sx[j]);
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(Frag{f.w[1][i], 0u}),
                                                                             operand(Frag{f.x[1][j], 0u}), acc[i][j], 4, 4,
                                                                             1, (int)f.sw[i], 1, (int)f.sx[j]);
    };
    Chunk f[D];
#pragma unroll
    for (int u = 0; u < D; ++u)
        if (wave + u * W < nch) load(wave + u * W, f[u]);
    for (int c = wave; c < nch; c += D * W) {
#pragma unroll
        for (int u = 0; u < D; ++u) {
            const int cu = c + u * W;
            if (cu < nch) {
                multiply(cu, f[u]);
                if (cu + D * W < nch) load(cu + D * W, f[u]);
            }
        }
    }
    // acc[i][j][4q + e] = (row 32 j + r, column 32 i + 8 q + 4 h + e)
    const int active = min(W, nch);
    if (wave < active) {
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<float4*>(sums + (wave * BM + 32 * j + r) * RS + 32 * i + 8 * q + 4 * h) =
                        make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
    }
    __syncthreads();
    return active;
}

}  // namespace kq
