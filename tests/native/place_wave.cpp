// csrc/kq_place.h on the CPU: one wave's 64 lanes as coroutines that meet at every operation across
// lanes.  Reads cases from stdin: "M N bn bm E blocks..." with counts before lists, prints for every
// block "-" (no tile) or "expert nb0 mb0 end".
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>
#include <ucontext.h>

#include <algorithm>
#include <memory>
#include <vector>

using std::max;
using std::min;

namespace wave {
constexpr int kLanes = 64;
struct Id {
    unsigned x;
};
Id block, grid;
int lane;  // the one that runs
ucontext_t scheduler, lanes[kLanes];
int slot[2][kLanes];
int turn[kLanes];  // operations across lanes so far

void meet() { swapcontext(&lanes[lane], &scheduler); }

// Every lane's v, once all have come here (slots alternate: no lane is two operations ahead).
const int* share(int v) {
    int* const s = slot[turn[lane]++ & 1];
    s[lane] = v;
    meet();
    return s;
}
}  // namespace wave

struct ThreadIdx {
    struct X {
        operator unsigned() const { return (unsigned)wave::lane; }
    } x;
};
static ThreadIdx threadIdx;
#define blockIdx wave::block
#define gridDim wave::grid

// Lanes that no enabled row or no source lane writes keep `old`.
static int dpp(int old, int v, int ctrl, int rows) {
    const int* const s = wave::share(v);
    const int l = wave::lane, row = l / 16;
    if (!(rows >> row & 1)) return old;
    if (ctrl > 0x110 && ctrl < 0x120) return l % 16 >= ctrl - 0x110 ? s[l - (ctrl - 0x110)] : old;  // row_shr
    if (ctrl == 0x142) return row ? s[16 * row - 1] : old;                                         // row_bcast 15
    if (ctrl == 0x143) return row >= 2 ? s[31] : old;                                              // row_bcast 31
    abort();
}
#define __builtin_amdgcn_update_dpp(old, v, ctrl, rows, banks, bound) dpp(old, v, ctrl, rows)
static int readlane(int v, int l) { return wave::share(v)[l]; }
#define __builtin_amdgcn_readlane readlane
static uint64_t ballot(bool b) {
    const int* const s = wave::share(b);
    uint64_t m = 0;
    for (int l = 0; l < wave::kLanes; ++l) m |= (uint64_t)(s[l] != 0) << l;
    return m;
}
#define __ballot ballot

#include "kq_place.h"

namespace {
kq::LinearParams params;
int bn, bm;
struct Result {
    bool tile;
    int64_t expert, nb0, mb0, end;
} result[wave::kLanes];

void lane_main() {
    kq::LinearParams p = params;
    Result r{};
    r.tile = kq::place<true>(p, bn, bm, r.nb0, r.mb0);
    if (r.tile) {
        r.expert = (p.g.b_codes - params.g.b_codes) / (params.g.N * (params.g.K / 2));
        r.end = p.g.M;
    }
    result[wave::lane] = r;
}
}  // namespace

int main() {
    std::vector<std::unique_ptr<char[]>> stack;
    constexpr size_t kStack = 64 << 10;
    for (int l = 0; l < wave::kLanes; ++l) stack.emplace_back(new char[kStack]);
    long long M, N, E, grid, blocks;
    static uint8_t base;
    while (scanf("%lld %lld %d %d %lld %lld", &M, &N, &bn, &bm, &grid, &E) == 6) {
        std::vector<int32_t> offsets(E + 1);
        for (auto& o : offsets)
            if (scanf("%d", &o) != 1) return 2;
        params = kq::LinearParams{};
        params.g.M = M;
        params.g.N = N;
        params.g.K = 32;
        params.g.b_codes = params.g.b_scales = &base;
        params.offsets = offsets.data();
        params.experts = E;
        wave::grid.x = (unsigned)grid;
        if (scanf("%lld", &blocks) != 1) return 2;
        for (; blocks; --blocks) {
            long long b;
            if (scanf("%lld", &b) != 1) return 2;
            wave::block.x = (unsigned)b;
            for (int l = 0; l < wave::kLanes; ++l) {
                getcontext(&wave::lanes[l]);
                wave::lanes[l].uc_stack.ss_sp = stack[l].get();
                wave::lanes[l].uc_stack.ss_size = kStack;
                wave::lanes[l].uc_link = &wave::scheduler;
                makecontext(&wave::lanes[l], lane_main, 0);
                wave::turn[l] = 0;
                result[l] = Result{false, -1, -1, -1, -1};
            }
            // a round runs every lane to its next meeting; they all end in the same one
            int last;
            do {
                last = wave::turn[wave::kLanes - 1];
                for (int l = 0; l < wave::kLanes; ++l) {
                    wave::lane = l;
                    swapcontext(&wave::scheduler, &wave::lanes[l]);
                }
                for (int l = 1; l < wave::kLanes; ++l)
                    if (wave::turn[l] != wave::turn[0]) return 3;  // lanes that part
            } while (wave::turn[wave::kLanes - 1] != last);
            for (int l = 1; l < wave::kLanes; ++l) {
                const Result &r = result[l], &s = result[0];
                if (r.tile != s.tile || r.expert != s.expert || r.nb0 != s.nb0 || r.mb0 != s.mb0 || r.end != s.end) return 4;
            }
            if (!result[0].tile) puts("-");
            else printf("%lld %lld %lld %lld\n", (long long)result[0].expert, (long long)result[0].nb0, (long long)result[0].mb0, (long long)result[0].end);
        }
    }
    return 0;
}
