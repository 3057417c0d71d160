// csrc/kq_split.h on the CPU: one wave's 64 lanes as coroutines that meet at every operation across
// lanes.  Reads cases from stdin: "B max_tokens window runs lengths... blocks..." with the number of
// blocks before them, prints for every block "b skip tiles each".
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <ucontext.h>

#include <memory>
#include <vector>

namespace wave {
constexpr int kLanes = 64;
int lane;  // the one that runs
ucontext_t scheduler, lanes[kLanes];
int64_t slot[2][kLanes];
int turn[kLanes];  // operations across lanes so far

// Every lane's v, once all have come here (slots alternate: no lane is two operations ahead).
const int64_t* share(int64_t v) {
    int64_t* const s = slot[turn[lane]++ & 1];
    s[lane] = v;
    swapcontext(&lanes[lane], &scheduler);
    return s;
}
}  // namespace wave

struct ThreadIdx {
    struct X {
        operator unsigned() const { return (unsigned)wave::lane; }
    } x;
};
static ThreadIdx threadIdx;

// Lanes that no enabled row or no source lane writes keep `old`.
static int dpp(int old, int v, int ctrl, int rows) {
    const int64_t* const s = wave::share(v);
    const int l = wave::lane, row = l / 16;
    if (!(rows >> row & 1)) return old;
    if (ctrl > 0x110 && ctrl < 0x120) return l % 16 >= ctrl - 0x110 ? (int)s[l - (ctrl - 0x110)] : old;  // row_shr
    if (ctrl == 0x142) return row ? (int)s[16 * row - 1] : old;                                         // row_bcast 15
    if (ctrl == 0x143) return row >= 2 ? (int)s[31] : old;                                              // row_bcast 31
    abort();
}
#define __builtin_amdgcn_update_dpp(old, v, ctrl, rows, banks, bound) dpp(old, v, ctrl, rows)
static int readlane(int v, int l) { return (int)wave::share(v)[l]; }
static uint64_t ballot(bool b) {
    const int64_t* const s = wave::share(b);
    uint64_t m = 0;
    for (int l = 0; l < wave::kLanes; ++l) m |= (uint64_t)(s[l] != 0) << l;
    return m;
}
#define __ballot ballot
#define __ffsll(v) __builtin_ffsll((long long)(v))
#define __builtin_amdgcn_readlane readlane

#include "kq_split.h"

namespace {
std::vector<int32_t> lengths;
long long B, max_tokens, window, runs, block;
kq::Run result[wave::kLanes];

void lane_main() {
    const int l = wave::lane;
    result[l] = kq::find_run(lengths.data(), (int)B, max_tokens, window, 1.0 / runs, (int)block);
}
}  // namespace

int main(int argc, char** argv) {
    if (argc == 5) {  // token end page_shift entry: the page's place in a sequence, and the page of 10
        printf("%d %lld\n", kq::page_index(atoi(argv[1]), atoi(argv[2]), atoi(argv[3])), (long long)kq::page_of(atoi(argv[4]), 10));
        return 0;
    }
    std::vector<std::unique_ptr<char[]>> stack;
    constexpr size_t kStack = 64 << 10;
    for (int l = 0; l < wave::kLanes; ++l) stack.emplace_back(new char[kStack]);
    long long blocks;
    while (scanf("%lld %lld %lld %lld", &B, &max_tokens, &window, &runs) == 4) {
        lengths.assign(B, 0);
        for (auto& n : lengths)
            if (scanf("%d", &n) != 1) return 2;
        if (scanf("%lld", &blocks) != 1) return 2;
        for (; blocks; --blocks) {
            if (scanf("%lld", &block) != 1) return 2;
            for (int l = 0; l < wave::kLanes; ++l) {
                getcontext(&wave::lanes[l]);
                wave::lanes[l].uc_stack.ss_sp = stack[l].get();
                wave::lanes[l].uc_stack.ss_size = kStack;
                wave::lanes[l].uc_link = &wave::scheduler;
                makecontext(&wave::lanes[l], lane_main, 0);
                wave::turn[l] = 0;
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
            const kq::Run& r = result[0];
            for (int l = 1; l < wave::kLanes; ++l)
                if (result[l].b != r.b || result[l].length != r.length || result[l].skip != r.skip || result[l].tiles != r.tiles || result[l].each != r.each) return 4;
            if (r.tiles && r.length != lengths[r.b]) return 5;
            printf("%d %d %lld %lld\n", r.b, r.skip, (long long)r.tiles, (long long)r.each);
        }
    }
    return 0;
}
