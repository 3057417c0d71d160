"""Where the workgroups of a grouped W4A4 product work (csrc/kq_place.h), on the CPU:
every tile of every group once for offsets as they should be, and for any others no
tile outside the array, sums of tiles past 32 bits among them."""
import os
import random
import shutil
import subprocess

import pytest

from conftest import ROOT

INT32_MAX = 2 ** 31 - 1


@pytest.fixture(scope="module")
def place(tmp_path_factory):
    """place(M, N, bn, bm, offsets, blocks): per block None or (expert, first column, first row, group's end)."""
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    if not shutil.which("g++") or not os.path.isdir(os.path.join(rocm, "include", "hip")):
        pytest.skip("no g++ or no HIP headers")
    binary = str(tmp_path_factory.mktemp("place") / "place_wave")
    built = subprocess.run(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__=1", "-fwrapv",
                            "-I", os.path.join(rocm, "include"), "-I", os.path.join(ROOT, "paper_2607_21446_amd", "csrc"),
                            "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "native", "place_wave.cpp"), "-o", binary],
                           capture_output=True, text=True)
    assert built.returncode == 0, built.stderr

    def run(M, N, bn, bm, offsets, blocks):
        words = [M, N, bn, bm, _grid(M, N, bn, bm, len(offsets) - 1), len(offsets) - 1, *offsets, len(blocks), *blocks]
        done = subprocess.run([binary], input=" ".join(map(str, words)), capture_output=True, text=True, timeout=100)
        assert done.returncode == 0, (done.returncode, done.stderr)
        return [None if line == "-" else tuple(map(int, line.split())) for line in done.stdout.splitlines()]

    return run


def _grid(M, N, bn, bm, E):
    """Workgroups of a launch: the most that any valid offsets can need."""
    return -(-N // bn) * (M // bm + min(E, M))


@pytest.mark.parametrize("counts", [[1], [0, 3, 0], [16, 15, 17, 0, 33], [0] * 64 + [2, 0, 1], [5] * 130, [0, 700, 0, 1100], [1] * 65,
                                    [129] * 64 + [1]])
@pytest.mark.parametrize("lead,tail", [(0, 0), (7, 40)])
@pytest.mark.parametrize("N,bn,bm", [(130, 16, 16), (65, 64, 64), (300, 128, 128)])
def test_every_tile_once(place, counts, lead, tail, N, bn, bm):
    offsets = [lead]
    for c in counts:
        offsets.append(offsets[-1] + c)
    M = offsets[-1] + tail
    got = [t for t in place(M, N, bn, bm, offsets, range(_grid(M, N, bn, bm, len(counts)))) if t]
    want = [(e, n, m, offsets[e + 1]) for e in range(len(counts)) for m in range(offsets[e], offsets[e + 1], bm) for n in range(0, N, bn)]
    assert sorted(got) == sorted(want)


def _inside(M, N, offsets, tiles):
    for t in filter(None, tiles):
        e, n, m, end = t
        assert 0 <= e < len(offsets) - 1 and 0 <= n < N, t
        first = min(max(offsets[e], 0), M)
        assert end == min(max(offsets[e + 1], first), M) and first <= m < end, (t, first)


@pytest.mark.parametrize("M,N,bn,bm,E", [
    (INT32_MAX, 16, 16, 16, 40),  # 20 groups of 2^27 tiles: 2.7e9
    (INT32_MAX, 16, 16, 16, 64), (INT32_MAX - 1, 128, 128, 128, 300), (INT32_MAX, 200, 16, 16, 31), (1 << 30, 20, 16, 16, 130),
    (1 << 24, 16, 16, 16, 20000), (3000, 64, 16, 16, 200), (100, 40, 64, 64, 70)])
def test_offsets_that_go_up_and_down_stay_inside(place, M, N, bn, bm, E):
    offsets = [0, M] * (E // 2) + [0] * (E % 2 + 1)
    grid = _grid(M, N, bn, bm, E)
    assert grid <= INT32_MAX
    rng = random.Random(M + E)
    some = 24 if E > 1000 else 300
    blocks = sorted({*range(min(grid, 16)), *range(max(0, grid - 16), grid), *(rng.randrange(grid) for _ in range(some))})
    _inside(M, N, offsets, place(M, N, bn, bm, offsets, blocks))


@pytest.mark.parametrize("seed", range(40))
def test_any_offsets_stay_inside(place, seed):
    rng = random.Random(seed)
    E, M = rng.choice([1, 3, 64, 65, 200]), rng.choice([1, 50, 3000, 1 << 22, INT32_MAX])
    bm = bn = rng.choice([16, 64, 128])
    N = rng.choice([1, 16, 100])
    offsets = [rng.choice([0, M, rng.randint(0, M), rng.randint(-2 ** 31, INT32_MAX), -2 ** 31, INT32_MAX]) for _ in range(E + 1)]
    grid = _grid(M, N, bn, bm, E)
    if grid > INT32_MAX:
        pytest.skip("more workgroups than a launch holds")
    blocks = sorted({*range(min(grid, 8)), grid - 1, *(rng.randrange(grid) for _ in range(100))})
    _inside(M, N, offsets, place(M, N, bn, bm, offsets, blocks))
