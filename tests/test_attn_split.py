"""How attention over a paged cache shares ragged sequences out to its workgroups
(csrc/kq_split.h), on the CPU: every tile of every sequence in one run, runs of equal
length, results of pieces in places of their own, and for any lengths no run, place or
page outside the arrays."""
import os
import random
import shutil
import subprocess

import pytest

from conftest import ROOT

TILE, LEAST, PIECE, MOST = 32, 4, 12, 2 ** 31 - 64


@pytest.fixture(scope="module")
def binary(tmp_path_factory):
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    if not shutil.which("g++") or not os.path.isdir(os.path.join(rocm, "include", "hip")):
        pytest.skip("no g++ or no HIP headers")
    out = str(tmp_path_factory.mktemp("split") / "split_wave")
    built = subprocess.run(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__=1", "-fwrapv",
                            "-I", os.path.join(rocm, "include"), "-I", os.path.join(ROOT, "paper_2607_21446_amd", "csrc"),
                            os.path.join(ROOT, "tests", "native", "split_wave.cpp"), "-o", out], capture_output=True, text=True)
    assert built.returncode == 0, built.stderr
    return out


def _split(binary, lengths, max_tokens, window, runs):
    """Per run (b, skip, tiles, each)."""
    words = [len(lengths), max_tokens, window, runs, *lengths, runs, *range(runs)]
    done = subprocess.run([binary], input=" ".join(map(str, words)), capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, (done.returncode, done.stderr)
    return [tuple(map(int, line.split())) for line in done.stdout.splitlines()]


def _tiles(n, max_tokens, window):
    end = min(max(n, 0), max_tokens)
    first = end - window if 0 < window < end else 0
    return (end - 1) // TILE + 1 - first // TILE if end else 1


def _check(lengths, max_tokens, window, runs, got):
    # PIECE tiles before a sequence's own stand for what a piece costs beside them
    all_ = [_tiles(n, max_tokens, window) + PIECE for n in lengths]
    total = sum(all_)
    each = got[0][3]
    # total / runs or, where rounding takes an even quotient up, one more
    assert each == max(LEAST, -(-total // runs)) or (total % runs == 0 and each == max(LEAST, total // runs + 1))
    assert len(got) == runs and all(r[3] == each for r in got)
    begin = [0]
    for t in all_:
        begin.append(begin[-1] + t)
    places, seen = [], [0] * len(lengths)
    for x, (b, skip, tiles, _) in enumerate(got):
        assert tiles == max(0, min(each, total - x * each)), (x, tiles)
        if not tiles:
            continue
        assert 0 <= b < len(lengths) and 0 <= skip < all_[b] and begin[b] + skip == x * each, (x, b, skip)
        while tiles:  # its pieces, as the kernel walks through them
            n = min(all_[b] - skip, tiles)
            done, own = max(skip - PIECE, 0), all_[b] - PIECE
            mine = skip + n - PIECE - done  # tiles of its own in this piece
            if mine > 0:
                seen[b] += mine
                if mine < own:
                    places.append(2 * x + (done == 0))
                if done == 0 and mine < own:  # where the join looks for the sequence's pieces
                    count = 2 + (own - mine - 1) // each
                    assert (begin[b + 1] - 1) // each - x + 1 == count
            tiles, b, skip = tiles - n, b + 1, 0
    assert seen == [t - PIECE for t in all_]
    assert len(set(places)) == len(places) and max(places, default=0) < 2 * runs


@pytest.mark.parametrize("lengths", [
    [0], [1], [31], [32], [33], [128], [129], [131072], [0, 0, 0], [1000, 0, 5, 128, 129, 40000], [7] * 64, [7] * 65, [0] * 64 + [100000],
    [300] * 70 + [0] * 3 + [9000], [2 ** 31 - 1, 5], [-1, 64, -2 ** 31]])
@pytest.mark.parametrize("runs", [1, 7, 40])
@pytest.mark.parametrize("window", [0, 33, 5000])
def test_every_tile_once(binary, lengths, runs, window):
    for max_tokens in (1 << 17, 96) if runs < 40 else (MOST,):
        _check(lengths, max_tokens, window, runs, _split(binary, lengths, max_tokens, window, runs))


@pytest.mark.parametrize("seed", range(20))
def test_any_lengths_stay_inside(binary, seed):
    rng = random.Random(seed)
    B, max_tokens = rng.choice([1, 2, 63, 64, 65, 130]), rng.choice([0, 16, 4096, 1 << 20, MOST])
    runs, window = rng.choice([1, 3, 64, 200]), rng.choice([0, 0, 1, 100, 2 ** 40])
    lengths = [rng.choice([0, 1, max_tokens % 2 ** 31, rng.randint(0, max_tokens), rng.randint(-2 ** 31, 2 ** 31 - 1)]) for _ in range(B)]
    _check(lengths, max_tokens, window, runs, _split(binary, lengths, max_tokens, window, runs))


@pytest.mark.parametrize("token,end,shift,entry,want", [
    (0, 1, 4, 0, (0, 0)), (31, 32, 4, 9, (1, 9)), (48, 33, 4, 10, (2, 9)), (2 ** 31 - 64, MOST, 15, -1, (65535, 0)),
    (16, 1, 4, 2 ** 31 - 1, (0, 9)), (64, 65, 6, -2 ** 31, (1, 0))])
def test_pages_stay_inside(binary, token, end, shift, entry, want):
    done = subprocess.run([binary, *map(str, (token, end, shift, entry))], capture_output=True, text=True, timeout=60)
    assert done.returncode == 0 and tuple(map(int, done.stdout.split())) == want


@pytest.mark.parametrize("B", [63, 64, 65, 128, 200])
@pytest.mark.parametrize("runs", [1, 8, 160])
def test_many_of_the_longest(binary, B, runs):
    """Sequences at the limit whose tiles, and what their pieces cost, are 2^32 and more together."""
    for longest, window in ((2 ** 31 - 1, 0), (MOST, 0), (MOST, MOST - 5)):
        lengths = [longest] * B
        _check(lengths, MOST, window, runs, _split(binary, lengths, MOST, window, runs))
    lengths = [MOST] * (B - 1) + [0]
    _check(lengths, MOST, 0, runs, _split(binary, lengths, MOST, 0, runs))
