"""How attention over a paged cache cuts ragged sequences into parts (csrc/kq_split.h),
on the CPU: every tile of every sequence once, results of parts in places of their
own, and for any lengths no part, place or page outside the arrays."""
import os
import random
import shutil
import subprocess

import pytest

from conftest import ROOT

TILE, LEAST, MOST = 32, 4, 2 ** 31 - 64


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


def _split(binary, lengths, max_tokens, window, parts, blocks):
    """Per block None or (b, index, count, slot, first, end, tile, tiles)."""
    words = [len(lengths), max_tokens, window, parts, *lengths, len(blocks), *blocks]
    done = subprocess.run([binary], input=" ".join(map(str, words)), capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, (done.returncode, done.stderr)
    return [None if line == "-" else tuple(map(int, line.split())) for line in done.stdout.splitlines()]


def _span(n, max_tokens, window):
    end = min(max(n, 0), max_tokens)
    first = end - window if 0 < window < end else 0
    return first, end, (end - 1) // TILE + 1 - first // TILE if end else 0


def _check(lengths, max_tokens, window, parts, got):
    """got: of every block of the grid, in order."""
    spans = [_span(n, max_tokens, window) for n in lengths]
    # tiles of a part: total / parts or, where rounding takes an even quotient up, one more
    total = sum(t for _, _, t in spans)
    c, ways = max(LEAST, -(-total // parts)), [p[2] for p in filter(None, got)]
    if total % parts == 0 and len(ways) == sum(max(1, -(-t // (c + 1))) for _, _, t in spans) != sum(max(1, -(-t // c)) for _, _, t in spans):
        c += 1
    found, slots = {b: [] for b in range(len(lengths))}, []
    for p in filter(None, got):
        b, index, count, slot, first, end, tile, tiles = p
        assert (first, end) == spans[b][:2] and count == max(1, -(-spans[b][2] // c)), p
        found[b].append((index, tile, tiles))
        if count > 1:
            slots.append(slot + index)
    for b, (first, _, tiles) in enumerate(spans):
        count = max(1, -(-tiles // c))
        want = [(i, first // TILE + i * c, min(c, tiles - i * c)) for i in range(count)]
        assert sorted(found[b]) == want, (b, found[b], want)
    assert sorted(slots) == list(range(len(slots))) and len(slots) <= min(2 * parts, parts + len(lengths))


@pytest.mark.parametrize("lengths", [
    [0], [1], [31], [32], [33], [128], [129], [131072], [0, 0, 0], [1000, 0, 5, 128, 129, 40000], [7] * 64, [7] * 65, [0] * 64 + [100000],
    [300] * 70 + [0] * 3 + [9000], [2 ** 31 - 1, 5], [-1, 64, -2 ** 31]])
@pytest.mark.parametrize("parts", [1, 7, 40])
@pytest.mark.parametrize("window", [0, 33, 5000])
def test_every_tile_once(binary, lengths, parts, window):
    for max_tokens in (1 << 17, 96) if parts < 40 else (MOST,):
        blocks = range(parts + len(lengths))
        _check(lengths, max_tokens, window, parts, _split(binary, lengths, max_tokens, window, parts, blocks))


@pytest.mark.parametrize("seed", range(20))
def test_any_lengths_stay_inside(binary, seed):
    rng = random.Random(seed)
    B, max_tokens = rng.choice([1, 2, 63, 64, 65, 130]), rng.choice([0, 16, 4096, 1 << 20, MOST])
    parts, window = rng.choice([1, 3, 64, 200]), rng.choice([0, 0, 1, 100, 2 ** 40])
    lengths = [rng.choice([0, 1, max_tokens % 2 ** 31, rng.randint(0, max_tokens), rng.randint(-2 ** 31, 2 ** 31 - 1)]) for _ in range(B)]
    _check(lengths, max_tokens, window, parts, _split(binary, lengths, max_tokens, window, parts, range(parts + B)))


@pytest.mark.parametrize("token,end,shift,entry,want", [
    (0, 1, 4, 0, (0, 0)), (31, 32, 4, 9, (1, 9)), (48, 33, 4, 10, (2, 9)), (2 ** 31 - 64, MOST, 15, -1, (65535, 0)),
    (16, 1, 4, 2 ** 31 - 1, (0, 9)), (64, 65, 6, -2 ** 31, (1, 0))])
def test_pages_stay_inside(binary, token, end, shift, entry, want):
    done = subprocess.run([binary, *map(str, (token, end, shift, entry))], capture_output=True, text=True, timeout=60)
    assert done.returncode == 0 and tuple(map(int, done.stdout.split())) == want
