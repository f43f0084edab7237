"""How the linear layer's products are cut into tiles (host code, compiled here): every product has its whole sum covered, and the
sizes that the GPU tests run reach the tile shapes that they are there for."""
import os
import random
import shutil
import subprocess

import pytest

import linear_tiles

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("cut") / "check")
    subprocess.run([gxx, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-o", exe, os.path.join(HERE, "host", "linear_cut_check.cpp")],
                   check=True, timeout=300)

    def run(cases):
        text = "\n".join(" ".join(str(int(v)) for v in c) for c in cases)
        out = subprocess.run([exe], input=text, check=True, capture_output=True, text=True, timeout=300).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return run


def test_sizes_reach_their_tiles(cut):
    for itemsize in (2, 4):
        for rows, cols, k, tile, split in linear_tiles.sizes(itemsize):
            for inner in (0, 1):
                got, parts, _ = cut([(rows, cols, k, itemsize, inner)])[0]
                assert (got, parts > 1) == (tile, split), (rows, cols, k, itemsize, got, parts)
            assert k % (128 // itemsize) or k >= 4 * (128 // itemsize)
    for (m, n, k), tile in linear_tiles.PAIRS:
        (dx, a, _), (dw, b, _) = cut([(m, k, n, 2, 0), (n, k, m, 2, 0)])
        assert dx <= 64 and dw <= 64 and a == b == 1
        tiles = -(-m // 64) * -(-k // 64) + -(-n // 64) * -(-k // 64)
        assert (64 if tiles >= 256 else 32) == tile


def test_parts_cover_the_sum(cut):
    rng = random.Random(1)
    size = lambda: int(2 ** rng.uniform(0, 14)) if rng.random() < 0.9 else 0          # noqa: E731
    cases = [(size(), size(), size(), rng.choice([2, 4]), rng.choice([0, 1])) for _ in range(4000)]
    cases += [(1, 1, 1 << 33, 2, 0), (1 << 31, 1, 64, 2, 1), (0, 1, 1 << 40, 2, 0), (1, 0, 1 << 40, 4, 1)]
    for (rows, cols, k, itemsize, inner), (tile, parts, each) in zip(cases, cut(cases)):
        assert tile in (0, 32, 64, 128, 256) and (tile or (inner and rows <= 16)) and (tile != 256 or itemsize == 2)
        assert 1 <= parts <= 16 and parts * each >= k and ((parts - 1) * each < k or parts == 1)
        assert parts == 1 or each % (128 // itemsize) == 0


def test_single_tokens_read_w_once_however_long_it_is(cut):
    """One to four rows at any number of columns, up to 16 in fp32 or of a shorter W: no tile."""
    for size in (2, 4):
        for cols in (1, 8192, 8193, 151936, 1 << 25):
            got = [t for t, _, _ in cut([(m, cols, 4096, size, 1) for m in range(1, 18)])]
            few = 16 if size == 4 or cols <= 8192 else 4
            assert got[:few] == [0] * few and all(got[few:])
        assert cut([(1, (1 << 25) + 1, 64, size, 1)])[0][0]          # beyond a launch of fewer than 2^32 threads
        assert all(t for t, _, _ in cut([(m, 100, 4096, size, 0) for m in range(1, 17)]))
