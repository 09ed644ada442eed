"""The counts of tiles of the products of 8-bit matrices (csrc/bsp_f8_tiles.cuh), compiled by the host compiler with a trap on every signed
overflow: right up to the largest sizes that the calls take."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2407_09453_b200", "csrc")
HARNESS = r"""
#include <cstdio>
#include "bsp_f8_tiles.cuh"
int main()
{
    long long M, N;
    int pairs, BN, split;
    while (std::scanf("%lld %lld %d %d %d", &M, &N, &pairs, &BN, &split) == 5) {
        bsp::F8PairTiles t = {-1, -1, -1};
        const bool ok = bsp::f8_pair_tiles(M, N, pairs, t);
        int across = -1;
        int64_t ctas = -1;
        const bool fits = bsp::f8_tile_grid(M, N, BN, split, across, ctas);
        std::printf("%d %d %d %d %d %d %lld\n", ok, t.across, t.whole, t.all, fits, across, (long long)ctas);
    }
}
"""
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def count(tmp_path_factory):
    d = tmp_path_factory.mktemp("tiles")
    (d / "tiles.cpp").write_text(HARNESS)
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fsanitize=undefined", "-fsanitize-undefined-trap-on-error", "-I" + CSRC, str(d / "tiles.cpp"), "-o", str(d / "tiles")])

    def run(rows):
        out = subprocess.run([str(d / "tiles")], input="\n".join(" ".join(map(str, r)) for r in rows), capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return run


def expected(M, N, pairs, BN, split):
    across, tiles = -(-N // 256), -(-M // 256) * -(-N // 256)
    if tiles > MOST - 2 * pairs:
        pair = (0, -1, -1, -1)
    else:
        last = tiles % pairs
        whole = tiles - last if 2 * last <= pairs else tiles
        pair = (1, across, whole, tiles + tiles - whole)
    ctas = -(-M // 128) * -(-N // BN) * split
    return pair + (int(ctas <= MOST), -(-N // BN), ctas)


def test_counts(count):
    sizes = [1, 127, 128, 129, 255, 256, 257, 4096, 8192, 70000, 2 ** 20 + 1, 2 ** 30, MOST - 256, MOST - 255, MOST - 254, MOST - 128, MOST - 127, MOST - 1, MOST]
    rows = [(M, N, pairs, BN, split) for M in sizes for N in sizes for pairs, BN, split in ((74, 16, 1), (74, 32, 8), (66, 64, 4), (1, 128, 2))]
    assert count(rows) == [expected(*r) for r in rows]


def test_pairs_step_past_the_last_tile_within_an_int(count):
    """A pair's next tile is the last one plus the number of pairs, in an int."""
    for pairs in (1, 74, 1024):
        for M, N in ((MOST, 65536), (2 ** 31 - 256 * 300, 256 * 256), (MOST, MOST)):
            ok, _, _, tiles = count([(M, N, pairs, 128, 1)])[0][:4]
            assert not ok or tiles + pairs <= MOST
