"""Which rows a workgroup of the products of rows in groups has: csrc/w4a16_group_place.h, compiled for the host, its threads one after the other."""
import os
import subprocess

import numpy as np
import pytest

from paper_2601_16536_amd import build

SOURCE = """
#define __host__
#define __device__
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "w4a16_group_place.h"
using namespace w4a16;
// arguments: threads, fill, E, count, tile_rows, cols, first block, last block, step, offsets; prints the number of row tiles, then block, group, row0, end, col
int main(int argc, char **argv)
{
    std::vector<long long> v;
    for (int i = 1; i < argc; ++i) v.push_back(atoll(argv[i]));
    const int threads = (int)v[0], fill = (int)v[1], E = (int)v[2];
    std::vector<int32_t> offsets(v.begin() + 9, v.end());
    if ((int)offsets.size() != E + 1) return 2;
    const GroupTiling g = {offsets.data(), E, fill ? E + 2 : E, (int)v[3], (int)v[4], (int)v[5]};
    std::vector<TileCount> ahead(threads + 1, 0);
    for (int t = 0; t < threads; ++t) ahead[t + 1] = ahead[t] + tiles_of_thread(g, t, threads);
    printf("%lld 0 0 0 0\\n", (long long)ahead[threads]);
    for (long long b = v[6]; b <= v[7]; b += v[8]) {
        TileCount pair;
        if (!pair_of_block(ahead[threads], g.cols, (unsigned)b, &pair)) continue;
        RowTile found;
        for (int t = 0; t < threads; ++t)
            if (tile_of_thread(g, t, threads, ahead[t], ahead[t + 1] - ahead[t], pair, &found)) printf("%lld %d %d %d %d\\n", b, found.group, found.row0, found.end, found.col);
    }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    folder = tmp_path_factory.mktemp("group_place")
    (folder / "place.cpp").write_text(SOURCE)
    path = str(folder / "place")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", build.CSRC, str(folder / "place.cpp"), "-o", path])

    def run(threads, fill, count, tile_rows, cols, offsets, blocks=None):
        E = len(offsets) - 1
        if blocks is None:
            groups = min(E + 2 if fill else E, count)
            blocks = (0, -(-((count + groups * (tile_rows - 1)) // tile_rows * cols) // 8) * 8 - 1, 1)
        args = [threads, int(fill), E, count, tile_rows, cols, *blocks, *offsets]
        out = subprocess.run([path] + [str(int(a)) for a in args], stdout=subprocess.PIPE, check=True, text=True).stdout
        rows = np.array([[int(x) for x in line.split()] for line in out.splitlines()])
        return int(rows[0, 0]), rows[1:]
    return run


@pytest.mark.parametrize("fill", [False, True])
@pytest.mark.parametrize("threads,E,count,tile_rows,cols", [(128, 1, 1, 16, 1), (256, 5, 100, 16, 3), (512, 64, 3000, 256, 5), (128, 1024, 900, 16, 2), (256, 700, 5000, 64, 1), (512, 1, 777, 128, 7)])
def test_every_row_of_every_column_tile_once(program, threads, E, count, tile_rows, cols, fill):
    rng = np.random.default_rng(E)
    offsets = np.sort(rng.integers(0, count + 1, E + 1))
    _, found = program(threads, fill, count, tile_rows, cols, offsets)
    times = np.zeros((cols, count), int)
    for block, group, row0, end, col in found:
        lo, hi = (offsets[group], offsets[group + 1]) if group < E else (offsets[E], count) if group == E else (0, offsets[0])
        assert lo <= row0 < end == hi
        times[col, row0:min(end, row0 + tile_rows)] += 1
    want = np.ones(count, int)
    if not fill:
        want[:offsets[0]] = want[offsets[-1]:] = 0
    assert (times == want).all() and len(set(found[:, 0])) == len(found)


@pytest.mark.parametrize("seed", range(4))
def test_offsets_that_descend_lead_nowhere_else(program, seed):
    rng = np.random.default_rng(seed)
    count = 2000
    _, found = program(256, bool(seed % 2), count, 64, 3, rng.integers(-5000, 5000, 41))
    assert (0 <= found[:, 2]).all() and (found[:, 2] < found[:, 3]).all() and (found[:, 3] <= count).all() and (0 <= found[:, 4]).all() and (found[:, 4] < 3).all()
    assert len(set(found[:, 0])) == len(found)


@pytest.mark.parametrize("tile_rows,step", [(128, 65537), (256, 32771)])
def test_more_tiles_than_32_bits_count(program, tile_rows, step):
    """2^30 - 1 rows for each of 512 groups."""
    count = (1 << 30) - 1
    offsets = [0, count] * 512 + [0]
    total, found = program(512, True, count, tile_rows, 2, offsets, (0, 1 << 24, step))
    assert total == 513 * (1 << 30) // tile_rows
    assert len(found) == len(range(0, (1 << 24) + 1, step)) == len(set(found[:, 0]))
    assert (0 <= found[:, 2]).all() and (found[:, 2] < found[:, 3]).all() and (found[:, 3] == count).all()
