"""Grids of the calls that train rows, as host arithmetic compiled by itself: every item in one block, no launch of 2^32 threads."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "%s/paper_2310_20419_amd/csrc/grid.h"
extern "C" uint64_t blocks_most(uint32_t threads) { return most_blocks(threads); }
extern "C" uint64_t items(uint64_t n, uint64_t wanted, uint64_t room) { return items_per_block(n, wanted, room); }
extern "C" int launches(uint64_t total, uint32_t threads, uint64_t *first, uint64_t *blocks)
{
    int n = 0;
    in_launches(total, threads, [&](uint64_t f, uint64_t b) { first[n] = f; blocks[n++] = b; });
    return n;
}
// rows of (launch, list, first, n, tile), and a row of (launch, -1, 0, 0, tiles) behind each launch
extern "C" int cut(int32_t count, const uint64_t *lengths, uint64_t tile, uint64_t room, uint32_t parts, int64_t *out)
{
    int n = 0, launch = 0;
    auto row = [&](int64_t a, int64_t b, int64_t c, int64_t d, int64_t e) {
        const int64_t v[5] = {a, b, c, d, e};
        for (int i = 0; i < 5; ++i) out[5 * n + i] = v[i];
        ++n;
    };
    cut_into_launches(count, tile, room, parts, [&](int32_t i) { return lengths[i]; },
                      [&](int32_t i, uint64_t first, uint64_t k, uint64_t at) { row(launch, i, first, k, at); },
                      [&](uint64_t tiles) { row(launch++, -1, 0, 0, tiles); });
    return n;
}
""" % ROOT


@pytest.fixture(scope="module")
def grid(tmp_path_factory):
    import ctypes
    at = tmp_path_factory.mktemp("grid")
    (at / "grid.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-o", str(at / "grid.so"), str(at / "grid.cpp")], check=True)
    lib = ctypes.CDLL(str(at / "grid.so"))
    u64 = ctypes.c_uint64
    lib.blocks_most.argtypes, lib.blocks_most.restype = [ctypes.c_uint32], u64
    lib.items.argtypes, lib.items.restype = [u64] * 3, u64
    lib.launches.argtypes = [u64, ctypes.c_uint32, ctypes.POINTER(u64), ctypes.POINTER(u64)]
    lib.cut.argtypes = [ctypes.c_int32, ctypes.POINTER(u64), u64, u64, ctypes.c_uint32, ctypes.POINTER(ctypes.c_int64)]
    return lib


@pytest.mark.parametrize("threads", [64, 256, 512, 1024])
def test_a_launch_holds_fewer_than_four_billion_threads(grid, threads):
    most = grid.blocks_most(threads)
    assert most * threads < 2**32 <= (most + 1) * threads


@pytest.mark.parametrize("items,wanted", [(1, 1), (186_000_000, 11), (2**31 - 2, 1), (2**31 - 2, 1024), (16_777_215, 1), (16_777_216, 1)])
def test_items_of_a_block(grid, items, wanted):
    most = grid.blocks_most(256)
    per = grid.items(items, wanted, most)
    assert per >= wanted and -(-items // per) <= most
    assert per == wanted or -(-items // (per - 1)) > most       # no more than it takes


@pytest.mark.parametrize("total", [0, 1, 8, 2**24 - 16, 2**24 - 8, 2**24 - 1, 2**24, 2**24 + 9, 2**26, 3 * 2**24 + 5])
def test_a_grid_in_several_launches(grid, total):
    import ctypes
    first, blocks = (ctypes.c_uint64 * 64)(), (ctypes.c_uint64 * 64)()
    n = grid.launches(total, 256, first, blocks)
    at = 0
    for i in range(n):
        assert first[i] == at and at % 8 == 0 and 0 < blocks[i] and blocks[i] * 256 < 2**32
        at += blocks[i]
    assert at == total


@pytest.mark.parametrize("lengths,tile,room,parts", [
    ([5, 0, 7, 1], 4, 100, 50), ([0, 0], 4, 10, 5), ([], 4, 10, 5), ([40], 4, 3, 5), ([41, 1, 2], 4, 3, 2), ([12, 12, 0, 5], 4, 3, 9),
    ([1] * 120, 2048, 2**24 - 1, 50), ([2**40, 5], 2048, 2**24 - 1, 71), ([8, 9, 100, 3, 0, 64], 8, 5, 3), ([0, 30, 0], 4, 2, 1)])
def test_tensors_cut_into_launches(grid, lengths, tile, room, parts):
    import ctypes
    out = (ctypes.c_int64 * 50_000)()
    n = grid.cut(len(lengths), (ctypes.c_uint64 * max(1, len(lengths)))(*lengths), tile, room, parts, out)
    rows = [tuple(out[5 * i:5 * i + 5]) for i in range(n)]
    done, launch, tiles, held = [0] * len(lengths), 0, 0, 0
    for number, i, first, k, at in rows:
        assert number == launch
        if i < 0:
            assert at == tiles and 0 < tiles <= room and held <= parts
            launch, tiles, held = launch + 1, 0, 0
            continue
        assert at == tiles and first == done[i] and first % tile == 0 and 0 < k and all(done[j] == lengths[j] for j in range(i))
        done[i] += k
        tiles += -(-k // tile)
        held += 1
    assert done == lengths and tiles == 0
