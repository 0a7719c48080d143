"""How the experts' products are cut into tiles (csrc/moe_tiles.h, built by g++), over the sizes that nmm_moe_experts takes."""
import ctypes
import os
import random
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIM = 1 << 31
i64 = ctypes.c_int64


@pytest.fixture(scope="module")
def tiles(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    so = str(tmp_path_factory.mktemp("tiles") / "tiles.so")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I" + os.path.join(ROOT, "paper_2609_16009_amd", "csrc"),
                        os.path.join(ROOT, "tests", "sanitize", "moe_tiles_shim.cpp"), "-o", so], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    lib = ctypes.CDLL(so)
    lib.tile_rows.argtypes = [i64] * 6
    lib.tile_rows_near.argtypes = [i64] * 7
    ints, i32 = np.ctypeslib.ndpointer(np.int32, flags="C"), ctypes.c_int
    lib.walk.argtypes, lib.walk.restype = [ints, i32, i32, i32, i32, i32, ints], i64
    lib.walk_dense.argtypes = [i32] * 5 + [ints]
    lib.bytes_of_tile.argtypes, lib.bytes_of_tile.restype = [i64] * 3, i64
    return lib


def accepted(hidden, inner):
    """An expert's matrices below 2^31 bytes, with the least leading dimensions."""
    up8 = lambda n: (n + 7) // 8 * 8
    return 4 * inner * up8(hidden) < LIM and 2 * hidden * up8(inner) < LIM


@pytest.mark.parametrize("hidden,inner", [(8, 1 << 23), (8, (1 << 22) + 5), (8, (1 << 26) - 1), (1, (1 << 26) - 1), (8, (1 << 26) - 9),
                                          (56, 9 << 20), (16, (1 << 25) - 1), (7168, 2048), (1037, 331), (8, 1 << 21)])
@pytest.mark.parametrize("T", [1, 4, 5, 8, 9, 16, 17, 41, 97, 300, 5000])
def test_rows_of_h_that_a_tile_addresses(tiles, hidden, inner, T):
    """The second product's tile ends below 2^31 bytes from its first row, in whatever part of h it lies."""
    assert accepted(hidden, inner)
    ld = (inner + 63) // 64 * 64
    for k, experts, local in ((1, 1, 1), (2, 64, 64), (8, 1024, 3)):
        sizes = (inner, hidden, T, T * k, experts, local)
        want, rows = tiles.tile_rows(*sizes), tiles.tile_rows_near(*sizes, ld)
        assert rows in (4, 8, 16, 64, 128, 256)
        reach = lambda n: ((min(n, T * k) - 1) * ld + (inner + 7) // 8 * 8) * 2
        assert reach(rows) == tiles.bytes_of_tile(min(rows, T * k), ld, inner) < LIM
        # the rule's choice wherever that is in reach, else the largest tile that is
        if reach(want) < LIM:
            assert rows == want
        else:
            assert rows == max(n for n in (4, 8, 16, 64, 128, 256) if n < want and reach(n) < LIM)


def test_any_accepted_size(tiles):
    rng = random.Random(3)
    seen = 0
    while seen < 20000:
        hidden, inner = int(2 ** rng.uniform(0, 28)), int(2 ** rng.uniform(0, 26))
        if not accepted(hidden, inner):
            continue
        seen += 1
        T, k, experts = int(2 ** rng.uniform(0, 20)), rng.randint(1, 32), rng.randint(1, 1024)
        ld = (inner + 63) // 64 * 64
        rows = tiles.tile_rows_near(inner, hidden, T, T * k, experts, rng.randint(1, experts), ld)
        assert rows in (4, 8, 16, 64, 128, 256) and ((min(rows, T * k) - 1) * ld + (inner + 7) // 8 * 8) * 2 < LIM


@pytest.mark.parametrize("tile", [4, 8, 16, 64, 128, 256])
@pytest.mark.parametrize("n_blocks,grid", [(1, 8), (7, 16), (8, 2048), (57, 64)])
def test_every_pair_and_block_of_a_choice_once(tiles, tile, n_blocks, grid):
    rng = np.random.default_rng(tile + n_blocks)
    for local in (1, 2, 65, 130):
        for counts in (np.zeros(local), rng.integers(0, 3 * tile, local) * (rng.random(local) < 0.6), np.eye(1, local, local // 2)[0] * 5 * tile):
            first = int(rng.integers(0, 9))               # pairs of experts elsewhere, before and behind
            offsets = (first + np.concatenate(([0], np.cumsum(counts)))).astype(np.int32)
            pairs = int(offsets[-1]) + int(rng.integers(0, 9))
            seen = np.zeros((max(pairs, 1), n_blocks), np.int32)
            walked = tiles.walk(offsets, local, pairs, tile, n_blocks, grid, seen)
            assert walked == sum(-(-int(c) // tile) for c in counts)
            want = np.zeros_like(seen)
            want[first:offsets[-1]] = 1
            assert np.array_equal(seen, want)


@pytest.mark.parametrize("tile", [4, 16, 256])
def test_offsets_of_no_choice(tiles, tile):
    """Whatever they hold: no row outside the pairs, no more tiles than a choice can fill."""
    rng = np.random.default_rng(tile)
    for n in range(300):
        local, pairs = int(rng.integers(1, 140)), int(rng.integers(1, 700))
        offsets = [lambda: rng.integers(-(1 << 31), 1 << 31, local + 1), lambda: rng.integers(-9, pairs + 9, local + 1),
                   lambda: np.arange(local + 1) % 2 * pairs, lambda: np.full(local + 1, (1 << 31) - 1),
                   lambda: np.arange(local + 1) % 2 * ((1 << 32) - 1) - (1 << 31)][n % 5]().astype(np.int32)
        seen = np.zeros((pairs, 3), np.int32)
        walked = tiles.walk(offsets, local, pairs, tile, 3, 16, seen)
        assert 0 <= walked <= pairs // tile + local, n


@pytest.mark.parametrize("ks", [1, 2, 4, 8])
@pytest.mark.parametrize("rows,tile", [(1, 4), (33, 32), (256, 128), (1000, 64)])
def test_every_row_block_and_slice_once(tiles, rows, tile, ks):
    for n_blocks, grid in ((1, 8), (7, 8), (8, 64), (33, 16)):
        seen = np.zeros((rows, n_blocks, ks), np.int32)
        assert tiles.walk_dense(rows, tile, n_blocks, ks, grid, seen) == 0
        assert (seen == 1).all()
