"""How many steps a tile of new tokens takes over its keys (TileSteps), compiled for the CPU from the header the kernels include: enough for what its last token
sees, at most one more, never more than the keys fill, and the sums over tiles in closed form."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2409_12490_amd", "csrc")
PROGRAM = """
#define __host__
#define __device__
#define __forceinline__ inline
#include "paged_steps.h"
extern "C" void steps(int tokens, int keys, int tile_shift, int step_shift, int tiles, unsigned* of, unsigned* before) {
    const cp::TileSteps t(tokens, keys, step_shift);
    for (int i = 0; i <= tiles; ++i) {
        if (i < tiles) of[i] = t.of(i, tile_shift, step_shift);
        before[i] = t.before(i, tile_shift, step_shift);
    }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    compiler = shutil.which("g++") or shutil.which("clang++") or shutil.which("c++")
    if compiler is None:
        pytest.skip("no C++ compiler")
    where = tmp_path_factory.mktemp("paged_steps")
    (where / "f.cpp").write_text(PROGRAM)
    subprocess.run([compiler, "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(where / "f.cpp"), "-o", str(where / "f.so")], check=True)
    lib = ctypes.CDLL(str(where / "f.so"))
    array = np.ctypeslib.ndpointer(np.uint32)
    lib.steps.argtypes, lib.steps.restype = [ctypes.c_int] * 5 + [array, array], None
    return lib


def _steps(lib, tokens, keys, tile_shift, step_shift):
    tiles = (tokens + (1 << tile_shift) - 1) >> tile_shift
    of, before = np.zeros(max(tiles, 1), np.uint32), np.zeros(tiles + 1, np.uint32)
    lib.steps(tokens, keys, tile_shift, step_shift, tiles, of, before)
    return of[:tiles].astype(np.int64), before.astype(np.int64)


@pytest.mark.parametrize("tile_shift", range(9))
@pytest.mark.parametrize("step_shift", [6, 7])
def test_tiles_take_what_their_last_token_sees(lib, tile_shift, step_shift):
    tile, step = 1 << tile_shift, 1 << step_shift
    rng = np.random.default_rng(tile_shift)
    cases = [(0, 0), (0, 9), (1, 0), (1, 1), (300, 1), (700, 63), (700, 64), (700, 65), (257, 257), (5, 64), (1000, 999), (1000, 100000)]
    cases += [(int(rng.integers(0, 3000)), int(rng.integers(0, 4000))) for _ in range(200)]
    for tokens, keys in cases:
        of, before = _steps(lib, tokens, keys, tile_shift, step_shift)
        end = np.minimum((np.arange(len(of)) + 1) * tile, tokens)            # behind a tile's last token
        sees = np.maximum(keys - tokens + end, 0)
        need, most = np.maximum(-(-sees // step), 1), max(-(-keys // step), 1)
        assert (of >= need).all() and (of <= most).all(), (tokens, keys)
        if keys >= tokens:
            assert (of <= need + 1).all(), (tokens, keys)
        if tokens:
            assert of[-1] == most
        assert (before == np.concatenate([[0], np.cumsum(of)])).all(), (tokens, keys)


def test_more_new_tokens_than_keys_stay_within_32_bits(lib):
    """4 M new tokens that 100 keys are held for, 64 to a tile: 2 steps each, where tiles that count on as if the keys were there come to 2 * 10^9 for one head."""
    of, before = _steps(lib, 1 << 22, 100, 6, 6)
    assert of.max() == 2 and before[-1] == 2 * len(of) - 1
