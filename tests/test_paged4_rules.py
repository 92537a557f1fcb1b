"""Attention over pages of 4 bits on the CPU: which kernel and which way to cut the work the library's own rules choose, on both sides of their lines, and that the lines of the other formats
are where they were."""
import ctypes

import pytest

from paper_2409_12490_amd import binding as B
from tests import test_cache_abi as A
from tests.cache_helpers import Shape, dealing, route

FOUR = 2                                           # HELD_MXFP4 of csrc/cache.h


@pytest.mark.parametrize("heads,seqs,max_q,max_kv,chunk", [
    # up to 64 rows a KV head tiles of 32 rows, then of 256
    ((32, 8), 2, 16, 9000, 0), ((32, 8), 2, 17, 9000, 1), ((8, 8), 64, 64, 500, 0), ((8, 8), 64, 65, 500, 1), ((32, 1), 9, 2, 9000, 0), ((32, 1), 9, 3, 9000, 1),
    # of up to 8 KV heads in all up to 128, and 256 where there are 4096 keys at most
    ((32, 8), 1, 32, 9000, 0), ((32, 8), 1, 33, 9000, 1), ((32, 8), 1, 64, 4096, 0), ((32, 8), 1, 64, 4097, 1), ((32, 8), 1, 65, 4096, 1), ((4, 1), 8, 64, 4096, 0), ((4, 1), 9, 64, 4096, 1),
    # more query heads than a tile has rows
    ((32, 1), 3, 1, 9000, 0), ((33, 1), 3, 1, 9000, 1), ((64, 1), 1, 1, 100, 1),
])
def test_the_kernel_goes_by_rows(heads, seqs, max_q, max_kv, chunk):
    assert route("bf16", FOUR, *heads, seqs, max_q, max_kv).chunk == chunk
    assert route("fp32", FOUR, *heads, seqs, max_q, max_kv).chunk == 0


@pytest.mark.parametrize("dtype,heads,seqs,max_q,line", [
    # by units: fewer than 64, than 128, than 256, and more; tiles of 32 rows are units too
    ("bf16", (32, 8), 7, 1, 768), ("bf16", (32, 8), 8, 1, 1024), ("bf16", (32, 8), 15, 1, 1024), ("bf16", (32, 8), 16, 1, 1536), ("bf16", (32, 8), 31, 1, 1536), ("bf16", (32, 8), 32, 1, 2048),
    ("bf16", (32, 8), 8, 16, 1536), ("bf16", (32, 8), 7, 9, 1024), ("bf16", (32, 8), 3, 16, 768),
    ("fp32", (8, 2), 31, 1, 512), ("fp32", (8, 2), 32, 1, 1024), ("fp32", (8, 2), 127, 1, 1024), ("fp32", (8, 2), 128, 1, 2048), ("fp32", (4, 2), 8, 200, 2048), ("fp32", (4, 2), 1, 200, 512),
    # tiles of 256 rows, as over 8-bit pages
    ("bf16", (32, 8), 1, 65, 512), ("bf16", (32, 8), 2, 64, 512), ("bf16", (32, 8), 8, 64, 768),
])
def test_short_sequences_are_not_cut(dtype, heads, seqs, max_q, line):
    assert route(dtype, FOUR, *heads, seqs, max_q, line).whole == 1 and route(dtype, FOUR, *heads, seqs, max_q, line + 1).whole == 0


@pytest.mark.parametrize("dtype,heads,seqs,max_q,rows,workgroups", [
    ("bf16", (32, 8), 1, 4, 16, 512), ("bf16", (32, 8), 1, 5, 32, 512), ("bf16", (32, 8), 2, 16, 32, 512), ("bf16", (17, 1), 1, 1, 32, 512), ("bf16", (28, 4), 9, 2, 16, 512), ("bf16", (28, 4), 9, 3, 32, 512),
    ("fp32", (4, 2), 20, 200, 16, 512), ("fp32", (17, 1), 1, 1, 32, 256), ("fp32", (33, 1), 1, 1, 64, 256), ("fp32", (64, 1), 5, 9, 64, 256),
])
def test_rows_of_a_tile(dtype, heads, seqs, max_q, rows, workgroups):
    r = route(dtype, FOUR, *heads, seqs, max_q, 9000)
    assert not r.chunk and r.rows == rows and r.workgroups == workgroups and (heads[0] // heads[1]) << r.tile_shift <= rows < (heads[0] // heads[1]) << (r.tile_shift + 1)
    assert r.step_shift == 7                        # 32 keys to each wave, whatever the type


def test_every_way_of_dealing_256_row_tiles_is_reached_by_the_gpu_cases():
    from tests.test_gpu_paged4 import TILES, tiles_route
    ways = {tiles_route(c) for c in TILES}
    assert {w.split(" + ")[-1].split()[-1] for w in ways if "+" in w} == {"nothing", "cut", "whole"} and {"whole", "host", "cut"} <= ways and "rows" not in ways


def test_the_gpu_cases_around_the_lines_are_on_both_sides():
    from tests.test_gpu_paged4 import AROUND, around_route
    routes = [around_route(c) for c in AROUND]
    assert {(r.chunk, r.rows) for r in routes} == {(0, 16), (0, 32), (0, 64), (1, 256)} and {(r.chunk, r.whole) for r in routes} == {(0, 0), (0, 1), (1, 0), (1, 1)}


def _few(held, heads, seqs, max_q, max_kv, tokens, dtype=1):
    f = B.load()._ZN2cp10few_tokensERKNS_10CacheShapeE
    f.argtypes, f.restype = [ctypes.POINTER(Shape)], ctypes.c_int
    return f(Shape(dtype=dtype, mxfp8=held, hq=heads[0], hkv=heads[1], group=heads[0] // heads[1], n_seqs=seqs, max_q=max_q, max_kv=max_kv, tokens=tokens))


@pytest.mark.parametrize("heads,seqs,max_q,max_kv,tokens,few", [
    ((32, 8), 64, 512, 8192, 575, 4), ((32, 4), 64, 512, 8192, 575, 2), ((32, 1), 64, 512, 4096, 575, 0), ((32, 1), 64, 512, 8192, 575, 1), ((33, 1), 64, 512, 8192 * 2, 575, 0),
    # the others 12 tokens on the average, and more; 6000 steps of 64 keys for all but one, and fewer
    ((32, 8), 11, 100, 8192, 220, 4), ((32, 8), 11, 100, 8192, 221, 0), ((32, 8), 11, 100, 4800, 200, 4), ((32, 8), 11, 100, 4736, 200, 0),
    # one sequence; no tiles of 256 rows; nothing known of the longest
    ((32, 8), 1, 512, 80000, 512, 0), ((32, 8), 64, 16, 8192, 64, 0), ((32, 8), 64, 64, 8192, 64, 4),
])
def test_single_tokens_beside_a_chunk(heads, seqs, max_q, max_kv, tokens, few):
    assert _few(FOUR, heads, seqs, max_q, max_kv, tokens) == few
    assert _few(0, heads, seqs, max_q, max_kv, tokens) == _few(1, heads, seqs, max_q, max_kv, tokens) == _few(FOUR, heads, seqs, max_q, max_kv, tokens, dtype=0) == 0


def test_the_gpu_cases_of_single_tokens_beside_a_chunk_go_to_both():
    from tests.test_gpu_paged4 import MIXED, few_of
    assert [few_of(c) for c in MIXED] == [c[4] for c in MIXED]


@pytest.mark.parametrize("dtype", [B.CP_DTYPE_FP32, B.CP_DTYPE_BF16])
@pytest.mark.parametrize("heads", [2, 8, 34, 66, 128])
def test_the_workspace_is_enough_for_any_number_of_sequences_and_keys(dtype, heads):
    """Parts of (rows, 128 + 2) fp32 for each workgroup's two units, and the records, of the route that a call takes."""
    for longest in (1, 5, 16, 17, 32, 33, 64, 65, 300):
        need = B.critiprefill_paged_workspace_bytes(A._params(cache_format=B.CP_CACHE_MXFP4, dtype=dtype, n_q_heads=heads, max_q_len=longest))
        for seqs in (1, 3, 5, 40):
            for keys in (100, 4096, 4097, 100000):
                r = route("bf16" if dtype else "fp32", FOUR, heads, 2, seqs, longest, keys)
                assert need >= r.workgroups * 2 * r.rows * 130 * 4 + (4 + 4 * r.workgroups) * 4
