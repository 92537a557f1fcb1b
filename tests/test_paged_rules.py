"""Attention over pages on the CPU: which kernel and which way to cut the work the library's own rules choose, on both sides of their lines, and that the GPU cases of the dealing are what
they are there for."""
import pytest

from tests.cache_helpers import dealing, route
from tests.test_gpu_paged_dealing import CASES, route_of


@pytest.mark.parametrize("mxfp8", [False, True], ids=["plain", "mxfp8"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}x{len(c[3])}x{c[3][0][0]}x{c[3][0][1]}")
def test_gpu_cases_are_dealt_as_they_say(case, mxfp8):
    assert route_of(case, mxfp8) == case[4]


def test_every_way_of_dealing_has_a_gpu_case():
    ways = {c[4].split(" + ")[-1].split()[-1] if "+" in c[4] else c[4] for c in CASES}
    assert ways >= {"nothing", "cut", "whole", "host"} and {"cut", "whole", "host"} <= {c[4] for c in CASES}
    assert {c[4].split(" ")[0] for c in CASES if "+" in c[4]} >= {"1", "2", "3", "4"}


@pytest.mark.parametrize("mxfp8,heads,seqs,max_q,max_kv,chunk", [
    # more than 16 rows a KV head over plain pages, more than 32 over 8-bit ones
    (0, (32, 8), 2, 4, 9000, 0), (0, (32, 8), 2, 5, 9000, 1), (1, (32, 8), 2, 8, 9000, 0), (1, (32, 8), 2, 9, 9000, 1), (0, (8, 8), 64, 16, 500, 0), (0, (8, 8), 64, 17, 500, 1),
    # 17 to 32 rows: not for up to 8 KV heads in all and 24576 keys, nor where a token alone has more than 16
    (0, (32, 8), 1, 8, 24576, 0), (0, (32, 8), 1, 8, 24577, 1), (0, (32, 8), 1, 9, 24576, 1), (0, (28, 4), 2, 4, 3000, 0), (0, (28, 4), 3, 4, 3000, 1), (0, (16, 1), 1, 2, 3000, 0),
    (0, (32, 1), 1, 1, 3000, 1), (1, (32, 1), 1, 1, 3000, 0), (1, (33, 1), 1, 1, 3000, 1),
])
def test_the_kernel_goes_by_rows(mxfp8, heads, seqs, max_q, max_kv, chunk):
    assert route("bf16", mxfp8, *heads, seqs, max_q, max_kv).chunk == chunk
    assert route("fp32", mxfp8, *heads, seqs, max_q, max_kv).chunk == 0


@pytest.mark.parametrize("dtype,mxfp8,heads,seqs,max_q,line", [
    ("bf16", 0, (32, 8), 7, 1, 512), ("bf16", 0, (32, 8), 8, 1, 768), ("bf16", 1, (32, 8), 7, 1, 512), ("bf16", 1, (32, 8), 8, 1, 1024), ("fp32", 0, (4, 2), 40, 1, 128), ("fp32", 1, (4, 2), 40, 9, 128),
    # tiles of 256 rows: fewer than 16 units, fewer than 64, more
    ("bf16", 0, (32, 8), 1, 64, 256), ("bf16", 0, (32, 8), 1, 65, 512), ("bf16", 0, (32, 8), 2, 64, 512), ("bf16", 0, (32, 8), 7, 64, 512), ("bf16", 0, (32, 8), 8, 64, 768), ("bf16", 1, (32, 4), 4, 500, 768),
])
def test_short_sequences_are_not_cut(dtype, mxfp8, heads, seqs, max_q, line):
    assert route(dtype, mxfp8, *heads, seqs, max_q, line).whole == 1 and route(dtype, mxfp8, *heads, seqs, max_q, line + 1).whole == 0


@pytest.mark.parametrize("dtype,mxfp8,heads,seqs,max_q,max_kv,rows,workgroups", [
    ("bf16", 0, (32, 8), 1, 1, 9000, 16, 512), ("bf16", 1, (32, 8), 1, 4, 9000, 16, 512), ("bf16", 1, (32, 8), 1, 5, 9000, 32, 512), ("bf16", 1, (17, 1), 1, 1, 9000, 32, 512),
    # fp32: 32 rows over plain pages where there are more than 256 steps (of 64 keys, tiles of 32 rows)
    ("fp32", 0, (4, 2), 1, 9, 8192, 32, 256), ("fp32", 0, (4, 2), 1, 9, 8191, 16, 512), ("fp32", 0, (4, 2), 8, 8, 9000, 16, 512), ("fp32", 1, (4, 2), 8, 9, 9000, 16, 512), ("fp32", 0, (33, 1), 1, 1, 70, 64, 256),
])
def test_rows_of_a_tile(dtype, mxfp8, heads, seqs, max_q, max_kv, rows, workgroups):
    r = route(dtype, mxfp8, *heads, seqs, max_q, max_kv)
    assert not r.chunk and r.rows == rows and r.workgroups == workgroups and (heads[0] // heads[1]) << r.tile_shift <= rows < (heads[0] // heads[1]) << (r.tile_shift + 1)


def test_dealing_names_the_other_kernel():
    assert dealing("bf16", False, 32, 8, [(1, 900)], 960) == "rows" and dealing("bf16", False, 32, 8, [(300, 600)] * 4, 640) == "host"
