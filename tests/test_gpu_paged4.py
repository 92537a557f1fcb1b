"""Attention of new tokens over pages of 4 bits against fp64: the cases of the other formats, what hidden places hold, arrays that say nonsense, captured calls."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2409_12490_amd import binding as B
from tests.cache4_helpers import Pool4, attend4
from tests.cache_helpers import DEV, HALF_STEP, Shape, check_attention, dealing, f64, randn, route
from tests.test_gpu_paged import CASES, DEALT, _starts
from tests.test_gpu_paged_dealing import _plain

pytestmark = pytest.mark.gpu


def _case(dtype, hq, hkv, page, seqs, seed=0, scale=1.0):
    """seqs: (new tokens, tokens in all)."""
    gen = torch.Generator().manual_seed(seed + 17 * len(seqs) + hq)
    new, total = zip(*seqs)
    pool = Pool4(gen, total, hkv, page, dtype, scale=scale)
    q = randn(gen, max(sum(new), 1), hq + 1, 128, dtype=dtype).to(DEV)[:sum(new), :hq]        # with a gap behind the heads
    return pool, q, _starts(new), list(total)


@pytest.mark.parametrize("case", CASES + DEALT, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}x{c[3]}x{len(c[4])}x{c[4][0][0]}x{c[4][0][1]}")
def test_against_fp64(case):
    dtype, hq, hkv, page, seqs = case
    pool, q, start, total = _case(dtype, hq, hkv, page, seqs)
    out, lse = attend4(pool, q, start, total, max_q_len=max(n for n, _ in seqs))
    check_attention(pool, q, start, total, out, lse)


@pytest.mark.parametrize("keys", [0, 1, 100000])
@pytest.mark.parametrize("hint", [0, 1, 7, 40, 2000])
def test_any_hint_of_the_longest_chunk_and_sequence_is_right(hint, keys):
    pool, q, start, total = _case("bf16", 8, 2, 32, [(1, 90), (33, 150), (300, 420), (1, 1700)])
    out, lse = attend4(pool, q, start, total, max_q_len=hint, max_kv_len=keys)
    check_attention(pool, q, start, total, out, lse)


@pytest.mark.parametrize("dtype,hint", [("bf16", 1), ("bf16", 0), ("fp32", 1), ("fp32", 0)])
def test_units_that_are_not_cut(dtype, hint):
    """Sequences said to be short, whatever they are: more units than workgroups, empty ones among them."""
    seqs = [(1, 1 + 5 * i % 111) if i % 7 else (0, 0) for i in range(100)] + [(40, 900), (1, 0), (3, 2)]
    pool, q, start, total = _case(dtype, 12, 6, 16, seqs)
    out, lse = attend4(pool, q, start, total, max_q_len=hint, max_kv_len=100)
    check_attention(pool, q, start, total, out, lse)


@pytest.mark.parametrize("hint", [1, 0])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("keys,scale", [(20.0, 0.5), (1.0, 1e-38), (1.0, 2e-30)])
def test_far_logits_and_scales(dtype, hint, keys, scale):
    """Logits of hundreds, and a scale next to nothing, under which all keys weigh the same."""
    pool, q, start, total = _case(dtype, 4, 2, 16, [(1, 900), (20, 700)], scale=keys)
    out, lse = attend4(pool, q, start, total, max_q_len=hint, scale=scale)
    check_attention(pool, q, start, total, out, lse, scale=scale)


@pytest.mark.parametrize("dtype,hint", [("bf16", 1), ("bf16", 0), ("fp32", 1), ("fp32", 0)])
def test_pages_outside_the_pool_hold_nothing(dtype, hint):
    pool, q, start, total = _case(dtype, 8, 2, 16, [(1, 200), (1, 40), (30, 150), (1, 9)])
    table = pool.table.clone()
    table[0, 3], table[0, 12], table[1, :] = -1, pool.n_pages, 2 ** 31 - 1
    table[2, 0], table[2, 8], table[3, 0] = -2 ** 31, -7, pool.n_pages
    out, lse = attend4(pool, q, start, total, table=table, max_q_len=hint)
    check_attention(pool, q, start, total, out, lse, table=table)


def test_arrays_that_say_nonsense_stay_inside_the_tensors():
    pool, q, start, total = _case("bf16", 8, 2, 16, [(3, 60), (2, 30), (4, 100)])
    guard = torch.full((q.shape[0] + 8, 8, 128), 5.0, dtype=q.dtype, device=DEV)
    out = guard[4:-4]
    for hint in (4, 0):
        for start_, total_ in (([-5, 3, 4, 2 ** 31 - 1], total), ([-2 ** 31, -7, 0, 9], [2 ** 31 - 1, -1, 2 ** 31 - 1]), ([0, 0, 2 ** 30, 2 ** 31 - 1], [-2 ** 31, 2 ** 31 - 1, 5])):
            attend4(pool, q, start_, total_, max_q_len=hint, out=out)
        out.fill_(5.0)
        for start_ in ([0, 9, 3, 9], [9, 9, 9, 0], [0, 3, 2, 9], [9, 9, 9, 9], [0, 0, 0, 0]):      # not ascending: nothing is done; or nothing to do
            attend4(pool, q, start_, total, max_q_len=hint, out=out)
        assert (guard == 5).all()
        out.fill_(7.0)
    assert (guard[:4] == 5).all() and (guard[-4:] == 5).all()


def test_rows_of_no_sequence_are_left_alone():
    pool, q, _, total = _case("bf16", 8, 2, 16, [(3, 60), (2, 30)])
    for hint in (4, 1000):
        out = torch.full((5, 8, 128), 5.0, dtype=q.dtype, device=DEV)
        got, lse = attend4(pool, q, [1, 2, 4], total, max_q_len=hint, out=out)
        assert (got[0] == 5).all() and (got[4] == 5).all() and torch.isnan(lse[0]).all() and torch.isfinite(lse[1:4]).all()


def test_pages_beyond_32_bits_of_offset():
    hkv, page, n_pages = 8, 64, 140000                              # 4.6 GB of K
    cache = B.alloc_cache(n_pages, hkv, page, mxfp4=True)
    gen = torch.Generator().manual_seed(1)
    pool = Pool4(gen, [300, 1000], hkv, page)
    pages = torch.arange(n_pages - pool.n_pages, n_pages, device=DEV)
    for mine, far in zip(pool.cache, cache):
        far[pages] = mine
    for new in ([1, 1], [200, 100]):
        q = randn(gen, sum(new), 32, 128).to(DEV)
        want = attend4(pool, q, _starts(new), [300, 1000], max_q_len=max(new))
        table = torch.where((pool.table >= 0) & (pool.table < pool.n_pages), pool.table + (n_pages - pool.n_pages), -1)
        far_pool = type("Far", (), dict(vars(pool), cache=list(cache), table=table))
        got = attend4(far_pool, q, _starts(new), [300, 1000], max_q_len=max(new))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 7), ("bf16", 70), ("fp32", 1), ("fp32", 20)])
def test_a_captured_call_follows_the_lengths(dtype, new):
    gen = torch.Generator().manual_seed(5)
    pool = Pool4(gen, [900, 400, 50 + new], 2, 16, dtype)
    table = pool.table.to(DEV)
    q = randn(gen, 3 * new, 8, 128, dtype=dtype).to(DEV)
    out, lse = torch.empty((3 * new, 8, 128), dtype=q.dtype, device=DEV), torch.empty((3 * new, 8), device=DEV)
    start = torch.tensor(_starts([new] * 3), dtype=torch.int32, device=DEV)
    lens = torch.tensor([900, 400, 50 + new], dtype=torch.int32, device=DEV)
    p = B.make_cache_params(8, 2, q.dtype, q=q, out=out, k_cache=pool.cache[0], mxfp4=True, page_table=table, max_q_len=new)
    ws = B.alloc_paged_workspace(p)

    def call():
        B.critiprefill_paged_attn(p, q, *pool.cache, table, start, lens, out, lse, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for held in ([900, 400, 50 + new], [new, 130, 17], [500, 399, new], [0, 1, 2], [900, 400, 50 + new]):
        lens.copy_(torch.tensor(held, dtype=torch.int32))
        q.copy_(randn(gen, 3 * new, 8, 128, dtype=dtype))
        call()
        torch.cuda.synchronize()
        eager = out.clone(), lse.clone()
        out.zero_(); lse.zero_(); ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
        check_attention(pool, q, _starts([new] * 3), held, out, lse)


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 8), ("bf16", 300), ("fp32", 9)])
def test_the_same_twice_and_beside_other_work(dtype, new):
    pool, q, start, total = _case(dtype, 8, 2, 64, [(new, 3000), (new, 700)])
    first = attend4(pool, q, start, total, max_q_len=new)
    side = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device=DEV)
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            busy = busy @ busy * 1e-3
        again = attend4(pool, q, start, total, max_q_len=new)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    torch.cuda.synchronize()


def _compare(pool, q, start, total, out, lse, dtype):
    with np.errstate(invalid="ignore"):
        want, want_lse, _, _ = O.paged_attention(f64(q), pool.held_k, pool.held_v, pool.page, pool.table.numpy(), start, total, 128 ** -0.5)
    got, got_lse = f64(out), f64(lse)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isnan(got_lse), np.isnan(want_lse)) and not np.isinf(got).any()
    fine = np.isfinite(want)
    assert fine.any() and not fine.all()
    # bf16: P and out rounded, 2^-8 of a term and of the result each at most, and fp32's roundings; both as shares of the largest
    assert np.abs(got[fine] - want[fine]).max() <= (2.0 ** -6 if dtype == "bf16" else 1e-5) * np.abs(want[fine]).max()


ODD = [("bf16", 4, 1, 16, [(4, 40), (2, 9)]), ("bf16", 8, 2, 64, [(100, 230), (5, 5)]), ("bf16", 8, 2, 16, [(70, 70), (1, 40)]), ("fp32", 4, 2, 16, [(6, 50), (40, 40)]),
       ("fp32", 1, 1, 64, [(16, 16)]), ("bf16", 4, 1, 64, [(300, 5000)]), ("bf16", 8, 1, 32, [(4, 900)])]


@pytest.mark.parametrize("dtype,hq,hkv,page,seqs", ODD)
def test_blocks_of_nan_stay_with_the_rows_that_see_them(dtype, hq, hkv, page, seqs):
    """32 channels of K or V of some new tokens are NaN: the rows before them must not notice, those that see them are NaN, of V in these channels alone."""
    pool, q, start, total = _case(dtype, hq, hkv, page, seqs)
    for i, (n, t) in enumerate(seqs):
        if n < 2:
            continue
        for u, which, block in ((t - 1, 0, 0), (t - n // 2, 1, 2), (t - n // 3 - 1, 1, 0), (t - n + 1, 1, 3)):
            slot = int(pool.slots[i][u])
            pool.spoil(which, slot // page, i % hkv, slot % page, block)
    out, lse = attend4(pool, q, start, total, max_q_len=max(n for n, _ in seqs))
    _compare(pool, q, start, total, out, lse, dtype)


@pytest.mark.parametrize("dtype,hq,hkv,page,seqs", [("bf16", 8, 2, 64, [(100, 230), (70, 5000)]), ("bf16", 16, 1, 16, [(40, 200), (33, 33)]), ("bf16", 1, 1, 32, [(700, 1000)]),
                                                     ("bf16", 4, 1, 16, [(4, 600)]), ("bf16", 8, 1, 16, [(4, 600)]), ("fp32", 4, 1, 16, [(40, 300)])])
@pytest.mark.parametrize("before", [0, 70])
def test_blocks_of_nan_at_any_key(dtype, hq, hkv, page, seqs, before):
    """Key after key of the new tokens, and of some before them, one block of V each; the fourth stays finite."""
    pool, q, start, total = _case(dtype, hq, hkv, page, seqs)
    for i, (n, t) in enumerate(seqs):
        for u in range(max(0, t - n + 1 - before), t, 1 if n < 60 else 7):
            slot = int(pool.slots[i][u])
            for h in range(hkv):
                pool.spoil(1, slot // page, h, slot % page, u % 3)
    out, lse = attend4(pool, q, start, total, max_q_len=max(n for n, _ in seqs))
    _compare(pool, q, start, total, out, lse, dtype)


# Tiles of 256 rows, in every way that their units are dealt out: rounds that leave nothing, that leave some to be cut, or whole; whole as the lengths turn out or as the host says; cut.
TILES = [(32, 8, 64, [(512, 812)] * 8), (64, 4, 16, [(48, 1000)] * 64), (28, 4, 32, [(512, 812)] * 17), (64, 1, 32, [(3100, 3311)]), (28, 4, 64, [(257, 900)] * 17),
         (32, 8, 32, [(130, 900)] * 4), (32, 8, 64, [(200 + 37 * i, 820 + 50 * i) for i in range(5)]), (32, 8, 64, [(300, 600)] * 4),
         (32, 8, 64, [(70, 4000), (300, 900), (0, 0), (1, 1700)]), (16, 4, 16, [(130, 1300)] * 70)]


def _width(seqs, page):
    return max(-(-t // page) for _, t in seqs) + 1                  # of Pool's page table


def tiles_route(case):
    hq, hkv, page, seqs = case
    return dealing("bf16", 2, hq, hkv, seqs, _width(seqs, page) * page)


@pytest.mark.parametrize("case", TILES, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}x{len(c[3])}x{c[3][0][0]}x{c[3][0][1]}")
def test_dealt_tiles(case):
    hq, hkv, page, seqs = case
    gen = torch.Generator().manual_seed(len(seqs) + hq)
    new, total = zip(*seqs)
    pool = Pool4(gen, total, hkv, page)
    assert pool.table.shape[1] == _width(seqs, page)
    q, start = randn(gen, sum(new), hq, 128).to(DEV), _starts(new)
    out, lse = attend4(pool, q, start, total, max_q_len=max(new))
    want, want_lse, size, logit = _plain(pool, q, start, total, 128 ** -0.5)
    # the bound of cache_helpers.check_attention
    delta = 2.0 ** -20 * (logit + want_lse.abs().clamp(min=1.0)) + 2.0 ** -20
    bound = HALF_STEP["bf16"] * (size + want.abs()) * 1.01 + 4 * delta[..., None] * size.amax(-1, keepdim=True) + 1e-30
    worst = float(((out.double() - want).abs() / bound).max())
    assert torch.isfinite(out).all() and worst <= 1.0, f"out: {worst:.2f} of the bound"
    assert ((lse.double() - want_lse).abs() <= 2 * delta).all()


# Both sides of the lines between the kernels, their tiles and units cut or whole: dtype, heads, page, sequences.
AROUND = [("bf16", 8, 2, 16, [(16, 700), (3, 90)] * 3), ("bf16", 8, 2, 16, [(17, 700), (3, 90)] * 3), ("bf16", 8, 2, 64, [(32, 5000)]), ("bf16", 8, 2, 64, [(33, 5000)]), ("bf16", 8, 2, 64, [(64, 3900)]),
          ("bf16", 8, 2, 64, [(65, 3900)]), ("bf16", 32, 1, 32, [(2, 300), (1, 40)]), ("bf16", 32, 1, 16, [(1, 800)]), ("bf16", 33, 1, 32, [(1, 300)]), ("bf16", 33, 1, 32, [(1, 200), (1, 31)]), ("bf16", 32, 8, 64, [(1, 700)] * 3),
          ("bf16", 32, 8, 64, [(1, 800)] * 3), ("bf16", 32, 8, 16, [(1, 1000)] * 8), ("bf16", 32, 8, 64, [(2, 1900 - 50 * i) for i in range(33)]), ("bf16", 4, 2, 16, [(1, 2100), (1, 5)] * 70),
          ("fp32", 8, 2, 16, [(1, 480)] * 3), ("fp32", 8, 2, 64, [(1, 700), (3, 90)]), ("fp32", 8, 2, 32, [(4, 1000 - 20 * i) for i in range(33)]), ("fp32", 17, 1, 16, [(2, 300), (1, 1)]),
          ("fp32", 40, 1, 64, [(3, 900), (1, 64)]), ("fp32", 64, 1, 16, [(2, 130)]), ("fp32", 4, 2, 16, [(200, 1500)])]


def around_route(case):
    dtype, hq, hkv, page, seqs = case
    return route(dtype, 2, hq, hkv, len(seqs), max(n for n, _ in seqs), _width(seqs, page) * page)


@pytest.mark.parametrize("case", AROUND, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}x{c[3]}x{len(c[4])}x{c[4][0][0]}x{c[4][0][1]}")
def test_around_the_lines(case):
    dtype, hq, hkv, page, seqs = case
    pool, q, start, total = _case(dtype, hq, hkv, page, seqs)
    assert pool.table.shape[1] == _width(seqs, page)
    out, lse = attend4(pool, q, start, total, max_q_len=max(n for n, _ in seqs))
    check_attention(pool, q, start, total, out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_units_of_one_step_one_after_another(dtype):
    """Workgroups that go through many units of one step each, empty ones and ones that see nothing among them, and of two and three steps: the next unit's keys are asked for in the last step."""
    seqs = [(1, (1, 128, 0, 129, 37, 257, 1, 384)[i % 8]) if i % 11 else (0, 0) for i in range(700)]
    pool, q, start, total = _case(dtype, 4, 2, 16, seqs)
    for max_kv in (0, 400):
        out, lse = attend4(pool, q, start, total, max_q_len=1, max_kv_len=max_kv)
        check_attention(pool, q, start, total, out, lse)


def test_fp32_queries_of_any_size():
    """Queries and keys from far apart ranges: three bf16 pieces hold all of an fp32 number, so that a logit is as exact as its sum."""
    pool, q, start, total = _case("fp32", 8, 2, 16, [(1, 300), (5, 90)], scale=2.0 ** -60)
    q = q * 2.0 ** 60 * (1 + torch.arange(128, device=DEV) * 2.0 ** -17)
    q[0, 0, 5], q[1, 1] = 3.4028234e38 * 2.0 ** -64, 0.0
    out, lse = attend4(pool, q, start, total, max_q_len=5)
    check_attention(pool, q, start, total, out, lse)


# Single tokens with a chunk or two among them: both kernels, each with its own sequences.  Of up to so many new tokens, and of more; none at all; keys that none of them sees.
MIXED = [(32, 8, 64, [(1, 100 + 30 * i) for i in range(38)] + [(300, 1400), (4, 700), (5, 710), (0, 500), (2, 1), (0, 0)], 4), (28, 4, 16, [(2, 1500 - 9 * i) for i in range(80)] + [(60, 60), (3, 900)], 2),
         (32, 1, 32, [(1, 5600 - 70 * i) for i in range(72)] + [(9, 300)], 1), (5, 1, 16, [(3, 4100), (1, 90)] * 50 + [(120, 700)], 3), (32, 8, 64, [(1, 1400)] * 40, 4)]


def few_of(case):
    hq, hkv, page, seqs, _ = case
    f = B.load()._ZN2cp10few_tokensERKNS_10CacheShapeE
    f.argtypes, f.restype = [ctypes.POINTER(Shape)], ctypes.c_int
    max_q = max(n for n, _ in seqs)
    return f(Shape(dtype=1, mxfp8=2, hq=hq, hkv=hkv, group=hq // hkv, n_seqs=len(seqs), max_q=max_q if max_q > 1 else 100, max_kv=_width(seqs, page) * page, tokens=sum(n for n, _ in seqs)))


@pytest.mark.parametrize("case", MIXED, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}x{len(c[3])}")
def test_single_tokens_beside_a_chunk(case):
    hq, hkv, page, seqs, few = case
    assert few_of(case) == few
    pool, q, start, total = _case("bf16", hq, hkv, page, seqs)
    assert pool.table.shape[1] == _width(seqs, page)
    longest = max(n for n, _ in seqs)
    out, lse = attend4(pool, q, start, total, max_q_len=longest if longest > 1 else 100)     # the last: a bound that no sequence comes near to
    check_attention(pool, q, start, total, out, lse)


def test_single_tokens_beside_a_chunk_captured_and_out_of_order():
    """Replays follow the lengths, sequences change sides; rows that do not ascend are nobody's, in either kernel; rows behind the last sequence stay as they are."""
    gen = torch.Generator().manual_seed(8)
    seqs = [(1, 1400 - 11 * i) for i in range(40)] + [(90, 700)]
    pool = Pool4(gen, [t for _, t in seqs], 8, 64)
    table, q = pool.table.to(DEV), randn(gen, 140, 32, 128).to(DEV)
    out, lse = torch.full((140, 32, 128), 5.0, dtype=q.dtype, device=DEV), torch.full((140, 32), 5.0, device=DEV)
    p = B.make_cache_params(32, 8, q.dtype, q=q, out=out, k_cache=pool.cache[0], mxfp4=True, page_table=table, max_q_len=100)
    ws = B.alloc_paged_workspace(p)
    start, lens = torch.zeros(42, dtype=torch.int32, device=DEV), torch.zeros(41, dtype=torch.int32, device=DEV)

    def call():
        B.critiprefill_paged_attn(p, q, *pool.cache, table, start, lens, out, lse, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for new, held in (([1] * 40 + [90], [t for _, t in seqs]), ([3] * 20 + [0] * 20 + [70], [900 - i for i in range(40)] + [700]), ([1] * 40 + [1], [5] * 41), ([0] * 40 + [100], [0] * 40 + [700])):
        start.copy_(torch.tensor(_starts(new), dtype=torch.int32))
        lens.copy_(torch.tensor(held, dtype=torch.int32))
        out.fill_(5.0); lse.fill_(5.0)
        call()
        torch.cuda.synchronize()
        eager = out.clone(), lse.clone()
        out.fill_(5.0); lse.fill_(5.0); ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
        n = sum(new)
        check_attention(pool, q[:n], _starts(new), held, out[:n], lse[:n])
        assert (out[n:] == 5).all() and (lse[n:] == 5).all()
    start.copy_(torch.tensor(list(range(20)) + [18] + list(range(21, 42)), dtype=torch.int32))
    out.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    assert (out == 7).all()


# Cut units by number, of rows that no group of the joining kernel divides: dtype, heads, page, sequences.
JOINED = [(dtype, hq, hkv, 32, [(new, 2500 - 70 * i) for i in range(n)]) for dtype in ("bf16", "fp32")
          for hq, hkv, new, n in ((32, 8, 1, 3), (32, 8, 1, 4), (24, 8, 1, 7), (24, 8, 1, 8), (40, 8, 1, 9), (8, 8, 1, 10), (28, 4, 3, 17))]


@pytest.mark.parametrize("case", JOINED, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}x{len(c[4])}x{c[4][0][0]}")
def test_parts_joined_by_few_and_many_groups(case):
    """The call's hint of the longest chunk may be too small: the joining kernel's workgroups then take the rows behind those that they were launched for in turn."""
    dtype, hq, hkv, page, seqs = case
    assert not route(dtype, 2, hq, hkv, len(seqs), seqs[0][0], _width(seqs, page) * page).whole
    pool, q, start, total = _case(dtype, hq, hkv, page, seqs)
    for hint in (seqs[0][0], 1):
        out, lse = attend4(pool, q, start, total, max_q_len=hint)
        check_attention(pool, q, start, total, out, lse)


@pytest.mark.parametrize("dtype,hint", [("bf16", 4), ("bf16", 0), ("fp32", 4)])
def test_nonsense_of_a_single_sequence(dtype, hint):
    """The share of a single sequence is found by loads of its own."""
    pool, q, start, total = _case(dtype, 8, 2, 16, [(4, 600)])
    rows = torch.full((12, 8, 128), 5.0, dtype=q.dtype, device=DEV)
    out = rows[4:-4]
    table = pool.table.clone()
    for start_, held in (([-5, 2 ** 31 - 1], 2 ** 31 - 1), ([-2 ** 31, 4], -1), ([1, 2 ** 30], -2 ** 31), ([0, 4], 2 ** 31 - 1)):
        attend4(pool, q, start_, [held], table=table, max_q_len=hint, out=out)
    out.fill_(5.0)
    for start_ in ([4, 0], [2 ** 31 - 1, -1], [4, 4], [0, 0], [9, 9]):
        attend4(pool, q, start_, total, max_q_len=hint, out=out)
    assert bool((rows == 5.0).all())
    table[0, :] = -1                                                 # no page is there: nothing to see
    got, lse = attend4(pool, q, start, total, table=table, max_q_len=hint)
    assert not got.any() and bool((lse == -float("inf")).all())


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 5), ("fp32", 3)])
def test_a_captured_single_sequence_follows_its_length(dtype, new):
    pool, q, start, total = _case(dtype, 8, 2, 32, [(new, 2100)])
    table = pool.table.to(DEV)
    out, lse = torch.empty((new, 8, 128), dtype=q.dtype, device=DEV), torch.empty((new, 8), device=DEV)
    starts, lens = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (start, total))
    p = B.make_cache_params(8, 2, q.dtype, q=q, out=out, k_cache=pool.cache[0], mxfp4=True, page_table=table, max_q_len=new)
    ws = B.alloc_paged_workspace(p)
    call = lambda: B.critiprefill_paged_attn(p, q, *pool.cache, table, starts, lens, out, lse, ws)      # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for held in (2100, new, 0, 1, 129, 1500, 2100):
        lens.fill_(held)
        out.zero_(); lse.zero_(); ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        check_attention(pool, q, start, [held], out, lse)


@pytest.mark.parametrize("dtype,seqs", [("bf16", [(1, 900), (1, 40)]), ("bf16", [(90, 900), (1, 40), (70, 70)]), ("fp32", [(3, 700)])])
def test_outputs_with_gaps_and_no_sum(dtype, seqs):
    pool, q, start, total = _case(dtype, 8, 2, 16, seqs)
    room = torch.full((2 * q.shape[0], 9, 136), 7.0, dtype=q.dtype, device=DEV)
    out = room[::2, 1:, :128]
    table = pool.table.to(DEV)
    p = B.make_cache_params(8, 2, q.dtype, q=q, out=out, k_cache=pool.cache[0], mxfp4=True, page_table=table)
    starts, lens = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (start, total))
    B.critiprefill_paged_attn(p, q, *pool.cache, table, starts, lens, out, None, B.alloc_paged_workspace(p))
    torch.cuda.synchronize()
    want, lse = attend4(pool, q, start, total)
    assert torch.equal(out, want)
    check_attention(pool, q, start, total, want, lse)
    out.fill_(7.0)
    assert bool((room == 7.0).all())


@pytest.mark.parametrize("dtype,hint", [("bf16", 1), ("bf16", 300), ("fp32", 2)])
def test_a_table_without_pages(dtype, hint):
    pool, q, start, total = _case(dtype, 8, 2, 16, [(2, 90), (1, 30)])
    out, lse = attend4(pool, q, start, total, table=torch.empty((2, 0), dtype=torch.int32), max_q_len=hint)
    assert not out.any() and bool((lse == -float("inf")).all())


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 100), ("fp32", 5)])
def test_two_calls_at_once(dtype, new):
    """On two streams, each with outputs and a workspace of its own."""
    cases = [_case(dtype, 8, 2, 16, [(new, 2000 - 90 * i) for i in range(n)], seed=n) for n in (1, 9)]
    want = [attend4(*c, max_q_len=new) for c in cases]
    calls = []
    for pool, q, start, total in cases:
        table, out, lse = pool.table.to(DEV), torch.zeros((q.shape[0], 8, 128), dtype=q.dtype, device=DEV), torch.zeros((q.shape[0], 8), device=DEV)
        p = B.make_cache_params(8, 2, q.dtype, q=q, out=out, k_cache=pool.cache[0], mxfp4=True, page_table=table, max_q_len=new)
        calls.append((p, q, *pool.cache, table, *(torch.tensor(x, dtype=torch.int32, device=DEV) for x in (start, total)), out, lse, B.alloc_paged_workspace(p)))
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, c in zip(streams, calls):
            with torch.cuda.stream(s):
                B.critiprefill_paged_attn(*c)
    torch.cuda.synchronize()
    for w, c in zip(want, calls):
        assert torch.equal(w[0], c[-3]) and torch.equal(w[1], c[-2])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [64, 65, 128, 129, 4096, 4097])
def test_many_sequences(dtype, n):
    """On both sides of the numbers up to which a run's beginning is found in one look, by the waves in turn, and by all of them."""
    lengths = [(1, 3000) if i % 997 == 5 else (1, 300) if i % 97 == 6 else ((0, 0), (1, 1 + 13 * i % 40), (1, 0), (2, 1), (1, 17))[i % 5] for i in range(n)]
    pool, q, start, total = _case(dtype, 4, 2, 16, lengths)
    for keys in (0, 200):                                            # cut, as the table is wide, and not cut
        assert route(dtype, 2, 4, 2, n, 1, keys or pool.table.shape[1] * 16).whole == (keys > 0)
        out, lse = attend4(pool, q, start, total, max_q_len=1, max_kv_len=keys)
        check_attention(pool, q, start, total, out, lse)
    rows = torch.full_like(q, 5.0, memory_format=torch.contiguous_format)
    for at in (1, n // 2, n):                                        # not ascending there: nothing is done
        wrong = list(start)
        wrong[at] = wrong[at - 1] - 1
        attend4(pool, q, wrong, total, max_q_len=1, out=rows)
    assert bool((rows == 5.0).all())


@pytest.mark.parametrize("power", [-100, -110, -118, -124])
def test_fp32_queries_next_to_nothing(power):
    """Queries of 2^power under keys as much larger: the third piece of an element below 2^-110 is a bf16 number of fewer bits, and what lies below the last of them, 2^-133, is cut off.  A logit is off by
    that much of each of its key's channels beside what cache_helpers.check_attention has."""
    scale = 128 ** -0.5
    pool, q, start, total = _case("fp32", 8, 2, 16, [(1, 300), (5, 90)], scale=2.0 ** -power)
    q = q * 2.0 ** power
    out, lse = attend4(pool, q, start, total, max_q_len=5)
    want, want_lse, size, logit = O.paged_attention(f64(q), pool.held_k, pool.held_v, pool.page, pool.table.numpy(), start, total, scale)
    lost = 2.0 ** -133 * np.nanmax(np.abs(pool.held_k).sum(-1)) * scale
    delta = 2.0 ** -20 * (logit + np.maximum(np.abs(want_lse), 1.0)) + 2.0 ** -20 + lost
    bound = 2.0 ** -24 * np.abs(want) * 1.01 + 4 * delta[..., None] * size.max(-1, keepdims=True)
    assert (np.abs(f64(out) - want) <= bound).all() and (np.abs(f64(lse) - want_lse) <= 2 * delta).all()
