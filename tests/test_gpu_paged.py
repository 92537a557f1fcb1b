"""Attention of new tokens over the pages of a cache against fp64: single tokens, chunks, mixed batches, every head layout, lengths of zero and one, pages that
end anywhere, what hidden places hold, and arrays that say nonsense."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2409_12490_amd import binding as B
from tests.cache_helpers import DEV, Pool, attend, check_attention, f64, randn

pytestmark = pytest.mark.gpu


def _starts(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(int).tolist()


def _case(dtype, mxfp8, hq, hkv, page, seqs, seed=0, scale=1.0):
    """seqs: (new tokens, tokens in all)."""
    gen = torch.Generator().manual_seed(seed + 17 * len(seqs) + hq)
    new, total = zip(*seqs)
    pool = Pool(gen, total, hkv, page, dtype, mxfp8, scale=scale)
    q = randn(gen, max(sum(new), 1), hq + 1, 128, dtype=dtype).to(DEV)[:sum(new), :hq]        # with a gap behind the heads
    return pool, q, _starts(new), list(total)


EDGES = [(1, n) for n in (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000)]
CASES = [
    # decode: every head layout, lengths around every edge
    ("bf16", 32, 8, 64, EDGES), ("bf16", 32, 4, 16, EDGES), ("bf16", 4, 4, 32, EDGES), ("bf16", 28, 4, 64, EDGES[::3]), ("bf16", 40, 8, 128, EDGES[::4]),
    ("bf16", 32, 1, 64, EDGES[::3]), ("bf16", 64, 1, 16, EDGES[::4]), ("bf16", 3, 3, 256, [(1, 700), (1, 3)]), ("bf16", 17, 1, 32, [(1, 100), (1, 33)]),
    ("fp32", 8, 2, 16, EDGES), ("fp32", 3, 3, 64, EDGES[::2]), ("fp32", 33, 1, 64, EDGES[::5]), ("fp32", 64, 1, 32, [(1, 70)]),
    # a long sequence over many workgroups
    ("bf16", 8, 2, 64, [(1, 20001)]), ("bf16", 2, 1, 16, [(1, 9000), (1, 40)]), ("fp32", 2, 1, 32, [(1, 5003)]),
    # more sequences than a wave has lanes
    ("bf16", 2, 1, 16, [(1, 1 + 7 * i % 90) for i in range(150)]),
    # a few tokens each
    ("bf16", 32, 8, 64, [(2, 2), (4, 100), (3, 65), (4, 4), (1, 1)]), ("bf16", 8, 2, 16, [(5, 5), (8, 300), (16, 64)]), ("fp32", 4, 2, 16, [(7, 31), (8, 8)]),
    # chunks, with and without a past
    ("bf16", 4, 1, 64, [(64, 64), (65, 65), (63, 700)]), ("bf16", 8, 2, 32, [(300, 300), (17, 1000)]), ("bf16", 5, 1, 16, [(130, 201)]),
    ("bf16", 7, 1, 64, [(257, 258)]), ("bf16", 2, 2, 128, [(515, 1030)]), ("bf16", 16, 1, 64, [(77, 400)]), ("bf16", 64, 1, 64, [(9, 200)]),
    ("fp32", 2, 1, 64, [(200, 333)]), ("fp32", 3, 3, 16, [(90, 90), (40, 290)]), ("fp32", 8, 1, 16, [(33, 150)]),
    # everything in one batch, sequences without new tokens and without any, new tokens that nothing is held for
    ("bf16", 8, 2, 64, [(1, 500), (200, 260), (0, 77), (1, 0), (0, 0), (5, 3), (1, 1), (64, 2000), (3, 0)]),
    ("fp32", 4, 2, 16, [(0, 0), (2, 1), (40, 100), (1, 300), (0, 10), (4, 0)]),
    # sequences that are alike, units for two and more rounds of workgroups: none left over, some left over, an odd number of rounds
    ("bf16", 32, 4, 16, [(512, 600)] * 8), ("bf16", 16, 2, 64, [(600, 600)] * 17), ("bf16", 64, 1, 64, [(3100, 3111)]),
]


@pytest.mark.parametrize("mxfp8", [False, True], ids=["plain", "mxfp8"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}x{c[3]}x{len(c[4])}x{c[4][0][0]}x{c[4][0][1]}")
def test_against_fp64(case, mxfp8):
    dtype, hq, hkv, page, seqs = case
    pool, q, start, total = _case(dtype, mxfp8, hq, hkv, page, seqs)
    out, lse = attend(pool, q, start, total, max_q_len=max(n for n, _ in seqs))
    check_attention(pool, q, start, total, out, lse)


@pytest.mark.parametrize("keys", [0, 1, 100000])
@pytest.mark.parametrize("hint", [0, 1, 7, 40, 2000])
def test_any_hint_of_the_longest_chunk_and_sequence_is_right(hint, keys):
    pool, q, start, total = _case("bf16", hint % 2 == 1, 8, 2, 32, [(1, 90), (33, 150), (300, 420), (1, 1700)])
    out, lse = attend(pool, q, start, total, max_q_len=hint, max_kv_len=keys)
    check_attention(pool, q, start, total, out, lse)


@pytest.mark.parametrize("mxfp8", [False, True], ids=["plain", "mxfp8"])
@pytest.mark.parametrize("dtype,hint", [("bf16", 1), ("bf16", 0), ("fp32", 1), ("fp32", 0)])
def test_units_that_are_not_cut(dtype, hint, mxfp8):
    """Sequences said to be short, whatever they are: more units than workgroups, empty ones among them."""
    seqs = [(1, 1 + 5 * i % 111) if i % 7 else (0, 0) for i in range(100)] + [(40, 900), (1, 0), (3, 2)]
    pool, q, start, total = _case(dtype, mxfp8, 12, 6, 16, seqs)
    out, lse = attend(pool, q, start, total, max_q_len=hint, max_kv_len=100)
    check_attention(pool, q, start, total, out, lse)


# The kernel of 256-row tiles leaves units whole where that takes no longer: all of them (alike, ragged, more sequences than a wave has lanes), those that rounds leave
# over, in a round of its own or two; and cuts them where it does.
DEALT = [("bf16", 32, 8, 32, [(300, 600)] * 4), ("bf16", 32, 8, 64, [(200 + 37 * i, 520 + 50 * i) for i in range(5)]), ("bf16", 8, 2, 16, [(5 + i % 40, 300 + 7 * i) for i in range(70)]),
         ("bf16", 32, 8, 64, [(130, 560)] * 12), ("bf16", 16, 4, 16, [(460, 700)] * 10), ("bf16", 32, 8, 64, [(70, 4000), (300, 600), (0, 0), (1, 700)]), ("bf16", 32, 1, 32, [(257, 9000)]),
         ("bf16", 4, 2, 64, [(128, 520)] * 129),
         # 17 to 32 rows: of one sequence, of a long one, of several
         ("bf16", 32, 8, 64, [(8, 3000)]), ("bf16", 28, 4, 16, [(3, 700), (4, 90)]), ("bf16", 8, 1, 32, [(4, 26000)]), ("bf16", 32, 8, 64, [(7, 900), (5, 400)]),
         # fp32, tiles of 16 and of 32 rows
         ("fp32", 4, 2, 16, [(60, 1500), (200, 700), (1, 2000)]), ("fp32", 4, 2, 64, [(9, 700)]), ("fp32", 20, 1, 16, [(5, 200), (1, 900)]), ("fp32", 3, 1, 32, [(40, 3000), (33, 33)])]


@pytest.mark.parametrize("mxfp8", [False, True], ids=["plain", "mxfp8"])
@pytest.mark.parametrize("case", DEALT, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}x{c[3]}x{len(c[4])}x{c[4][0][0]}x{c[4][0][1]}")
def test_units_whole_and_cut(case, mxfp8):
    dtype, hq, hkv, page, seqs = case
    pool, q, start, total = _case(dtype, mxfp8, hq, hkv, page, seqs)
    out, lse = attend(pool, q, start, total, max_q_len=max(n for n, _ in seqs))
    check_attention(pool, q, start, total, out, lse)


@pytest.mark.parametrize("hint", [1, 0])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_far_logits_and_a_scale(dtype, hint):
    pool, q, start, total = _case(dtype, False, 4, 2, 16, [(1, 300), (20, 200)], scale=20.0)
    out, lse = attend(pool, q, start, total, max_q_len=hint, scale=0.5)
    check_attention(pool, q, start, total, out, lse, scale=0.5)


@pytest.mark.parametrize("hint", [1, 0])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [1e-38, 2e-30])
def test_a_scale_next_to_nothing(scale, dtype, hint):
    """All keys weigh the same; units of several steps that are not cut."""
    pool, q, start, total = _case(dtype, False, 4, 2, 16, [(1, 900), (20, 700)])
    out, lse = attend(pool, q, start, total, max_q_len=hint, max_kv_len=100, scale=scale)
    check_attention(pool, q, start, total, out, lse, scale=scale)


@pytest.mark.parametrize("dtype,mxfp8,hint", [("bf16", False, 1), ("bf16", True, 1), ("bf16", False, 0), ("bf16", True, 0), ("fp32", False, 1), ("fp32", True, 0)])
def test_pages_outside_the_pool_hold_nothing(dtype, mxfp8, hint):
    pool, q, start, total = _case(dtype, mxfp8, 8, 2, 16, [(1, 200), (1, 40), (30, 150), (1, 9)])
    table = pool.table.clone()
    table[0, 3], table[0, 12], table[1, :] = -1, pool.n_pages, 2 ** 31 - 1
    table[2, 0], table[2, 8], table[3, 0] = -2 ** 31, -7, pool.n_pages
    out, lse = attend(pool, q, start, total, table=table, max_q_len=hint)
    check_attention(pool, q, start, total, out, lse, table=table)


def test_arrays_that_say_nonsense_stay_inside_the_tensors():
    pool, q, start, total = _case("bf16", False, 8, 2, 16, [(3, 60), (2, 30), (4, 100)])
    guard = torch.full((q.shape[0] + 8, 8, 128), 5.0, dtype=q.dtype, device=DEV)
    out = guard[4:-4]
    for hint in (4, 0):
        for start_, total_ in (([-5, 3, 4, 2 ** 31 - 1], total), ([-2 ** 31, -7, 0, 9], [2 ** 31 - 1, -1, 2 ** 31 - 1]), ([0, 0, 2 ** 30, 2 ** 31 - 1], [-2 ** 31, 2 ** 31 - 1, 5])):
            attend(pool, q, start_, total_, max_q_len=hint, out=out)
        out.fill_(5.0)
        for start_ in ([0, 9, 3, 9], [9, 9, 9, 0], [0, 3, 2, 9], [9, 9, 9, 9], [0, 0, 0, 0]):      # not ascending: nothing is done; or nothing to do
            attend(pool, q, start_, total, max_q_len=hint, out=out)
        assert (guard == 5).all()
        out.fill_(7.0)
    assert (guard[:4] == 5).all() and (guard[-4:] == 5).all()


def test_rows_of_no_sequence_are_left_alone():
    pool, q, _, total = _case("bf16", False, 8, 2, 16, [(3, 60), (2, 30)])
    out = torch.full((5, 8, 128), 5.0, dtype=q.dtype, device=DEV)
    got, lse = attend(pool, q, [1, 2, 4], total, max_q_len=4, out=out)
    assert (got[0] == 5).all() and (got[4] == 5).all() and torch.isnan(lse[0]).all() and torch.isfinite(lse[1:4]).all()


def test_pages_beyond_32_bits_of_offset():
    hkv, page, n_pages = 8, 64, 36000                               # 4.7 GB of K
    cache = B.alloc_cache(n_pages, hkv, page)
    gen = torch.Generator().manual_seed(1)
    pool = Pool(gen, [300, 1000], hkv, page)
    pages = torch.arange(n_pages - pool.n_pages, n_pages, device=DEV)
    for mine, far in zip(pool.cache[:2], cache[:2]):
        far[pages] = mine
    for new in ([1, 1], [200, 100]):
        q = randn(gen, sum(new), 32, 128).to(DEV)
        want = attend(pool, q, _starts(new), [300, 1000], max_q_len=max(new))
        table = torch.where((pool.table >= 0) & (pool.table < pool.n_pages), pool.table + (n_pages - pool.n_pages), -1)
        far_pool = type("Far", (), dict(vars(pool), cache=list(cache), table=table))
        got = attend(far_pool, q, _starts(new), [300, 1000], max_q_len=max(new))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("mxfp8", [False, True], ids=["plain", "mxfp8"])
@pytest.mark.parametrize("new", [1, 70])
def test_a_captured_call_follows_the_lengths(new, mxfp8):
    gen = torch.Generator().manual_seed(5)
    pool = Pool(gen, [900, 400, 50 + new], 2, 16, "bf16", mxfp8)
    table = pool.table.to(DEV)
    q = randn(gen, 3 * new, 8, 128).to(DEV)
    out, lse = torch.empty((3 * new, 8, 128), dtype=q.dtype, device=DEV), torch.empty((3 * new, 8), device=DEV)
    start = torch.tensor(_starts([new] * 3), dtype=torch.int32, device=DEV)
    lens = torch.tensor([900, 400, 50 + new], dtype=torch.int32, device=DEV)
    p = B.make_cache_params(8, 2, q.dtype, q=q, out=out, k_cache=pool.cache[0], mxfp8=mxfp8, page_table=table, max_q_len=new)
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
        q.copy_(randn(gen, 3 * new, 8, 128))
        call()
        torch.cuda.synchronize()
        eager = out.clone(), lse.clone()
        out.zero_(); lse.zero_(); ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
        check_attention(pool, q, _starts([new] * 3), held, out, lse)


@pytest.mark.parametrize("dtype,mxfp8,new", [("bf16", False, 1), ("bf16", True, 40), ("bf16", False, 300), ("fp32", False, 9)])
def test_the_same_twice_and_beside_other_work(dtype, mxfp8, new):
    pool, q, start, total = _case(dtype, mxfp8, 8, 2, 64, [(new, 3000), (new, 700)])
    first = attend(pool, q, start, total, max_q_len=new)
    side = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device=DEV)
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            busy = busy @ busy * 1e-3
        again = attend(pool, q, start, total, max_q_len=new)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    torch.cuda.synchronize()


@pytest.mark.parametrize("mxfp8", [False, True], ids=["plain", "mxfp8"])
@pytest.mark.parametrize("dtype,hq,hkv,page,seqs", [("bf16", 4, 1, 16, [(4, 40), (2, 9)]), ("bf16", 8, 2, 64, [(100, 230), (5, 5)]), ("bf16", 8, 2, 16, [(70, 70), (1, 40)]),
                                                     ("fp32", 4, 2, 16, [(6, 50), (40, 40)]), ("fp32", 1, 1, 64, [(16, 16)]), ("bf16", 4, 1, 64, [(300, 5000)])])
def test_what_is_not_finite_stays_with_the_rows_that_see_it(dtype, hq, hkv, page, seqs, mxfp8):
    """K and V of some new tokens hold infinities and NaN: the rows before them must not notice, those that see them get what the formula gives."""
    pool, q, start, total = _case(dtype, mxfp8, hq, hkv, page, seqs)
    for i, (n, t) in enumerate(seqs):
        if n < 2:
            continue
        for u, what, ch in ((t - 1, "k", 3), (t - n // 2, "v", 77), (t - n // 3 - 1, "v", 5), (t - n + 1, "inf", 120)):
            slot = int(pool.slots[i][u])
            at = (slot // page, i % hkv, slot % page, ch)
            value = float("-inf") if what == "inf" and not mxfp8 else float("nan")
            which = 0 if what == "k" else 1
            pool.cache[which][at] = 0x7f if mxfp8 else value
            (pool.held_k, pool.held_v)[which][at] = value
    hint = max(n for n, _ in seqs)
    out, lse = attend(pool, q, start, total, max_q_len=hint)
    with np.errstate(invalid="ignore"):
        want, want_lse, _, _ = O.paged_attention(f64(q), pool.held_k, pool.held_v, page, pool.table.numpy(), start, total, 128 ** -0.5)
    got, got_lse = f64(out), f64(lse)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want)) and np.array_equal(np.isnan(got_lse), np.isnan(want_lse))
    fine = np.isfinite(want)
    assert fine.any() and not fine.all() and (got[np.isinf(want)] < 0).all()
    assert np.abs(got[fine] - want[fine]).max() <= (2.0 ** -6 if dtype == "bf16" else 1e-5) * np.abs(want[fine]).max()


@pytest.mark.parametrize("mxfp8", [False, True], ids=["plain", "mxfp8"])
@pytest.mark.parametrize("dtype,hq,hkv,page,seqs", [("bf16", 8, 2, 64, [(100, 230), (70, 5000)]), ("bf16", 16, 1, 16, [(40, 200), (33, 33)]), ("bf16", 1, 1, 32, [(700, 1000)]),
                                                     ("bf16", 4, 1, 16, [(4, 600)]), ("fp32", 4, 1, 16, [(40, 300)])])
@pytest.mark.parametrize("spread", [1, 5])
def test_what_is_not_finite_at_any_key(dtype, hq, hkv, page, seqs, mxfp8, spread):
    """Every ``spread``-th key from a little before the new tokens on holds a NaN or an infinity in a channel of its own: a row has one where a key that it sees has it."""
    pool, q, start, total = _case(dtype, mxfp8, hq, hkv, page, seqs)
    for i, (n, t) in enumerate(seqs):
        for u in range(max(0, t - n - 70), t, spread):
            if u % 128 >= 120:                                       # channels that stay finite
                continue
            slot = int(pool.slots[i][u])
            for h in range(hkv):
                at = (slot // page, h, slot % page, u % 128)
                value = float("-inf") if u % 3 == 0 and not mxfp8 else float("nan")
                pool.cache[1][at] = 0x7f if mxfp8 else value
                pool.held_v[at] = value
    out, lse = attend(pool, q, start, total, max_q_len=max(n for n, _ in seqs))
    with np.errstate(invalid="ignore"):
        want, want_lse, _, _ = O.paged_attention(f64(q), pool.held_k, pool.held_v, page, pool.table.numpy(), start, total, 128 ** -0.5)
    got, got_lse = f64(out), f64(lse)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want)) and np.isfinite(got_lse).all()
    fine = np.isfinite(want)
    assert fine.any() and not fine.all()
    assert np.abs(got[fine] - want[fine]).max() <= (2.0 ** -6 if dtype == "bf16" else 1e-5) * np.abs(want[fine]).max()
