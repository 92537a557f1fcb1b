"""Pages of 4 bits whose values are NaN for some rows of a tile alone, where a workgroup goes from one unit of work to the next: what it does for the one must not reach the other."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from tests.cache4_helpers import Pool4, attend4
from tests.cache_helpers import DEV, HALF_STEP, f64, randn, route
from tests.test_gpu_paged import _starts
from tests.test_gpu_paged4 import few_of

pytestmark = pytest.mark.gpu


def _spoiled(dtype, hq, hkv, page, seqs):
    """seqs: (new tokens, tokens in all).  Every third sequence of two new tokens and more has NaN in V of its second and its last new token, 32 channels each, every ninth in K of its last too."""
    gen = torch.Generator().manual_seed(len(seqs) + hq)
    new, total = zip(*seqs)
    pool = Pool4(gen, total, hkv, page, dtype)
    for i, (n, t) in enumerate(seqs):
        if i % 3 or n < 2:
            continue
        for u, which, block in ((t - n + 1, 1, i % 4), (t - 1, 1, (i + 2) % 4), (t - 1, 0, 1))[:3 if i % 9 == 0 else 2]:
            slot = int(pool.slots[i][u])
            for h in range(hkv):
                pool.spoil(which, slot // page, h, slot % page, block)
    return pool, randn(gen, sum(new), hq, 128, dtype=dtype).to(DEV), _starts(new), list(total)


def _check(pool, q, start, total, out, lse):
    """NaN where fp64 has it, and only there; the rest within the bound of cache_helpers.check_attention, whose reasons stand there."""
    with np.errstate(invalid="ignore"):
        want, want_lse, size, logit = O.paged_attention(f64(q), pool.held_k, pool.held_v, pool.page, pool.table.numpy(), start, total, 128 ** -0.5)
    got, got_lse = f64(out), f64(lse)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isnan(got_lse), np.isnan(want_lse))
    fine, fine_lse = np.isfinite(want), np.isfinite(want_lse)
    assert fine.any() and not fine.all() and fine_lse.any() and not fine_lse.all()
    delta = 2.0 ** -20 * (logit + np.maximum(np.abs(np.where(fine_lse, want_lse, 0.0)), 1.0)) + 2.0 ** -20
    rounding = HALF_STEP["bf16"] * size * (pool.dtype == "bf16") + HALF_STEP[pool.dtype] * np.abs(want)
    with np.errstate(invalid="ignore"):
        bound = rounding * 1.01 + 4 * delta[..., None] * size.max(-1, keepdims=True) + 1e-30
        worst = (np.abs(got - want) / bound)[fine].max()
    assert worst <= 1.0, f"out: {worst:.2f} of the bound"
    worst = (np.abs(got_lse - want_lse) / (2 * delta))[fine_lse].max()
    assert worst <= 1.0, f"lse: {worst:.2f} of the bound"


# Two to four new tokens each, with lengths of one to four steps; tiles of 16 and of 32 rows, of 64 in fp32.  dtype, heads, page, sequences.
FEW = [("bf16", 8, 2, 16, 900), ("bf16", 4, 2, 64, 700), ("bf16", 16, 2, 32, 700), ("fp32", 4, 2, 16, 700), ("fp32", 17, 1, 32, 600), ("fp32", 40, 1, 16, 500)]


@pytest.mark.parametrize("keys", [400, 3000])
@pytest.mark.parametrize("dtype,hq,hkv,page,n", FEW)
def test_few_tokens_each(dtype, hq, hkv, page, n, keys):
    seqs = [(2 + i % 3, (5, 129, 60, 130, 257, 384, 17, 4)[i % 8] + i // 300) for i in range(n)]
    r = route(dtype, 2, hq, hkv, n, 4, keys)
    assert not r.chunk and r.whole == (keys == 400) and n * hkv > r.workgroups
    pool, q, start, total = _spoiled(dtype, hq, hkv, page, seqs)
    _check(pool, q, start, total, *attend4(pool, q, start, total, max_q_len=4, max_kv_len=keys))


# Tiles of 256 rows: of different lengths, and all alike, which are dealt out in rounds.
CHUNKS = [(32, 8, 64, [(66 + 13 * i % 70, 100 + 17 * i) for i in range(40)]), (32, 8, 16, [(90, 300)] * 45), (16, 4, 32, [(70 + i % 60, 200 + i) for i in range(75)])]


@pytest.mark.parametrize("keys", [700, 3000])
@pytest.mark.parametrize("hq,hkv,page,seqs", CHUNKS)
def test_chunks(hq, hkv, page, seqs, keys):
    longest = max(n for n, _ in seqs)
    r = route("bf16", 2, hq, hkv, len(seqs), longest, keys)
    units = hkv * sum(-(-n // (1 << r.tile_shift)) for n, _ in seqs)
    assert r.chunk and r.whole == (keys == 700) and units > r.workgroups
    pool, q, start, total = _spoiled("bf16", hq, hkv, page, [(n, max(n, t)) for n, t in seqs])
    _check(pool, q, start, total, *attend4(pool, q, start, total, max_q_len=longest, max_kv_len=keys))


def test_few_tokens_beside_a_chunk():
    """Both kernels, and in each sequences behind spoiled ones."""
    seqs = [(1 + i % 4, 900 + 7 * i) for i in range(60)] + [(200, 900), (30, 700), (90, 650), (300, 1000), (2, 300)]
    seqs = seqs[-5:-1] + seqs[:-5] + seqs[-1:]
    assert few_of((32, 8, 64, seqs, 4)) == 4
    pool, q, start, total = _spoiled("bf16", 32, 8, 64, seqs)
    _check(pool, q, start, total, *attend4(pool, q, start, total, max_q_len=300))
