"""The kernel of 256-row tiles deals its units out in seven ways, by lengths that the device sees: each is reached here, which the library's own rules say of each case, and compared with fp64.

Beside each case: heads, page, (new tokens, tokens in all) of the sequences, and how they are dealt over plain and over 8-bit pages, see cache_helpers.dealing."""
import numpy as np
import pytest
import torch

from tests.cache_helpers import DEV, HALF_STEP, Pool, attend, dealing, randn

pytestmark = pytest.mark.gpu

CASES = [
    # rounds of whole units that leave nothing: several sequences and heads, one head, sequences as many as a wave has lanes, odd numbers of rounds
    (32, 8, 64, [(512, 812)] * 8, "2 + nothing"), (64, 1, 64, [(512, 812)] * 8, "4 + nothing"), (64, 8, 64, [(40, 900)] * 64, "4 + nothing"),
    (64, 4, 32, [(16, 1000)] * 64, "1 + nothing"), (64, 4, 16, [(48, 1000)] * 64, "3 + nothing"),
    # rounds, and what they leave over cut: what is skipped spans heads and sequences, or ends inside the only one
    (28, 4, 64, [(400, 900)] * 10, "2 + cut"), (28, 4, 32, [(512, 812)] * 17, "4 + cut"), (28, 4, 16, [(100, 1300)] * 17, "1 + cut"), (16, 2, 16, [(512, 812)] * 17, "2 + cut"),
    (64, 1, 32, [(3100, 3311)], "2 + cut"),
    # rounds, and a last one or two that are not full
    (32, 8, 16, [(130, 1300)] * 17, "1 + 1 whole"), (28, 4, 64, [(257, 900)] * 17, "2 + 1 whole"), (32, 8, 64, [(400, 900)] * 17, "2 + 2 whole"),
    # none, as the lengths turn out: alike, one sequence, ragged, empty ones among more than a wave has lanes
    (32, 8, 32, [(130, 900)] * 4, "whole"), (64, 4, 16, [(700, 1500)], "whole"), (32, 8, 64, [(200 + 37 * i, 820 + 50 * i) for i in range(5)], "whole"),
    (64, 8, 64, [(40, 900) if i % 5 else (0, 0) for i in range(70)], "whole"),
    # none, the host says so
    (32, 8, 64, [(300, 600)] * 4, "host"),
    # all cut: a long one among short ones, more sequences than a wave has lanes, alike
    (32, 8, 64, [(70, 4000), (300, 900), (0, 0), (1, 1700)], "cut"), (16, 4, 16, [(130, 1300)] * 70, "cut"), (16, 4, 64, [(460, 1100)] * 10, "cut"), (32, 8, 16, [(2049, 2300)], "cut"),
]


def _width(seqs, page):
    return max(-(-t // page) for _, t in seqs) + 1                  # of Pool's page table


def route_of(case, mxfp8):
    hq, hkv, page, seqs, _ = case
    return dealing("bf16", mxfp8, hq, hkv, seqs, _width(seqs, page) * page)


def _plain(pool, q, start, total, scale):
    """fp64 on the GPU: out, lse, sum_u p_u |v_u|, and the largest sum_c |q_c k_c| scale of each row."""
    T, hq, d = q.shape
    hkv, group = pool.hkv, hq // pool.hkv
    held = [torch.from_numpy(x).to(DEV).transpose(1, 2).flatten(0, 1) for x in (pool.held_k, pool.held_v)]      # [slots, kv heads, channels]
    out, size = (torch.zeros((T, hq, d), dtype=torch.float64, device=DEV) for _ in range(2))
    lse, logit = (torch.zeros((T, hq), dtype=torch.float64, device=DEV) for _ in range(2))
    for i, keys in enumerate(total):
        n, u = start[i + 1] - start[i], torch.arange(keys, device=DEV)
        if n == 0:
            continue
        see = u <= (keys - n + torch.arange(n, device=DEV))[:, None, None]
        for h in range(hkv):
            k, v = (x[pool.slots[i].to(DEV).long(), h] for x in held)
            x = q[start[i]:start[i + 1], h * group:(h + 1) * group].double()
            z = (x.reshape(-1, d) @ k.t().contiguous() * scale).view(n, group, keys).masked_fill_(~see, -np.inf)
            at = (slice(start[i], start[i + 1]), slice(h * group, (h + 1) * group))
            lse[at] = z.logsumexp(-1)
            p = (z - lse[at][..., None]).exp_().view(-1, keys)
            out[at], size[at] = (p @ v).view(n, group, d), (p @ v.abs()).view(n, group, d)
            logit[at] = (x.abs().reshape(-1, d) @ k.abs().t().contiguous() * scale).amax(-1).view(n, group)
    return out, lse, size, logit


@pytest.mark.parametrize("mxfp8", [False, True], ids=["plain", "mxfp8"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}x{len(c[3])}x{c[3][0][0]}x{c[3][0][1]}")
def test_dealt_units(case, mxfp8):
    hq, hkv, page, seqs, path = case
    assert route_of(case, mxfp8) == path
    gen = torch.Generator().manual_seed(len(seqs) + hq)
    new, total = zip(*seqs)
    pool = Pool(gen, total, hkv, page, "bf16", mxfp8)
    assert pool.table.shape[1] == _width(seqs, page)
    q, start = randn(gen, sum(new), hq, 128).to(DEV), np.concatenate([[0], np.cumsum(new)]).astype(int).tolist()
    out, lse = attend(pool, q, start, total, max_q_len=max(new))
    want, want_lse, size, logit = _plain(pool, q, start, total, 128 ** -0.5)
    # the bound of cache_helpers.check_attention
    delta = 2.0 ** -20 * (logit + want_lse.abs().clamp(min=1.0)) + 2.0 ** -20
    bound = HALF_STEP["bf16"] * (size + want.abs()) * 1.01 + 4 * delta[..., None] * size.amax(-1, keepdim=True) + 1e-30
    worst = float(((out.double() - want).abs() / bound).max())
    assert torch.isfinite(out).all() and worst <= 1.0, f"out: {worst:.2f} of the bound"
    assert ((lse.double() - want_lse).abs() <= 2 * delta).all()
