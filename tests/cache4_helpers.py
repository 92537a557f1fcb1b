"""The plumbing of cache_helpers.py for pages of 4 bits."""
from __future__ import annotations

import torch

from oracle import cache_oracle as O
from paper_2409_12490_amd import binding as B
from tests.cache_helpers import DEV, Pool, f64


class Pool4(Pool):
    """A Pool whose pages hold 4 bits: what no token lies in has any elements, and scales under which these are infinite or NaN."""

    def __init__(self, gen, lengths, hkv, page, dtype="bf16", spare=3, scale=1.0):
        super().__init__(gen, lengths, hkv, page, dtype, False, spare, scale)
        used = torch.zeros(self.n_pages * page, dtype=torch.bool)
        for s in self.slots:
            used[s.long()] = True
        used = used.view(self.n_pages, 1, page, 1)
        (kc, ks), (vc, vs) = (O.mx4_quantise(f64(x)) for x in (self.k, self.v))
        fill = lambda x, w: torch.where(used, torch.from_numpy(x), torch.tensor(w, dtype=torch.uint8))   # noqa: E731
        self.held_k, self.held_v = (torch.where(used, torch.from_numpy(O.mx4_values(c, s)), float("nan")).numpy() for c, s in ((kc, ks), (vc, vs)))
        far = torch.randint(253, 256, (2, *ks.shape), generator=gen, dtype=torch.uint8)
        self.cache = [fill(kc, 0x7a).to(DEV), fill(vc, 0xf1).to(DEV)] + [torch.where(used, torch.from_numpy(s), f).to(DEV) for s, f in zip((ks, vs), far)]

    def spoil(self, which, page, head, offset, block):
        """32 channels of a token's K (0) or V (1) become NaN."""
        self.cache[2 + which][page, head, offset, block] = 0xff
        (self.held_k, self.held_v)[which][page, head, offset, 32 * block:32 * block + 32] = float("nan")


def attend4(pool, q, q_start, kv_len, table=None, max_q_len=0, out=None, scale=0.0, max_kv_len=0):
    table = (pool.table if table is None else table).to(DEV)
    out = torch.full((q.shape[0], q.shape[1], 128), float("nan"), dtype=q.dtype, device=DEV) if out is None else out
    lse = torch.full(q.shape[:2], float("nan"), device=DEV)
    p = B.make_cache_params(q.shape[1], pool.hkv, q.dtype, q=q, out=out, k_cache=pool.cache[0], mxfp4=True, page_table=table, max_q_len=max_q_len,
                            max_kv_len=max_kv_len, attn_scale=scale)
    ws = B.alloc_paged_workspace(p)
    ws.fill_(0xff)                                                   # whatever it holds
    start, lens = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (q_start, kv_len))
    B.critiprefill_paged_attn(p, q, *pool.cache, table, start, lens, out, lse, ws)
    torch.cuda.synchronize()
    return out, lse
