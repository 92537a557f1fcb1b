"""A sequence past its prefill: the operators around the paged cache, together, on one Llama3-8B-shaped attention layer.

    python -m paper_2409_12490_amd.continuation [--prompt 16384] [--follow 700] [--steps 16] [--plain]

A prompt's queries and keys get their norms and positions (critiprefill_norm_rope), go through the pruned prefill (estimate, select, block-sparse attention),
and its keys and values into the pages of a cache, in 8 bits unless --plain (critiprefill_cache_write).  A follow-up of some hundred tokens goes on from there
as a chunk, then single tokens: norms, positions and the write in one call (critiprefill_norm_rope_write), then attention over the pages
(critiprefill_paged_attn).  The single step is captured into a graph that follows the lengths on the device.  Prints the time of each part, and how far the
rows of the follow-up and of the captured steps over the cache are from the same rows of dense attention over the keys and values as they were.
"""
from __future__ import annotations

import argparse

import torch

from paper_2409_12490_amd import binding as B

HQ, HKV, D, PAGE = 32, 8, 128, 64
SEGMENT, BLOCK, BUDGET, LOCAL = 512, 64, 32, 1


class Layer:
    """One sequence's cache of one layer, and what its calls need beside the tensors."""

    def __init__(self, longest: int, mxfp8: bool = True, device: str = "cuda", seed: int = 0):
        self.device, self.mxfp8, self.held = device, mxfp8, 0
        pages = -(-longest // PAGE)
        gen = torch.Generator().manual_seed(seed)
        self.cache = B.alloc_cache(pages, HKV, PAGE, mxfp8=mxfp8, device=device)
        self.table = torch.randperm(pages, generator=gen).int().view(1, pages).to(device)          # any pages, in any order
        self.freq = B.rotary_frequencies(D, device=device)
        self.weights = [(1 + 0.1 * torch.randn(D, generator=gen)).bfloat16().to(device) for _ in range(2)]

    def slots(self, first: int, count: int) -> torch.Tensor:
        u = torch.arange(first, first + count, device=self.device)
        return self.table[0, u // PAGE] * PAGE + (u % PAGE).int()

    def prefill(self, qkv: torch.Tensor):
        """qkv [tokens, HQ + 2 HKV, D] as a joint projection writes it.  Returns the output [tokens, HQ, D] and the keys as attention saw them."""
        n = qkv.shape[0]
        q, k, v = qkv.split([HQ, HKV, HKV], 1)
        qr, kr, out = (torch.empty((n, heads, D), dtype=q.dtype, device=self.device) for heads in (HQ, HKV, HQ))
        p = B.make_cache_params(HQ, HKV, q.dtype, q=q, k=k, out=qr, k_out=kr, rotary_dim=D, norm_eps=1e-5)
        pos = torch.arange(n, dtype=torch.int32, device=self.device)
        B.critiprefill_norm_rope(p, q, k, *self.weights, self.freq, pos, qr, kr)
        # the prefill's tensors are [batch, head, token, channel] by strides; values are read with the strides of the keys
        heads = lambda x: x.transpose(0, 1)[None]                                                  # noqa: E731
        vc = v.contiguous()
        a = B.make_params(heads(qr), heads(kr), SEGMENT, BLOCK, BUDGET, LOCAL, out=heads(out))
        scores, (idx, cnt) = B.alloc_scores(a, self.device), B.alloc_lists(a, self.device)
        B.critiprefill_estimate(a, heads(qr), heads(kr), None, scores, B.alloc_workspace(a, self.device))
        B.critiprefill_select(a, scores, idx, cnt)
        B.critiprefill_sparse_attn(a, heads(qr), heads(kr), heads(vc), idx, cnt, heads(out))
        p = B.make_cache_params(HQ, HKV, q.dtype, k=kr, v=v, k_cache=self.cache[0], mxfp8=self.mxfp8)
        B.critiprefill_cache_write(p, kr, v, self.slots(0, n), *self.cache)
        self.held = n
        return out, kr

    def plan(self, qkv: torch.Tensor) -> dict:
        """Buffers and parameters of extend() for as many new tokens as qkv has; kept from step to step."""
        n = qkv.shape[0]
        q, k, v = qkv.split([HQ, HKV, HKV], 1)
        s = {"q": q, "k": k, "v": v, "qr": torch.empty((n, HQ, D), dtype=q.dtype, device=self.device), "out": torch.empty((n, HQ, D), dtype=q.dtype, device=self.device)}
        s["p"] = B.make_cache_params(HQ, HKV, q.dtype, q=q, k=k, v=v, out=s["qr"], k_cache=self.cache[0], mxfp8=self.mxfp8, rotary_dim=D, norm_eps=1e-5)
        s["pa"] = B.make_cache_params(HQ, HKV, q.dtype, q=s["qr"], out=s["out"], k_cache=self.cache[0], mxfp8=self.mxfp8, page_table=self.table, max_q_len=n)
        s["workspace"] = B.alloc_paged_workspace(s["pa"], self.device)
        s["start"] = torch.tensor([0, n], dtype=torch.int32, device=self.device)
        s["pos"], s["slots"], s["kv"] = (torch.zeros(c, dtype=torch.int32, device=self.device) for c in (n, n, 1))
        return s

    def place(self, s: dict) -> None:
        """Where the new tokens of a step go: positions, slots, and the length with them, as tensors that a captured step reads."""
        n = s["pos"].numel()
        s["pos"].copy_(torch.arange(self.held, self.held + n, device=self.device))
        s["slots"].copy_(self.slots(self.held, n))
        s["kv"].fill_(self.held + n)
        self.held += n

    def extend(self, s: dict) -> torch.Tensor:
        """New tokens (one or many) over the cache."""
        B.critiprefill_norm_rope_write(s["p"], s["q"], s["k"], s["v"], *self.weights, self.freq, s["pos"], s["slots"], s["qr"], *self.cache)
        B.critiprefill_paged_attn(s["pa"], s["qr"], *self.cache, self.table, s["start"], s["kv"], s["out"], None, s["workspace"])
        return s["out"]


def _timed(f):
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    f()
    torch.cuda.synchronize()
    a.record()
    r = f()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) * 1e3, r


def decode(layer: Layer, tokens: torch.Tensor):
    """One token after another through a captured step, which reads positions, slots and the length from tensors.  Outputs [steps, HQ, D], and the time of each step in us."""
    token = tokens[:1].clone()
    s = layer.plan(token)
    held = layer.held
    layer.place(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.extend(s)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.extend(s)
    layer.held = held
    outs, us = [], []
    for i in range(tokens.shape[0]):
        token.copy_(tokens[i:i + 1])
        layer.place(s)
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        graph.replay()
        b.record()
        torch.cuda.synchronize()
        us.append(a.elapsed_time(b) * 1e3)
        outs.append(s["out"].clone())
    return torch.cat(outs), us


def _dense_rows(layer: Layer, kr: torch.Tensor, qkv: torch.Tensor, follow: torch.Tensor):
    """The rows of all tokens behind the prompt by dense attention over keys and values that no cache has held."""
    n, m = kr.shape[0], follow.shape[0]
    q, k, v = follow.split([HQ, HKV, HKV], 1)
    qr, kn = torch.empty((m, HQ, D), dtype=q.dtype, device=q.device), torch.empty((m, HKV, D), dtype=q.dtype, device=q.device)
    p = B.make_cache_params(HQ, HKV, q.dtype, q=q, k=k, out=qr, k_out=kn, rotary_dim=D, norm_eps=1e-5)
    B.critiprefill_norm_rope(p, q, k, *layer.weights, layer.freq, torch.arange(n, n + m, dtype=torch.int32, device=q.device), qr, kn)
    keys, values = torch.cat([kr, kn]), torch.cat([qkv[:, HQ + HKV:], v])
    every = torch.zeros((n + m, HQ, D), dtype=q.dtype, device=q.device)
    every[n:] = qr
    heads = lambda x: x.transpose(0, 1)[None]                                                      # noqa: E731
    out = torch.empty_like(every)
    a = B.make_params(heads(every), heads(keys), SEGMENT, BLOCK, BUDGET, LOCAL, out=heads(out))
    B.critiprefill_dense_causal_attn(a, heads(every), heads(keys), heads(values), heads(out))
    return out[n:]


def run(prompt: int = 16384, follow: int = 700, steps: int = 16, mxfp8: bool = True, seed: int = 0, verbose: bool = True) -> dict:
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def projected(n):
        x = torch.randn((n, HQ + 2 * HKV, D), generator=gen, device="cuda")
        return (x + 0.1 * torch.randn((n, HQ + 2 * HKV, D), generator=gen, device="cuda").cumsum(0)).bfloat16()

    layer = Layer(prompt + follow + steps + 1, mxfp8, seed=seed)
    qkv, more = projected(prompt), projected(follow)
    prefill_us, (_, kr) = _timed(lambda: layer.prefill(qkv))

    s = layer.plan(more)
    layer.place(s)
    chunk_us, out = _timed(lambda: layer.extend(s))

    tokens = torch.cat([projected(1) for _ in range(steps)])
    outs, step_us = decode(layer, tokens)
    dense = _dense_rows(layer, kr, qkv, torch.cat([more, tokens])).float()
    off = float((out.float() - dense[:follow]).norm() / dense[:follow].norm())
    step_off = ((outs.float() - dense[follow:]).flatten(1).norm(dim=1) / dense[follow:].flatten(1).norm(dim=1)).tolist()
    found = {"prefill_us": prefill_us, "chunk_us": chunk_us, "step_us": sorted(step_us)[steps // 2], "off": off, "step_off": step_off, "held": layer.held,
             "finite": bool(torch.isfinite(outs).all() and torch.isfinite(out).all())}
    if verbose:
        print(f"prompt of {prompt}: norms, positions, pruned prefill and cache {prefill_us:.0f} us")
        print(f"follow-up of {follow} over the cache ({'8 bits' if mxfp8 else 'bf16'}): {chunk_us:.0f} us, {off:.2e} from dense attention over what was cached")
        print(f"single tokens, captured: {found['step_us']:.1f} us each, {max(step_off):.2e} at most from dense attention; {layer.held} tokens held")
    return found


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--prompt", type=int, default=16384)
    ap.add_argument("--follow", type=int, default=700)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--plain", action="store_true", help="pages of bf16")
    args = ap.parse_args()
    run(args.prompt, args.follow, args.steps, not args.plain)
