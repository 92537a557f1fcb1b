"""Shared plumbing of the tests of the cache operators: pools, page tables, calls through the binding.  No arithmetic of the operators lives here."""
from __future__ import annotations

import ctypes
import functools
import os
import shutil
import subprocess
import tempfile

import numpy as np
import torch

from oracle import cache_oracle as O
from paper_2409_12490_amd import binding as B

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def f64(t):
    return t.detach().to("cpu").to(torch.float64).numpy()


def randn(gen, *shape, dtype="bf16", scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(DTYPES[dtype])


def side_by_side(gen, tokens, heads, dtype, extra=0, scale=1.0):
    """Tensors [tokens, h, 128] for h in heads that lie in one [tokens, sum(heads) + extra, 128], on the GPU."""
    wide = randn(gen, tokens, sum(heads) + extra, 128, dtype=dtype, scale=scale).to(DEV)
    return wide.split(list(heads) + [extra], 1)[:len(heads)]


class Pool:
    """Pages for sequences of given lengths, in random order, everything that no token lies in filled with NaN."""

    def __init__(self, gen, lengths, hkv, page, dtype="bf16", mxfp8=False, spare=3, scale=1.0):
        self.page, self.mxfp8, self.hkv, self.dtype = page, mxfp8, hkv, dtype
        counts = [-(-n // page) for n in lengths]
        self.n_pages = sum(counts) + spare
        order = torch.randperm(self.n_pages, generator=gen)
        self.table = torch.full((len(lengths), max(counts + [1]) + 1), 0, dtype=torch.int32)
        self.table[:] = torch.tensor([-1, 2 ** 30, -2 ** 31])[torch.arange(self.table.shape[1]) % 3].int()    # what no token lies in may be anything
        at = 0
        for i, c in enumerate(counts):
            self.table[i, :c] = order[at:at + c].int()
            at += c
        self.slots = [(self.table[i, torch.arange(n) // page] * page + torch.arange(n) % page).int() for i, n in enumerate(lengths)]
        shape = (self.n_pages, hkv, page, 128)
        self.k, self.v = randn(gen, *shape, dtype=dtype, scale=scale), randn(gen, *shape, dtype=dtype)
        used = torch.zeros(self.n_pages * page, dtype=torch.bool)
        for s in self.slots:
            used[s.long()] = True
        used = used.view(self.n_pages, 1, page, 1)
        if mxfp8:
            (kc, ks), (vc, vs) = (O.mx_quantise(f64(x)) for x in (self.k, self.v))
            fill = lambda x, w: torch.where(used, torch.from_numpy(x), torch.tensor(w, dtype=torch.uint8))   # noqa: E731
            self.held_k, self.held_v = (torch.where(used, torch.from_numpy(O.mx_values(c, s)), float("nan")).numpy() for c, s in ((kc, ks), (vc, vs)))
            self.cache = [fill(kc, 0x7f).to(DEV), fill(vc, 0xff).to(DEV), fill(ks, 0xff).to(DEV), fill(vs, 0xff).to(DEV)]
        else:
            k, v = (x.masked_fill(~used, float("nan")) for x in (self.k, self.v))
            self.held_k, self.held_v = f64(k), f64(v)
            self.cache = [k.to(DEV), v.to(DEV), None, None]


def attend(pool, q, q_start, kv_len, table=None, max_q_len=0, out=None, scale=0.0, workspace=None, max_kv_len=0):
    table = (pool.table if table is None else table).to(DEV)
    out = torch.full((q.shape[0], q.shape[1], 128), float("nan"), dtype=q.dtype, device=DEV) if out is None else out
    lse = torch.full(q.shape[:2], float("nan"), device=DEV)
    p = B.make_cache_params(q.shape[1], pool.hkv, q.dtype, q=q, out=out, k_cache=pool.cache[0], mxfp8=pool.mxfp8, page_table=table, max_q_len=max_q_len,
                            max_kv_len=max_kv_len, attn_scale=scale)
    ws = B.alloc_paged_workspace(p) if workspace is None else workspace
    ws.fill_(0xff)                                                   # whatever it holds
    start, lens = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (q_start, kv_len))
    B.critiprefill_paged_attn(p, q, *pool.cache, table, start, lens, out, lse, ws)
    torch.cuda.synchronize()
    return out, lse


def check_attention(pool, q, q_start, kv_len, out, lse, table=None, scale=128 ** -0.5):
    """Against fp64.  A logit's error: each product and sum in fp32, 2^-24 of its terms a rounding, fewer than 16 deep, and as much again for scaling and
    exp2; out: twice that times the largest |v| for each of numerator and denominator, the rounding of P to bf16 (not fp32), sums of
    fp32, and its own rounding."""
    table = pool.table if table is None else table
    dtype = pool.dtype
    want, want_lse, size, logit = O.paged_attention(f64(q), pool.held_k, pool.held_v, pool.page, table.numpy(), q_start, kv_len, scale)
    delta = 2.0 ** -20 * (logit + np.maximum(np.abs(np.where(np.isfinite(want_lse), want_lse, 0.0)), 1.0)) + 2.0 ** -20
    got, got_lse = f64(out), f64(lse)
    rounding = HALF_STEP["bf16"] * size * (dtype == "bf16") + HALF_STEP[dtype] * np.abs(want)
    bound = rounding * 1.01 + 4 * delta[..., None] * size.max(-1, keepdims=True) + 1e-30
    assert np.isfinite(got).all(), f"{(~np.isfinite(got)).sum()} values are not finite"
    worst = np.max(np.abs(got - want) / bound) if got.size else 0.0
    assert worst <= 1.0, f"out: {worst:.2f} of the bound, at {np.unravel_index(np.argmax(np.abs(got - want) / bound), got.shape)}"
    empty = ~np.isfinite(want_lse)
    assert (got_lse[empty] == -np.inf).all() and (got[empty] == 0).all()
    err = np.abs(np.where(empty, 0.0, got_lse) - np.where(empty, 0.0, want_lse))
    assert (err <= 2 * delta).all(), f"lse: {np.max(err / delta) / 2:.2f} of the bound"


class Shape(ctypes.Structure):                   # cp::CacheShape of csrc/cache.h
    _fields_ = ([(x, ctypes.c_int) for x in ("hq", "hkv", "group", "dtype", "mxfp8", "page", "page_shift", "n_pages", "tokens", "n_seqs", "max_pages", "max_q")]
                + [("max_kv", ctypes.c_longlong)] + [(x, ctypes.c_int) for x in ("rotary", "interleaved")] + [(x, ctypes.c_float) for x in ("eps", "scale")]
                + [(x, ctypes.c_int64 * 2) for x in ("qs", "ks", "vs", "os", "kos")])


class Route(ctypes.Structure):                   # cp::PagedRoute of csrc/cache.h
    _fields_ = [(x, ctypes.c_int) for x in ("chunk", "rows", "tile_shift", "step_shift", "workgroups", "least", "setup", "whole")]


def streams(dtype, mxfp8, tokens, rows, held):
    """Whether the library takes a call past the caches: its own rule."""
    f = B.load()._ZN2cp18cache_call_streamsERKNS_10CacheShapeEii
    f.argtypes, f.restype = [ctypes.POINTER(Shape), ctypes.c_int, ctypes.c_int], ctypes.c_bool
    return f(Shape(dtype=int(dtype == "bf16"), mxfp8=int(mxfp8), tokens=tokens), rows, held)


def route(dtype, mxfp8, hq, hkv, seqs, max_q, max_kv):
    """Which kernel attention over pages takes, and how it cuts the work, as far as the host decides: its own rule."""
    f = B.load()._ZN2cp11paged_routeERKNS_10CacheShapeE
    f.argtypes, f.restype = [ctypes.POINTER(Shape)], Route
    return f(Shape(dtype=int(dtype == "bf16"), mxfp8=int(mxfp8), hq=hq, hkv=hkv, group=hq // hkv, n_seqs=seqs, max_q=max_q, max_kv=max_kv))


# How the kernel of 256-row tiles deals its units out, from the header that it takes its rules from; what is written out here is the sum over sequences, units in order.
_DEALING = """
#define __host__
#define __device__
#define __forceinline__ inline
#include "paged_steps.h"
extern "C" void dealing(int n, const int* tokens, const int* keys, int hkv, int tile_shift, int step_shift, unsigned workgroups, unsigned least, unsigned setup, int mxfp8, unsigned* found) {
    unsigned units = 0, total = 0, longest = 0, first = 0, last = 0;
    bool alike = n <= 64;
    for (int i = 0; i < n; ++i) {
        const cp::TileSteps t(tokens[i], keys[i], step_shift);
        const unsigned tiles = (tokens[i] + (1u << tile_shift) - 1) >> tile_shift;
        if (tiles == 0) { alike = false; continue; }
        first = t.of(0, tile_shift, step_shift); last = t.of(tiles - 1, tile_shift, step_shift);
        units += tiles * hkv; total += (tiles * setup + t.before(tiles, tile_shift, step_shift)) * hkv;
        if (setup + last > longest) longest = setup + last;
        alike = alike && tokens[i] == tokens[0] && keys[i] == keys[0];
    }
    unsigned rounds = alike && units >= workgroups ? cp::whole_rounds(units, workgroups, first, last) : 0;
    if (rounds) {                                                  // all are as the first
        const cp::TileSteps t(tokens[0], keys[0], step_shift);
        const unsigned tiles = (tokens[0] + (1u << tile_shift) - 1) >> tile_shift, cut = rounds * workgroups, heads = cut / tiles, rest = cut - heads * tiles;
        total -= heads * (tiles * setup + t.before(tiles, tile_shift, step_shift)) + rest * setup + t.before(rest, tile_shift, step_shift);
    }
    unsigned share = (total + workgroups - 1) / workgroups;
    if (share < least) share = least;
    const unsigned used = (total + share - 1) / share, over = units - rounds * workgroups, turns = (over + workgroups - 1) / workgroups;
    const bool uncut = total && cp::uncut_pays(turns, longest, used, share, mxfp8);
    found[0] = units; found[1] = rounds; found[2] = over; found[3] = uncut; found[4] = turns; found[5] = used; found[6] = share;
}
"""


@functools.lru_cache(maxsize=None)
def _dealing_library():
    compiler = shutil.which("g++") or shutil.which("clang++") or shutil.which("c++")
    assert compiler, "no C++ compiler"
    csrc = os.path.join(os.path.dirname(os.path.abspath(B.__file__)), "csrc")
    with tempfile.TemporaryDirectory() as where:
        with open(os.path.join(where, "f.cpp"), "w") as f:
            f.write(_DEALING)
        subprocess.run([compiler, "-O1", "-std=c++17", "-shared", "-fPIC", "-I", csrc, os.path.join(where, "f.cpp"), "-o", os.path.join(where, "f.so")], check=True)
        return ctypes.CDLL(os.path.join(where, "f.so"))


def dealing(dtype, mxfp8, hq, hkv, seqs, max_kv, max_q=None):
    """How the units of sequences (new tokens, tokens in all) are dealt: "rows" (the kernel whose waves split the keys), or of the other "host" (not cut, the host says so), "whole" (not cut,
    as the lengths turn out), "cut", or rounds and "+ nothing", "+ cut", "+ whole" for what they leave over."""
    r = route(dtype, mxfp8, hq, hkv, len(seqs), max_q or max(n for n, _ in seqs), max_kv)
    if not r.chunk:
        return "rows"
    if r.whole:
        return "host"
    found = (ctypes.c_uint * 7)()
    array = ctypes.c_int * len(seqs)
    _dealing_library().dealing(len(seqs), array(*[n for n, _ in seqs]), array(*[k for _, k in seqs]), hkv, r.tile_shift, r.step_shift, r.workgroups, r.least, r.setup,
                               int(mxfp8), found)
    _, rounds, over, uncut, turns, _, _ = found
    if not rounds:
        return "whole" if uncut else "cut"
    return f"{rounds} + " + ("nothing" if not over else f"{turns} whole" if uncut else "cut")
