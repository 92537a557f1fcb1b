"""The operators around a prefill that keep a sequence going, as cases that can be timed and checked one by one.

``rope``        norms of queries and keys for each head with the position rotation, as tensors (what estimate and attention take)
``rope_write``  the same with keys and values going straight into the pages of a cache (what a decode step does)
``write``       keys and values of a finished prefill into the pages
``read``        and back, as tensors
``attn``        attention of each sequence's new tokens (one: decode; many: a follow-up chunk) over its pages

Cache formats: ``plain``, the elements as they are; ``mxfp8``, e4m3 elements with one power of two for each 32 channels.  8-bit values are
returned in their own types (e4m3 elements in units of their block's scale, and the scales).
"""
import random

import torch

own = False

D = 128
DEV = "cuda"
BASE = 500000.0                                    # of the rotation
EPS = 1e-5
SCALE = D ** -0.5
NEAREST, FURTHEST = 1, 254                         # biased exponents that a scale may have


def _rope(name, op, dtype, hq, hkv, tokens, start, page=64, fmt="plain", rotary=128, interleaved=False, norm=True, fused=True):
    return {"name": name, "op": op, "dtype": dtype, "hq": hq, "hkv": hkv, "tokens": tokens, "start": start, "page": page, "fmt": fmt, "rotary": rotary,
            "interleaved": interleaved, "norm": norm, "fused": fused}


def _cache(name, op, dtype, hq, hkv, tokens, page, fmt, fused=True):
    return {"name": name, "op": op, "dtype": dtype, "hq": hq, "hkv": hkv, "tokens": tokens, "page": page, "fmt": fmt, "fused": fused}


def _attn(name, dtype, fmt, hq, hkv, seqs, new, past, page, lengths=0, ragged=False, lse=False, fused=False):
    """``new`` tokens of each sequence over ``past`` tokens and themselves; ragged: up to these, by the number ``lengths``."""
    return {"name": name, "op": "attn", "dtype": dtype, "fmt": fmt, "hq": hq, "hkv": hkv, "seqs": seqs, "new": new, "past": past, "page": page,
            "lengths": lengths, "ragged": ragged, "lse": lse, "fused": fused}


def listed():
    return [
        # a 16K prompt on its way into the pruned prefill: Q and K as the projection leaves them, side by side
        _rope("rope_bf16_16384", "rope", "bf16", 32, 8, 16384, 0),
        # one decode step of 64 sequences, into an 8-bit cache
        _rope("rope_write_mxfp8_64", "rope_write", "bf16", 32, 8, 64, -1, fmt="mxfp8"),
        # the fp32 path, odd length, half of the channels rotated in neighbouring pairs, far positions
        _rope("rope_write_fp32_2777", "rope_write", "fp32", 8, 2, 2777, 100000, page=16, rotary=64, interleaved=True, fused=False),
        # a 64K prompt goes into an 8-bit cache
        _cache("write_mxfp8_65536", "write", "bf16", 32, 8, 65536, 64, "mxfp8"),
        # a prefix comes back for a prefill that goes on from it
        _cache("read_mxfp8_20001", "read", "bf16", 32, 4, 20001, 32, "mxfp8", fused=False),
        # the smallest decode: one sequence with a short past
        _attn("decode_bf16_1x2000", "bf16", "plain", 32, 8, 1, 1, 1999, 64),
        # one sequence at the length of the headline
        _attn("decode_bf16_1x131072", "bf16", "plain", 32, 8, 1, 1, 131071, 64),
        # a batch of decoding sequences of all lengths over an 8-bit cache
        _attn("decode_mxfp8_48", "bf16", "mxfp8", 32, 8, 48, 1, 32768, 64, lengths=3, ragged=True, lse=True),
        # short follow-ups and single tokens in one batch, Yi-9B-shaped
        _attn("mixed_mxfp8_12", "bf16", "mxfp8", 32, 4, 12, 300, 12000, 32, lengths=5, ragged=True),
        # fp32: the reference that a bf16 result is compared with
        _attn("chunk_fp32_3x200", "fp32", "plain", 4, 2, 3, 200, 3000, 16, lengths=2, ragged=True, lse=True),
        # a follow-up question after a 16K prompt
        _attn("chunk_bf16_512_16384", "bf16", "plain", 32, 8, 1, 512, 16384, 64, fused=True),
        # the last quarter of a 32K prompt that comes in chunks
        _attn("chunk_bf16_8192_32768", "bf16", "plain", 32, 8, 1, 8192, 24576, 64, lse=True),
    ]


def _spread(rng, low, high):
    return int(low * (high / low) ** rng.random())


def draw(rng):
    while True:
        op = rng.choice(["rope", "rope_write", "rope_write", "write", "read", "attn", "attn", "attn", "attn", "attn"])
        fp32 = rng.random() < 0.2
        dtype = "fp32" if fp32 else "bf16"
        hq, hkv = rng.choice([(4, 2), (8, 2), (3, 3), (1, 1)] if fp32 else [(32, 8), (32, 8), (32, 4), (8, 2), (4, 4), (28, 4), (40, 8), (2, 1)])
        page, fmt = rng.choice([16, 32, 64, 64, 128]), rng.choice(["plain", "mxfp8"])
        if op == "attn":
            kind = rng.choice(["decode", "decode", "few", "chunk", "chunk"])
            new = {"decode": 1, "few": rng.randint(2, 16), "chunk": _spread(rng, 17, 512 if fp32 else 8192)}[kind]
            past = _spread(rng, 1, 8192 if fp32 else 131072) - 1
            seqs = _spread(rng, 1, 64)
            case = _attn("", dtype, fmt, hq, hkv, seqs, new, past, page, rng.randint(1, 1 << 20), rng.random() < 0.7, rng.random() < 0.4, rng.random() < 0.5)
            _, ends = _lengths(case)
            padded = seqs * hq * new * max(ends)                    # what the plain form lays out
            if padded > 2 ** 31 or seqs * hkv * max(ends) > 2 ** 23 or work(case)["flops"] > (3e11 if fp32 else 4e12):
                continue
        elif op in ("rope", "rope_write"):
            case = _rope("", op, dtype, hq, hkv, _spread(rng, 1, 16384), rng.choice([-1, 0, _spread(rng, 1, 1 << 20)]), page, fmt if op == "rope_write" else "plain",
                         rng.choice([128, 128, 64, 32]), rng.random() < 0.3, rng.random() < 0.7, rng.random() < 0.6)
        else:
            case = _cache("", op, dtype, hq, hkv, _spread(rng, 1, 65536), page, fmt, rng.random() < 0.6)
        del case["name"]
        return case


def _lengths(case):
    """New tokens of each sequence, and where each ends (its past and its new tokens)."""
    rng = random.Random(case["lengths"])
    new, ends = [], []
    for i in range(case["seqs"]):
        n, past = case["new"], case["past"]
        if case["ragged"] and i:                                   # the first has them in full
            n, past = (_spread(rng, 1, n) if n > 1 else 1), _spread(rng, 1, past + 1) - 1
        new.append(n)
        ends.append(n + past)
    return new, ends


def _size(case):
    return 2 if case["dtype"] == "bf16" else 4


def _row(case):
    """Bytes of a token's K or V of one head in the cache."""
    return D + 4 if case["fmt"] == "mxfp8" else D * _size(case)


def work(case):
    e, hq, hkv = _size(case), case["hq"], case["hkv"]
    if case["op"] == "attn":
        new, ends = _lengths(case)
        total = sum(new)
        pairs = sum(n * (e_ - n) + n * (n + 1) // 2 for n, e_ in zip(new, ends))
        size = 2 * total * hq * D * e + sum(ends) * hkv * 2 * _row(case) + (total * hq * 4 if case["lse"] else 0)
        return {"bytes": size, "flops": 4 * D * hq * pairs}
    t = case["tokens"]
    if case["op"] == "rope":
        return {"bytes": 2 * t * (hq + hkv) * D * e + 4 * t, "flops": 10 * t * (hq + hkv) * D}
    if case["op"] == "rope_write":
        return {"bytes": t * (2 * hq + 2 * hkv) * D * e + t * hkv * 2 * _row(case) + 8 * t, "flops": 10 * t * (hq + hkv) * D}
    return {"bytes": t * hkv * 2 * (D * e + _row(case)) + 4 * t, "flops": 2 * t * hkv * 2 * D}


# ---- the cache's 8-bit format ---------------------------------------------------------------------------------------
def _exponents(x):
    """Biased exponents [..., 4] of the smallest powers of two that bring a block of 32 channels within e4m3's 448."""
    most = x.abs().unflatten(-1, (4, 32)).amax(-1)
    m, e = torch.frexp(most)                                       # most = 2 m 2^(e - 1), and 448 = 1.75 * 2^8
    return torch.where(most == 0, NEAREST, e + 118 + (m > 0.875).int()).clamp(NEAREST, FURTHEST)


def _in_units(x):
    """x in units of its blocks' scales, and the scales' bytes."""
    e = _exponents(x)
    return torch.ldexp(x.unflatten(-1, (4, 32)), (127 - e).unsqueeze(-1)).flatten(-2), e.to(torch.uint8)


def _quantise(x):
    units, e = _in_units(x)
    return units.to(torch.float8_e4m3fn).view(torch.uint8), e


def _values(elements, e):
    x = elements.view(torch.float8_e4m3fn).float().unflatten(-1, (4, 32))
    return torch.ldexp(x, (e.int() - 127).unsqueeze(-1)).flatten(-2)


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _walk(gen, tokens, heads):
    """Neighbouring tokens are alike, as in a text: a random walk and noise, scaled to unit variance."""
    x = torch.randn((tokens, heads, D), generator=gen, device=DEV).mul_(0.1).cumsum(0)
    x += torch.randn((tokens, heads, D), generator=gen, device=DEV)
    return x.div_(x.std() + 1e-6)


def _projected(case, gen, tokens):
    """q, k, v [tokens, heads, channels], side by side in one tensor as a joint projection writes them, or each by itself."""
    hq, hkv = case["hq"], case["hkv"]
    x = torch.randn((tokens, hq + 2 * hkv, D), generator=gen, device=DEV)
    x *= 1.5 * torch.rand((hq + 2 * hkv, D), generator=gen, device=DEV) + 0.25           # channels differ in size
    parts = x.to(_dtype(case)).split([hq, hkv, hkv], 1)
    return parts if case["fused"] else [p.contiguous() for p in parts]


def _pages(case, gen, count):
    """Pages that hold something already: earlier sequences' keys and values."""
    shape = (count, case["hkv"], case["page"], D)
    caches, scales = [], []
    for _ in range(2):
        x = torch.randn(shape, generator=gen, device=DEV)
        if case["fmt"] == "mxfp8":
            x, e = _quantise(x)
            scales.append(e)
        else:
            x = x.to(_dtype(case))
        caches.append(x)
    return caches + (scales or [None, None])


def _order(gen, count):
    return torch.randperm(count, generator=gen, device=DEV).int()


def _put(case, st, slots, k, v):
    """k, v [tokens, kv heads, channels] into the pages, in plain torch."""
    page, off = slots.long() // case["page"], slots.long() % case["page"]
    for x, cache, scale in ((k, st["k_cache"], st["k_scale"]), (v, st["v_cache"], st["v_scale"])):
        if case["fmt"] == "mxfp8":
            x, e = _quantise(x.float())
            scale[page, :, off] = e
        cache[page, :, off] = x.to(cache.dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    st = {"case": case}
    if case["op"] == "attn":
        new, ends = _lengths(case)
        total, page = sum(new), case["page"]
        counts = [-(-e // page) for e in ends]
        order = _order(gen, sum(counts) + 1 + sum(counts) // 8)
        st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"] = _pages(case, gen, order.numel())
        table = torch.full((case["seqs"], max(counts)), -1, dtype=torch.int32)
        at = 0
        for i, c in enumerate(counts):
            table[i, :c] = torch.arange(at, at + c)
            at += c
        table = table.to(DEV)
        st["table"] = torch.where(table < 0, 0, order[table.clamp(min=0).long()])      # a row's tail is of no meaning, as in a reused table
        for i, e in enumerate(ends):
            u = torch.arange(e, device=DEV)
            _put(case, st, st["table"][i, u // page] * page + u % page, _walk(gen, e, case["hkv"]), _walk(gen, e, case["hkv"]))
        q = torch.cat([_walk(gen, e, case["hq"])[e - n:] for n, e in zip(new, ends)]).to(_dtype(case))
        if case["fused"]:                                           # as a joint projection leaves it
            wide = torch.zeros((total, case["hq"] + 2 * case["hkv"], D), dtype=q.dtype, device=DEV)
            wide[:, :case["hq"]] = q
            q = wide[:, :case["hq"]]
        starts = torch.tensor([0] + new).cumsum(0)
        st.update(q=q, q_start=starts.int().to(DEV), kv_len=torch.tensor(ends, dtype=torch.int32, device=DEV), longest=max(ends),
                  out=torch.empty((total, case["hq"], D), dtype=q.dtype, device=DEV),
                  lse=torch.empty((total, case["hq"]), dtype=torch.float32, device=DEV) if case["lse"] else None)
        torch.cuda.synchronize()
        return st
    t = case["tokens"]
    st["q"], st["k"], st["v"] = _projected(case, gen, t)
    if case["op"] in ("rope", "rope_write"):
        if case["start"] < 0:                                       # a step of many sequences: each has a position of its own
            st["positions"] = torch.randint(0, 131072, (t,), generator=gen, device=DEV).int()
        else:
            st["positions"] = torch.arange(case["start"], case["start"] + t, device=DEV).int()
        half = case["rotary"] // 2
        st["frequency"] = BASE ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
        st["weights"] = [(1 + 0.2 * torch.randn(D, generator=gen, device=DEV)).to(_dtype(case)) if case["norm"] else None for _ in range(2)]
        st["q_out"] = torch.empty((t, case["hq"], D), dtype=_dtype(case), device=DEV)
    if case["op"] == "rope":
        st["k_out"] = torch.empty((t, case["hkv"], D), dtype=_dtype(case), device=DEV)
    else:
        count = -(-t // case["page"])
        order = _order(gen, count + 1 + count // 8)
        st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"] = _pages(case, gen, order.numel())
        u = torch.arange(t, device=DEV)
        if case.get("start", 0) < 0:                                # each sequence's next place, in pages of its own
            order = torch.randperm(order.numel() * case["page"], generator=gen, device=DEV).int()
            st["slots"] = order[:t].contiguous()
        else:
            st["slots"] = order[u // case["page"]] * case["page"] + (u % case["page"]).int()
    if case["op"] == "read":
        st["k"], st["v"] = torch.empty_like(st["k"]), torch.empty_like(st["v"])
    torch.cuda.synchronize()
    return st


# ---- one pass -------------------------------------------------------------------------------------------------------
def _held(case, st):
    """The cache as the values that it stands for."""
    if case["fmt"] == "plain":
        return [st["k_cache"], st["v_cache"]]
    return [st[n].view(torch.float8_e4m3fn) for n in ("k_cache", "v_cache")] + [st[n].view(torch.float8_e8m0fnu) for n in ("k_scale", "v_scale")]


def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    from paper_2409_12490_amd import binding as B
    case = st["case"]
    op, rope = case["op"], case["op"] in ("rope", "rope_write")
    if "params" not in st:                                          # what a program keeps: the parameter block and the workspace
        st["params"] = B.make_cache_params(
            case["hq"], case["hkv"], _dtype(case), q=st["q"], k=st.get("k"), v=st.get("v"), out=st.get("q_out") if rope else st.get("out"),
            k_out=st.get("k_out"), k_cache=st.get("k_cache"), mxfp8=case["fmt"] == "mxfp8", page_table=st.get("table"), max_q_len=case.get("new", 0),
            rotary_dim=case["rotary"] if rope else 0, interleaved=rope and case["interleaved"], norm_eps=EPS)
        st["workspace"] = B.alloc_paged_workspace(st["params"]) if op == "attn" else None
    p = st["params"]
    if op == "rope":
        B.critiprefill_norm_rope(p, st["q"], st["k"], *st["weights"], st["frequency"], st["positions"], st["q_out"], st["k_out"])
        return [st["q_out"], st["k_out"]]
    cache = (st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"])
    if op == "rope_write":
        B.critiprefill_norm_rope_write(p, st["q"], st["k"], st["v"], *st["weights"], st["frequency"], st["positions"], st["slots"], st["q_out"], *cache)
        return [st["q_out"]] + _held(case, st)
    if op == "write":
        B.critiprefill_cache_write(p, st["k"], st["v"], st["slots"], *cache)
        return _held(case, st)
    if op == "read":
        B.critiprefill_cache_read(p, st["slots"], *cache, st["k"], st["v"])
        return [st["k"], st["v"]]
    B.critiprefill_paged_attn(p, st["q"], *cache, st["table"], st["q_start"], st["kv_len"], st["out"], st["lse"], st["workspace"])
    return [st["out"]] + ([st["lse"]] if case["lse"] else [])


def _turned(case, x, weight, positions, frequency):
    """The norm of each head, then the rotation; sums and products in 32 bits, the angles in 64."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
    angle = positions.double()[:, None] * frequency
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    turn, rest = x[..., :case["rotary"]], x[..., case["rotary"]:]
    if case["interleaved"]:
        a, b = turn[..., ::2], turn[..., 1::2]
        turn = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = turn.chunk(2, -1)
        turn = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turn, rest], -1)


def _gathered(case, st, cache, scale, page, off):
    x = cache[page, :, off]
    return _values(x, scale[page, :, off]) if case["fmt"] == "mxfp8" else x.float()


def _run_plain(st):
    case = st["case"]
    op, dtype = case["op"], _dtype(case)
    if op in ("rope", "rope_write"):
        q = _turned(case, st["q"], st["weights"][0], st["positions"], st["frequency"]).to(dtype)
        k = _turned(case, st["k"], st["weights"][1], st["positions"], st["frequency"])
        if op == "rope":
            return [q, k.to(dtype)]
        _put(case, st, st["slots"], k, st["v"])
        return [q] + _held(case, st)
    if op == "write":
        _put(case, st, st["slots"], st["k"], st["v"])
        return _held(case, st)
    if op == "read":
        page, off = st["slots"].long() // case["page"], st["slots"].long() % case["page"]
        return [_gathered(case, st, st[c], st[s], page, off).to(dtype) for c, s in (("k_cache", "k_scale"), ("v_cache", "v_scale"))]
    # all sequences at once, filled up to the longest
    hq, hkv, seqs, new = case["hq"], case["hkv"], case["seqs"], case["new"]
    start, ends = st["q_start"].long(), st["kv_len"].long()
    t, u = torch.arange(new, device=DEV), torch.arange(st["longest"], device=DEV)
    count = start[1:] - start[:-1]
    there = u < ends[:, None]
    page = st["table"].long()[:, u // case["page"]]
    off = (u % case["page"]).expand_as(page)
    k, v = (_gathered(case, st, st[c], st[s], page, off).masked_fill_(~there[..., None, None], 0).transpose(1, 2)
            for c, s in (("k_cache", "k_scale"), ("v_cache", "v_scale")))
    total = st["q"].shape[0]
    q = st["q"].float()[(start[:-1, None] + t).clamp(max=total - 1)]                    # [seqs, new, heads, channels]
    q = q.unflatten(2, (hkv, hq // hkv)).permute(0, 2, 3, 1, 4).flatten(2, 3)           # [seqs, kv heads, group * new, channels]
    x = torch.matmul(q, k.transpose(-1, -2)).mul_(SCALE).unflatten(2, (-1, new))
    seen = (u <= (ends - count)[:, None, None] + t[:, None]) & there[:, None]           # [seqs, new, tokens]
    x.masked_fill_(~seen[:, None, None], float("-inf"))
    most = x.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)
    x.sub_(most).exp_()
    mass = x.sum(-1, keepdim=True)
    out = torch.matmul(x.flatten(2, 3), v).unflatten(2, (-1, new)) / mass
    rows = torch.arange(total, device=DEV)
    seq = torch.searchsorted(start[1:].contiguous(), rows, right=True)                  # whose each row is
    at = rows - start[seq]
    out = out[seq, :, :, at].flatten(1, 2).to(dtype)
    return [out, (mass.log() + most)[seq, :, :, at, 0].flatten(1, 2)] if case["lse"] else [out]


# ---- what is right --------------------------------------------------------------------------------------------------
def _turned64(case, x, weight, positions, frequency):
    y = x.double().clone()
    if weight is not None:
        y = y / (y.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt() * weight.double()
    half = case["rotary"] // 2
    first = torch.arange(half, device=DEV) * (2 if case["interleaved"] else 1)
    second = first + (1 if case["interleaved"] else half)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), positions.double()[:, None] * frequency)[:, None]
    z = torch.complex(y[..., first], y[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _stored64(case, st, slots, k, v):
    """The cache after the write, without the last rounding; the scales, whole powers of two, are not judged."""
    caches = []
    for x, cache in ((k, st["k_cache"]), (v, st["v_cache"])):
        held = cache.view(torch.float8_e4m3fn) if case["fmt"] == "mxfp8" else cache
        held = held.double()
        if case["fmt"] == "mxfp8":
            blocks = x.reshape(*x.shape[:2], 4, 32)
            size = torch.log2(blocks.abs().amax(-1, keepdim=True) / 448).ceil()
            x = (blocks / torch.exp2(size)).reshape(x.shape)
        for i in range(case["page"]):
            mine = (slots % case["page"] == i).nonzero()[:, 0]
            held[(slots[mine] // case["page"]).long(), :, i] = x[mine]
        caches.append(held)
    return caches + ([None, None] if case["fmt"] == "mxfp8" else [])


def _held64(case, st):
    found = []
    for cache, scale in ((st["k_cache"], st["k_scale"]), (st["v_cache"], st["v_scale"])):
        if case["fmt"] == "mxfp8":
            found.append(cache.view(torch.float8_e4m3fn).double() * torch.exp2(scale.double() - 127).repeat_interleave(32, -1))
        else:
            found.append(cache.double())
    return [x.transpose(1, 2).flatten(0, 1) for x in found]                             # [slots, kv heads, channels]


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("rope", "rope_write"):
        q, k = (_turned64(case, st[n], w, st["positions"], st["frequency"]) for n, w in zip("qk", st["weights"]))
        return [q, k] if case["op"] == "rope" else [q] + _stored64(case, st, st["slots"], k, st["v"].double())
    if case["op"] == "write":
        return _stored64(case, st, st["slots"], st["k"].double(), st["v"].double())
    held = _held64(case, st)
    if case["op"] == "read":
        return [x[st["slots"].long()] for x in held]
    new, ends = _lengths(case)
    group = case["hq"] // case["hkv"]
    out = torch.empty(st["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(st["q"].shape[:2], dtype=torch.float64, device=DEV)
    row = 0
    for i, (n, e) in enumerate(zip(new, ends)):
        u = torch.arange(e, device=DEV)
        slots = st["table"][i, u // case["page"]].long() * case["page"] + u % case["page"]
        for h in range(case["hkv"]):
            k, v = (x[slots, h] for x in held)
            for a in range(0, n, 1024):
                b = min(n, a + 1024)
                q = st["q"][row + a:row + b, h * group:(h + 1) * group].double()
                z = (q.reshape(-1, D) @ k.t().contiguous() * SCALE).view(b - a, group, e)
                z.masked_fill_((u > torch.arange(e - n + a, e - n + b, device=DEV)[:, None])[:, None], float("-inf"))
                total = z.logsumexp(-1)
                lse[row + a:row + b, h * group:(h + 1) * group] = total
                out[row + a:row + b, h * group:(h + 1) * group] = ((z - total[..., None]).exp().view(-1, e) @ v).view(b - a, group, D)
        row += n
    return [out, lse] if case["lse"] else [out]
