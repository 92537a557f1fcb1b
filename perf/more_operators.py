"""A cache held in 4 bits, as cases that can be timed and checked one by one.

``append``  norms of queries and keys for each head, the position rotation, and keys and values into the pages (what a decode step and a prompt's chunk do)
``write``   keys and values of a finished prefill into the pages
``read``    and back, as tensors
``attn``    attention of each sequence's new tokens (one: decode; many: a follow-up chunk) over the pages

A row of the cache is 128 e2m1 elements (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign), two to a byte, the even channel in the lower half, and a power of two for each
32 channels: the byte e stands for 2^(e - 127), the smallest with max |x| <= 7 * 2^(e - 127), which leaves no element off by more than one unit.  ``append`` and
``write`` return the whole pool as the values that it stands for, which a call of ``read`` gives; ``append``'s keys, rounded to 4 bits from sums that two
programs may add in another order, in an 8-bit type that has these values too.
"""
import random

import torch

own = False

D = 128
DEV = "cuda"
BASE = 500000.0                                    # of the rotation
EPS = 1e-5
SCALE = D ** -0.5
NEAREST, FURTHEST = 2, 252                         # biased exponents that a scale may have
KEYS = torch.float8_e4m3fn                         # 2^-9 to 448: of the keys here no element but 0 is smaller than 2^-7 or larger than 24
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _append(name, dtype, hq, hkv, tokens, start, page=64, rotary=128, interleaved=False, norm=True, fused=True):
    return {"name": name, "op": "append", "dtype": dtype, "hq": hq, "hkv": hkv, "tokens": tokens, "start": start, "page": page, "rotary": rotary,
            "interleaved": interleaved, "norm": norm, "fused": fused}


def _store(name, op, dtype, hkv, tokens, page, fused=True):
    return {"name": name, "op": op, "dtype": dtype, "hq": hkv, "hkv": hkv, "tokens": tokens, "page": page, "fused": fused}


def _attn(name, dtype, hq, hkv, seqs, new, past, page, lengths=0, ragged=False, lse=False, fused=False):
    """``new`` tokens of each sequence over ``past`` tokens and themselves; ragged: up to these, by the number ``lengths``."""
    return {"name": name, "op": "attn", "dtype": dtype, "hq": hq, "hkv": hkv, "seqs": seqs, "new": new, "past": past, "page": page, "lengths": lengths,
            "ragged": ragged, "lse": lse, "fused": fused}


def listed():
    return [
        # one decode step of 64 sequences, each at a place of its own
        _append("append_64", "bf16", 32, 8, 64, -1),
        # the fp32 path: a chunk far into a document, odd length, half of the channels rotated in neighbouring pairs
        _append("append_fp32_2777", "fp32", 8, 2, 2777, 100000, page=16, rotary=64, interleaved=True, fused=False),
        # a 64K prompt goes into the cache
        _store("write_65536", "write", "bf16", 8, 65536, 64),
        # a short one in fp32, an odd number of heads
        _store("write_fp32_1001", "write", "fp32", 3, 1001, 128, fused=False),
        # a short prefix comes back for a prefill that goes on from it
        _store("read_700", "read", "bf16", 8, 700, 64),
        # a long one, Yi-9B-shaped
        _store("read_50001", "read", "bf16", 4, 50001, 32, fused=False),
        # the smallest decode: one sequence with a short past
        _attn("decode_1x2000", "bf16", 32, 8, 1, 1, 1999, 64),
        # what 4 bits are for: one sequence of a million tokens
        _attn("decode_1x1000000", "bf16", 32, 8, 1, 1, 999999, 64),
        # a batch of decoding sequences of all lengths
        _attn("decode_64", "bf16", 32, 8, 64, 1, 32768, 64, lengths=3, ragged=True, lse=True),
        # follow-ups and single tokens in one batch, Yi-9B-shaped
        _attn("mixed_20", "bf16", 32, 4, 20, 300, 12000, 32, lengths=5, ragged=True),
        # fp32: the reference that a bf16 result is compared with
        _attn("chunk_fp32_3x200", "fp32", 4, 2, 3, 200, 3000, 16, lengths=2, ragged=True, lse=True),
        # a chunk of 4096 at the end of a 32K prompt
        _attn("chunk_4096_32768", "bf16", 32, 8, 1, 4096, 28672, 64, lse=True, fused=True),
    ]


def _spread(rng, low, high):
    return int(low * (high / low) ** rng.random())


def draw(rng):
    while True:
        op = rng.choice(["append", "append", "write", "read", "attn", "attn", "attn", "attn"])
        fp32 = rng.random() < 0.2
        dtype = "fp32" if fp32 else "bf16"
        hq, hkv = rng.choice([(4, 2), (8, 2), (3, 3), (1, 1)] if fp32 else [(32, 8), (32, 8), (32, 4), (8, 2), (4, 4), (28, 4), (40, 8), (2, 1), (16, 1)])
        page = rng.choice([16, 32, 64, 64, 128])
        if op == "attn":
            kind = rng.choice(["decode", "decode", "few", "chunk", "chunk"])
            new = {"decode": 1, "few": rng.randint(2, 16), "chunk": _spread(rng, 17, 512 if fp32 else 4096)}[kind]
            past = _spread(rng, 1, 8192 if fp32 else 1000000) - 1
            seqs = _spread(rng, 1, 64)
            case = _attn("", dtype, hq, hkv, seqs, new, past, page, rng.randint(1, 1 << 20), rng.random() < 0.7, rng.random() < 0.4, rng.random() < 0.5)
            _, ends = _lengths(case)
            padded = seqs * hq * new * max(ends)                    # what the plain form lays out
            if padded > 2 ** 31 or seqs * hkv * max(ends) > 2 ** 23 or work(case)["flops"] > (1e11 if fp32 else 2e12):
                continue
        elif op == "append":
            case = _append("", dtype, hq, hkv, _spread(rng, 1, 16384), rng.choice([-1, 0, _spread(rng, 1, 1 << 20)]), page, rng.choice([128, 128, 64, 32]),
                           rng.random() < 0.3, rng.random() < 0.7, rng.random() < 0.6)
        else:
            case = _store("", op, dtype, hkv, _spread(rng, 1, 65536), page, rng.random() < 0.6)
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


ROW = D // 2 + 4                                   # bytes of a token's K or V of one head in the cache


def _pool_pages(case):
    count = -(-case["tokens"] // case["page"])
    return count + 1 + count // 8


def work(case):
    e, hq, hkv = _size(case), case["hq"], case["hkv"]
    if case["op"] == "attn":
        new, ends = _lengths(case)
        total = sum(new)
        pairs = sum(n * (e_ - n) + n * (n + 1) // 2 for n, e_ in zip(new, ends))
        size = 2 * total * hq * D * e + sum(ends) * hkv * 2 * ROW + (total * hq * 4 if case["lse"] else 0)
        return {"bytes": size, "flops": 4 * D * hq * pairs}
    t = case["tokens"]
    if case["op"] == "read":
        return {"bytes": t * hkv * 2 * (ROW + D * e) + 4 * t, "flops": 2 * t * hkv * 2 * D}
    held = _pool_pages(case) * case["page"]                        # rows that come back as values
    size, flops = t * hkv * 2 * (D * e + ROW) + 4 * t + held * hkv * 2 * (ROW + D * e), 2 * (t + held) * hkv * 2 * D
    if case["op"] == "append":
        size, flops = size + 2 * t * hq * D * e + 4 * t, flops + 10 * t * (hq + hkv) * D
    return {"bytes": size, "flops": flops}


# ---- the cache's 4-bit format, in plain torch -----------------------------------------------------------------------
def _quantise(x):
    """x [..., 128] in fp32: bytes [..., 64] and scales [..., 4]."""
    blocks = x.unflatten(-1, (4, 32))
    most = blocks.abs().amax(-1)
    m, e = torch.frexp(most)                                       # most = 2 m 2^(e - 1), and 7 = 1.75 * 2^2
    e = torch.where(most == 0, NEAREST, e + 124 + (m > 0.875).int()).clamp(NEAREST, FURTHEST)
    units = torch.ldexp(blocks, (127 - e).unsqueeze(-1))
    a = units.abs()
    # steps of 0.5 below 2, of 1 below 4, of 2 up to 6; round() takes ties to the even number, which is the even code
    code = torch.where(a < 2, (2 * a).round(), torch.where(a < 4, 2 + a.round(), 4 + (a / 2).round())).clamp_(max=7).to(torch.uint8)
    code = (code + 8 * torch.signbit(units).to(torch.uint8)).flatten(-2)
    return code[..., ::2] + 16 * code[..., 1::2], e.to(torch.uint8)


_pairs = {}


def _values(held, e):
    """Bytes [..., 64] and scales [..., 4] as fp32 values [..., 128]."""
    if DEV not in _pairs:
        one = torch.tensor(LEVELS + [-x for x in LEVELS], device=DEV)
        _pairs[DEV] = torch.stack([one.repeat(16), one.repeat_interleave(16)], 1)       # both values of each byte
    x = _pairs[DEV][held.int()].flatten(-2).unflatten(-1, (4, 32))
    return torch.ldexp(x, (e.int() - 127).unsqueeze(-1)).flatten(-2)


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _walk(gen, tokens, heads):
    """Neighbouring tokens are alike, as in a text: a random walk and noise, scaled to unit variance."""
    x = torch.randn((tokens, heads, D), generator=gen, device=DEV).mul_(0.1).cumsum(0)
    x += torch.randn((tokens, heads, D), generator=gen, device=DEV)
    return x.div_(x.std() + 1e-6)


def _uneven(gen, heads):
    """Channels differ in size, as a projection's do."""
    return 1.5 * torch.rand((heads, D), generator=gen, device=DEV) + 0.25


def _projected(case, gen, tokens):
    """q, k, v [tokens, heads, channels], side by side in one tensor as a joint projection writes them, or each by itself."""
    hq, hkv = case["hq"], case["hkv"]
    x = torch.randn((tokens, hq + 2 * hkv, D), generator=gen, device=DEV)
    x *= _uneven(gen, hq + 2 * hkv)
    parts = x.to(_dtype(case)).split([hq, hkv, hkv], 1)
    return parts if case["fused"] else [p.contiguous() for p in parts]


def _pages(case, gen, count):
    """Pages that hold something already: earlier sequences' keys and values."""
    (k, ks), (v, vs) = (_quantise(torch.randn((count, case["hkv"], case["page"], D), generator=gen, device=DEV)) for _ in range(2))
    return k, v, ks, vs


def _order(gen, count):
    return torch.randperm(count, generator=gen, device=DEV).int()


def _put(case, st, slots, k, v):
    """k, v [tokens, kv heads, channels] into the pages, in plain torch."""
    page, off = slots.long() // case["page"], slots.long() % case["page"]
    for x, cache, scale in ((k, st["k_cache"], st["k_scale"]), (v, st["v_cache"], st["v_scale"])):
        cache[page, :, off], scale[page, :, off] = _quantise(x.float())


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    st = {"case": case}
    page = case["page"]
    if case["op"] == "attn":
        new, ends = _lengths(case)
        total = sum(new)
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
            k, v = _walk(gen, e, case["hkv"]) * _uneven(gen, case["hkv"]), _walk(gen, e, case["hkv"])
            _put(case, st, st["table"][i, u // page] * page + u % page, k, v)
        q = torch.cat([_walk(gen, e, case["hq"])[e - n:] if n > 1 else torch.randn((1, case["hq"], D), generator=gen, device=DEV) for n, e in zip(new, ends)])
        q = q.to(_dtype(case))
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
    order = _order(gen, _pool_pages(case))
    st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"] = _pages(case, gen, order.numel())
    u, held = torch.arange(t, device=DEV), order.numel() * page
    if case.get("start", 0) < 0:                                    # a step of many sequences: each has a position and a next place of its own
        st["slots"] = _order(gen, held)[:t].contiguous()
    else:
        st["slots"] = order[u // page] * page + (u % page).int()
    if case["op"] == "read":
        st["k_back"], st["v_back"] = (torch.empty((t, case["hkv"], D), dtype=_dtype(case), device=DEV) for _ in range(2))
    else:
        st["every"] = torch.arange(held, dtype=torch.int32, device=DEV)
        st["k_back"], st["v_back"] = (torch.empty((held, case["hkv"], D), dtype=_dtype(case), device=DEV) for _ in range(2))
    if case["op"] == "append":
        if case["start"] < 0:
            st["positions"] = torch.randint(0, 131072, (t,), generator=gen, device=DEV).int()
        else:
            st["positions"] = torch.arange(case["start"], case["start"] + t, device=DEV).int()
        half = case["rotary"] // 2
        st["frequency"] = BASE ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
        st["weights"] = [(1 + 0.2 * torch.randn(D, generator=gen, device=DEV)).to(_dtype(case)) if case["norm"] else None for _ in range(2)]
        st["q_out"] = torch.empty((t, case["hq"], D), dtype=_dtype(case), device=DEV)
    torch.cuda.synchronize()
    return st


# ---- one pass -------------------------------------------------------------------------------------------------------
def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    from paper_2409_12490_amd import binding as B
    case = st["case"]
    op, shape = case["op"], (case["hq"], case["hkv"], _dtype(case))
    cache = (st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"])
    if "params" not in st:                                          # what a program keeps: the parameter blocks and the workspace
        pool = dict(k_cache=st["k_cache"], mxfp4=True)
        if op == "attn":
            st["params"] = B.make_cache_params(*shape, q=st["q"], out=st["out"], page_table=st["table"], max_q_len=case["new"], **pool)
            st["workspace"] = B.alloc_paged_workspace(st["params"])
        else:
            if op == "append":
                st["params"] = B.make_cache_params(*shape, q=st["q"], k=st["k"], v=st["v"], out=st["q_out"], rotary_dim=case["rotary"],
                                                   interleaved=case["interleaved"], norm_eps=EPS, **pool)
            else:
                st["params"] = B.make_cache_params(*shape, k=st["k"], v=st["v"], **pool)
            st["back"] = B.make_cache_params(*shape, k=st["k_back"], v=st["v_back"], **pool)
    p = st["params"]
    if op == "attn":
        B.critiprefill_paged_attn(p, st["q"], *cache, st["table"], st["q_start"], st["kv_len"], st["out"], st["lse"], st["workspace"])
        return [st["out"]] + ([st["lse"]] if case["lse"] else [])
    if op == "append":
        B.critiprefill_norm_rope_write(p, st["q"], st["k"], st["v"], *st["weights"], st["frequency"], st["positions"], st["slots"], st["q_out"], *cache)
    elif op == "write":
        B.critiprefill_cache_write(p, st["k"], st["v"], st["slots"], *cache)
    B.critiprefill_cache_read(st["back"], st["slots"] if op == "read" else st["every"], *cache, st["k_back"], st["v_back"])
    return [st["q_out"], st["k_back"].to(KEYS), st["v_back"]] if op == "append" else [st["k_back"], st["v_back"]]


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


def _gathered(case, st, slots):
    """Keys and values of slots of any shape, [..., kv heads, channels] in fp32."""
    page, off = slots.long() // case["page"], slots.long() % case["page"]
    return [_values(st[c][page, :, off], st[s][page, :, off]) for c, s in (("k_cache", "k_scale"), ("v_cache", "v_scale"))]


def _run_plain(st):
    case = st["case"]
    op, dtype = case["op"], _dtype(case)
    if op == "read":
        return [x.to(dtype) for x in _gathered(case, st, st["slots"])]
    if op == "write":
        _put(case, st, st["slots"], st["k"], st["v"])
        return [x.to(dtype) for x in _gathered(case, st, st["every"])]
    if op == "append":
        q = _turned(case, st["q"], st["weights"][0], st["positions"], st["frequency"]).to(dtype)
        _put(case, st, st["slots"], _turned(case, st["k"], st["weights"][1], st["positions"], st["frequency"]), st["v"])
        k, v = _gathered(case, st, st["every"])
        return [q, k.to(KEYS), v.to(dtype)]
    # all sequences at once, filled up to the longest
    hq, hkv, new = case["hq"], case["hkv"], case["new"]
    start, ends = st["q_start"].long(), st["kv_len"].long()
    t, u = torch.arange(new, device=DEV), torch.arange(st["longest"], device=DEV)
    count = start[1:] - start[:-1]
    there = u < ends[:, None]
    slots = st["table"].long()[:, u // case["page"]] * case["page"] + u % case["page"]
    k, v = (x.masked_fill_(~there[..., None, None], 0).transpose(1, 2) for x in _gathered(case, st, slots))
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


def _held64(case, st, name, head):
    """What the cache holds of a KV head, [slots, channels]."""
    held, e = st[name + "_cache"][:, head].flatten(0, 1), st[name + "_scale"][:, head].flatten(0, 1)
    x = torch.empty((held.shape[0], D), dtype=torch.float64, device=DEV)
    for half in range(2):
        code = held.long() >> 4 * half & 15
        m, power = code & 1, code >> 1 & 3
        size = torch.where(power == 0, m / 2, (1 + m.double() / 2) * torch.exp2(power.double() - 1))
        x[:, half::2] = torch.where(code > 7, -size, size)
    return x * torch.exp2(e.double() - 127).repeat_interleave(32, -1)


def _rounded64(x):
    """The values of the 4-bit format nearest to x, halfway ones at the even code, under the scale of their 32 channels."""
    blocks = x.reshape(*x.shape[:-1], 4, 32)
    size = torch.exp2(torch.log2(blocks.abs().amax(-1, keepdim=True) / 7).ceil().clamp(NEAREST - 127, FURTHEST - 127))
    u = blocks.abs() / size
    found = torch.zeros_like(u)
    for i, (low, high) in enumerate(zip(LEVELS, LEVELS[1:])):
        border = (low + high) / 2
        found += (high - low) * (u > border if i % 2 == 0 else u >= border)
    return torch.copysign(found * size, blocks).reshape(x.shape)


def _stored64(case, st, slots, k, v):
    """The pool after the write, [slots, kv heads, channels]."""
    found = []
    for name, x in (("k", k), ("v", v)):
        pool = torch.stack([_held64(case, st, name, h) for h in range(case["hkv"])], 1)
        pool[slots.long()] = _rounded64(x)
        found.append(pool)
    return found


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "append":
        q, k = (_turned64(case, st[n], w, st["positions"], st["frequency"]) for n, w in zip("qk", st["weights"]))
        return [q] + _stored64(case, st, st["slots"], k, st["v"].double())
    if case["op"] == "write":
        return _stored64(case, st, st["slots"], st["k"].double(), st["v"].double())
    if case["op"] == "read":
        return [torch.stack([_held64(case, st, n, h)[st["slots"].long()] for h in range(case["hkv"])], 1) for n in "kv"]
    new, ends = _lengths(case)
    group = case["hq"] // case["hkv"]
    out = torch.empty(st["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(st["q"].shape[:2], dtype=torch.float64, device=DEV)
    for h in range(case["hkv"]):
        held_k, held_v = (_held64(case, st, n, h) for n in "kv")
        row = 0
        for i, (n, e) in enumerate(zip(new, ends)):
            u = torch.arange(e, device=DEV)
            slots = st["table"][i, u // case["page"]].long() * case["page"] + u % case["page"]
            k, v = held_k[slots], held_v[slots]
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
