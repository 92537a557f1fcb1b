"""The cache of 4 bits: keys and values written, with and without head norms and rotation on the way, and read back, against fp64."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2409_12490_amd import binding as B
from tests.cache_helpers import DEV, f64, side_by_side, streams
from tests.test_gpu_cache import ROPES, _check, _rope_inputs, _wanted
from tests.test_gpu_cache_stream import PART, _inputs, _parts, _same, _slots

pytestmark = pytest.mark.gpu


def _store(x, slots=None, y=None, page=16, spare=1):
    """x (and y) [tokens, heads, 128] written: the cache."""
    y = x if y is None else y
    tokens, hkv = x.shape[:2]
    slots = torch.arange(tokens, dtype=torch.int32, device=DEV) if slots is None else slots
    cache = B.alloc_cache(tokens // page + spare, hkv, page, x.dtype, mxfp4=True)
    p = B.make_cache_params(hkv, hkv, x.dtype, k=x, v=y, k_cache=cache[0], mxfp4=True)
    B.critiprefill_cache_write(p, x, y, slots, *cache)
    return cache, slots


def _load(cache, slots, dtype, heads_more=0):
    tokens, hkv = slots.numel(), cache[0].shape[1]
    back = [torch.full((tokens, hkv + heads_more, 128), float("nan"), dtype=dtype, device=DEV)[:, :hkv] for _ in range(2)]
    p = B.make_cache_params(hkv, hkv, dtype, k=back[0], v=back[1], k_cache=cache[0], mxfp4=True)
    B.critiprefill_cache_read(p, slots, *cache, *back)
    return back


def _flat(cache):
    return [c.transpose(1, 2).flatten(0, 1).cpu().numpy() for c in cache]                     # [slots, heads, row]


def test_borders_of_the_4_bit_format():
    """Every value of the format, every border between two and the fp32 numbers next to it, in blocks whose maxima are around the borders of the scale, from its smallest to its largest."""
    levels = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
    ties = np.concatenate([(levels[1:] + levels[:-1]) / 2, [7.0]])
    near = np.unique(np.concatenate([levels, ties, ties * (1 + 2.0 ** -23), ties * (1 - 2.0 ** -23), [1e-30, 0.24, 6.5]]))
    near = np.concatenate([near, -near])
    rows = []
    for power in (0, -5, 40, -124, -125, -126, -100, 100, 125):
        for top in (7.0, 7 * (1 - 2.0 ** -22), 6.0, 4.0, 3.5 * (1 + 2.0 ** -22), 3.6):
            for part in np.array_split(near, 3):
                b = np.zeros(32)
                b[:len(part)] = np.clip(part, -top, top)
                b[31] = top
                rows.append(b * 2.0 ** power)
    rows += [np.zeros(32), np.full(32, -0.0), np.full(32, 2.0 ** -149), np.full(32, -2.0 ** -126), np.full(32, 3.4e38), np.array([3.4e38] + [1e-38] * 31), np.array([-2.5e38] + [1e37] * 31)]
    with np.errstate(over="ignore"):
        x = np.concatenate(rows + [np.zeros(32)] * (-len(rows) % 4)).reshape(-1, 1, 128).astype(np.float32)
    x[~np.isfinite(x)] = 3e38
    x = torch.from_numpy(x).to(DEV)
    cache, slots = _store(x)
    back = _load(cache, slots, torch.float32)
    torch.cuda.synchronize()
    held, e = O.mx4_quantise(f64(x))
    n = x.shape[0]
    for c, s, y in zip(_flat(cache[:2]), _flat(cache[2:]), back):
        assert np.array_equal(s[:n], e) and np.array_equal(c[:n], held)
        assert np.array_equal(f64(y), O.mx4_values(held, e)) and torch.isfinite(y).all()


def test_every_byte_under_every_scale_comes_back():
    """All 256 bytes under all scales that a write gives, 2 to 252, and 255."""
    rows = [list(range(2, 253)) + [255]]
    n = len(rows[0])
    cache = [c.zero_() for c in B.alloc_cache(n * 4 // 16, 1, 16, torch.float32, mxfp4=True)]  # slot 4 s + x: bytes 64 x .. 64 x + 63 under scale s
    b = torch.arange(256, dtype=torch.uint8, device=DEV).view(4, 64).repeat(n, 1)
    e = torch.tensor(rows[0], dtype=torch.uint8, device=DEV).repeat_interleave(4)[:, None].expand(-1, 4)
    for c in cache[:2]:
        c.view(-1, 64)[:] = b
    for s in cache[2:]:
        s.view(-1, 4)[:] = e
    slots = torch.arange(4 * n, dtype=torch.int32, device=DEV)
    want = O.mx4_values(b.cpu().numpy(), e.cpu().numpy())[:, None]
    for dtype in (torch.float32, torch.bfloat16):                   # both hold all of these
        for y in _load(cache, slots, dtype):
            assert np.array_equal(f64(y), want, equal_nan=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_values_that_are_not_finite_take_their_block_along(dtype):
    x = torch.ones((4, 1, 128), device=DEV, dtype=dtype)
    x[0, 0, 5], x[1, 0, 40], x[2, 0, 127], x[3, 0, 64] = float("inf"), float("nan"), float("-inf"), 3e38
    cache, slots = _store(x)
    y, z = _load(cache, slots, dtype)
    gone = torch.zeros((4, 1, 128), dtype=torch.bool, device=DEV)
    gone[0, :, :32] = gone[1, :, 32:64] = gone[2, :, 96:] = True
    assert torch.equal(torch.isnan(y), gone) and (y[:3][~gone[:3]] == 1).all() and torch.equal(torch.isnan(z), gone) and torch.isfinite(y[3]).all()
    assert (cache[2][0, 0, :3].cpu() == torch.tensor([[255, 125, 125, 125], [125, 255, 125, 125], [125, 125, 125, 255]])).all()   # 1 = 4 * 2^-2, and 7 * 2^-3 is less


@pytest.mark.parametrize("dtype,hkv,page,tokens,fused", [("bf16", 8, 64, 1, True), ("bf16", 1, 16, 777, False), ("fp32", 3, 32, 130, True), ("bf16", 4, 256, 5000, True), ("fp32", 1, 16, 1, False)])
def test_write_and_read(dtype, hkv, page, tokens, fused):
    gen = torch.Generator().manual_seed(tokens)
    k, v = side_by_side(gen, tokens, (hkv, hkv), dtype, extra=3 if fused else 0)
    k = (k * 2.0 ** torch.randint(-30, 30, (tokens, hkv, 1), generator=gen).to(DEV)).to(v.dtype)
    if fused:
        wide = torch.cat([k, v, v], 1)
        k, v = wide[:, :hkv], wide[:, hkv:2 * hkv]
    n_pages = tokens // page + 2
    slots = torch.randperm(n_pages * page, generator=gen)[:tokens].int().to(DEV)
    cache, _ = _store(k, slots, v, page, 2)
    ko, vo = _load(cache, slots, k.dtype, 1)
    torch.cuda.synchronize()
    for x, y in ((k, ko), (v, vo)):
        assert np.array_equal(f64(y), O.mx4_values(*O.mx4_quantise(f64(x))))                  # whole powers of two: nothing else is rounded
    more = torch.cat([slots, torch.tensor([-1, n_pages * page, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=DEV), slots[:1]])
    two = _load(cache, more, k.dtype)
    for a, b in zip(two, (ko, vo)):
        assert torch.equal(a[:tokens], b) and not a[tokens:-1].any() and torch.equal(a[-1], b[0])


def _check_held(got, want, size):
    """Half a step of e2m1 under the scale of the block (0.25, 0.5, 1 unit up to 2, 4, 7), from a value that is itself off by under 32 roundings of its terms; the scale can be the next one
    where the maximum is that near to 7 units."""
    unit = 2.0 ** (O.mx4_scale(want * (1 + 2.0 ** -16)).astype(np.float64) - 127.0)
    unit = (unit[..., None] * np.ones(32)).reshape(want.shape)
    a = np.abs(want) / unit * (1 + 2.0 ** -16)
    bound = unit * np.where(a <= 2, 0.25, np.where(a <= 4, 0.5, 1.0)) + 32 * 2.0 ** -24 * size
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= bound).all(), f"{np.max(np.abs(got - want) / bound):.2f} of the bound"


@pytest.mark.parametrize("case", ROPES, ids=lambda c: "x".join(map(str, c)))
def test_norm_rope_write(case):
    dtype, hq, hkv, tokens, rotary, inter, _, _ = case
    q, k, v, w, pos, freq = _rope_inputs(case)
    page, n_pages = 16, tokens // 16 + 3
    gen = torch.Generator().manual_seed(3)
    slots = torch.randperm(n_pages * page, generator=gen)[:tokens].int()
    outside = torch.rand(tokens, generator=gen) < 0.1
    slots = torch.where(outside, torch.tensor([-1, n_pages * page, -2 ** 31, 2 ** 31 - 1])[torch.arange(tokens) % 4].int(), slots).to(DEV)
    cache = [c.fill_(3) for c in B.alloc_cache(n_pages, hkv, page, q.dtype, mxfp4=True)]
    q_out = torch.full((tokens, hq, 128), float("nan"), dtype=q.dtype, device=DEV)
    p = B.make_cache_params(hq, hkv, q.dtype, q=q, k=k, v=v, out=q_out, k_cache=cache[0], mxfp4=True, rotary_dim=rotary, interleaved=inter, norm_eps=1e-5)
    B.critiprefill_norm_rope_write(p, q, k, v, *w, freq, pos if rotary else None, slots, q_out, *cache)
    torch.cuda.synchronize()
    _check(f64(q_out), *_wanted(case, q, w[0], pos, freq), dtype)
    flat = _flat(cache)
    kept = (~outside).nonzero()[:, 0].numpy()
    at = slots.cpu().numpy()[kept]
    rest = np.ones(n_pages * page, dtype=bool)
    rest[at] = False
    assert all((c[rest] == 3).all() for c in flat)                                            # nothing else is written
    wk, sk = _wanted(case, k, w[1], pos, freq)
    _check_held(O.mx4_values(flat[0][at], flat[2][at]), wk[kept], sk[kept])
    assert np.array_equal(O.mx4_values(flat[1][at], flat[3][at]), O.mx4_values(*O.mx4_quantise(f64(v)))[kept])      # as they are: no rounding but the format's


def test_norm_rope_write_with_what_is_not_finite():
    """What is not finite goes through norm and rotation: an infinity of K becomes NaN in its own pair, channels 36 and 100, whether a norm makes it inf / inf (and the finite ones 0) or not; a NaN of
    V takes its block along, one of Q reaches its row; no other head and token."""
    gen = torch.Generator().manual_seed(9)
    q, k, v = side_by_side(gen, 5, (4, 2, 2), "bf16")
    q[1, 2, 3], k[2, 1, 100], v[4, 0, 33] = float("nan"), float("inf"), float("nan")
    cache = B.alloc_cache(1, 2, 16, q.dtype, mxfp4=True)
    q_out = torch.zeros((5, 4, 128), dtype=q.dtype, device=DEV)
    slots = torch.arange(5, dtype=torch.int32, device=DEV)
    weight = torch.ones(128, dtype=q.dtype, device=DEV)
    for w in (weight, None):
        p = B.make_cache_params(4, 2, q.dtype, q=q, k=k, v=v, out=q_out, k_cache=cache[0], mxfp4=True, rotary_dim=128, norm_eps=1e-5)
        B.critiprefill_norm_rope_write(p, q, k, v, w, w, B.rotary_frequencies(), slots + 1000, slots, q_out, *cache)
        torch.cuda.synchronize()
        want_k, want_v = np.zeros((5, 2, 4), dtype=bool), np.zeros((5, 2, 4), dtype=bool)
        want_k[2, 1, [1, 3]], want_v[4, 0, 1] = True, True
        ks, vs = _flat(cache[2:])
        assert np.array_equal(ks[:5] == 255, want_k) and np.array_equal(vs[:5] == 255, want_v)
        bad = torch.isnan(q_out).any(-1).cpu()
        assert bad[1, 2] and bad.sum() == 1
        if w is not None:
            assert (ks[2, 1, [0, 2]] == 2).all()                    # zeros


def test_places_beyond_32_bits_of_offset():
    hkv, page, n_pages = 8, 64, 140000                              # 4.6 GB of K
    cache = B.alloc_cache(n_pages, hkv, page, mxfp4=True)
    gen = torch.Generator().manual_seed(1)
    k, v = side_by_side(gen, 100, (hkv, hkv), "bf16")
    slots = (torch.randperm(5000, generator=gen)[:100] + (n_pages * page - 5000)).int().to(DEV)
    p = B.make_cache_params(hkv, hkv, k.dtype, k=k, v=v, k_cache=cache[0], mxfp4=True)
    B.critiprefill_cache_write(p, k, v, slots, *cache)
    for x, y in zip((k, v), _load(cache, slots, k.dtype)):
        assert np.array_equal(f64(y), O.mx4_values(*O.mx4_quantise(f64(x))))


@pytest.mark.parametrize("rotary,interleaved", [(128, False), (64, False), (96, True), (0, False)])
@pytest.mark.parametrize("dtype,tokens", [("bf16", 7601), ("fp32", 3803)])
def test_calls_past_the_caches_give_the_same_bits(dtype, tokens, rotary, interleaved):
    hq, hkv, page, n_pages = 32, 8, 64, 130
    q_bytes, held = 128 * (2 if dtype == "bf16" else 4) * 2 * (hq + hkv), 2 * hkv * 64
    assert tokens * (q_bytes + held) > 150 << 20 and PART * (q_bytes + held) < 150 << 20
    (q, k, v), pos, w = _inputs(dtype, tokens, (hq, hkv, hkv), rotary + 1)
    freq = B.rotary_frequencies(rotary) if rotary else None
    slots = _slots(n_pages, page, tokens, 5)
    caches = [[c.fill_(3) for c in B.alloc_cache(n_pages, hkv, page, q.dtype, mxfp4=True)] for _ in range(2)]
    outs = [torch.full((tokens, hq, 128), float("nan"), dtype=q.dtype, device=DEV) for _ in range(2)]

    def call(s, out, cache):
        p = B.make_cache_params(hq, hkv, q.dtype, q=q[s], k=k[s], v=v[s], out=out[s], k_cache=cache[0], mxfp4=True, rotary_dim=rotary, interleaved=interleaved, norm_eps=1e-5)
        B.critiprefill_norm_rope_write(p, q[s], k[s], v[s], *w, freq, pos[s], slots[s], out[s], *cache)

    call(slice(0, tokens), outs[0], caches[0])
    for s in _parts(tokens):
        call(s, outs[1], caches[1])
    assert _same(*outs) and all(_same(a, b) for a, b in zip(*caches))


@pytest.mark.parametrize("dtype,tokens", [("bf16", 34001), ("fp32", 17501)])
def test_write_and_read_past_the_caches(dtype, tokens):
    hkv, page = 8, 64
    row = 128 * (2 if dtype == "bf16" else 4) + 64
    assert tokens * 2 * hkv * row > 150 << 20 and PART * 2 * hkv * row < 150 << 20 and not streams(dtype, False, PART, 2 * hkv, 0)
    (k, v), _, _ = _inputs(dtype, tokens, (hkv, hkv), 7)
    n_pages = tokens // page + 3
    slots = _slots(n_pages, page, tokens, 6)
    caches = [[c.fill_(3) for c in B.alloc_cache(n_pages, hkv, page, k.dtype, mxfp4=True)] for _ in range(2)]
    p = B.make_cache_params(hkv, hkv, k.dtype, k=k, v=v, k_cache=caches[0][0], mxfp4=True)
    B.critiprefill_cache_write(p, k, v, slots, *caches[0])
    for s in _parts(tokens):
        p = B.make_cache_params(hkv, hkv, k.dtype, k=k[s], v=v[s], k_cache=caches[1][0], mxfp4=True)
        B.critiprefill_cache_write(p, k[s], v[s], slots[s], *caches[1])
    assert all(_same(a, b) for a, b in zip(*caches))
    back = _load(caches[0], slots, k.dtype)
    some = torch.arange(0, tokens, 401, device=DEV)
    for x, y in ((k, back[0]), (v, back[1])):
        want = O.mx4_values(*O.mx4_quantise(f64(x[some])))
        want[(slots[some] < 0).cpu().numpy()] = 0.0
        assert np.array_equal(f64(y[some]), want) and not y[slots < 0].any() and torch.isfinite(y).all()
    for s in _parts(tokens):
        assert all(_same(a, b[s]) for a, b in zip(_load(caches[0], slots[s], k.dtype), back))


def test_a_captured_append_follows_positions_and_slots():
    """Replayed with other tokens, positions and places, some of them none; on another stream than the tensors' own; compared with the same call outside of the graph."""
    gen = torch.Generator().manual_seed(4)
    q, k, v = (x.contiguous() for x in side_by_side(gen, 9, (8, 2, 2), "bf16"))
    pos, slots = torch.zeros(9, dtype=torch.int32, device=DEV), torch.arange(9, dtype=torch.int32, device=DEV)
    w, freq = torch.ones(128, dtype=q.dtype, device=DEV), B.rotary_frequencies(64)
    caches = [[c.fill_(7) for c in B.alloc_cache(3, 2, 16, mxfp4=True)] for _ in range(2)]
    outs = [torch.zeros((9, 8, 128), dtype=q.dtype, device=DEV) for _ in range(2)]
    p = B.make_cache_params(8, 2, q.dtype, q=q, k=k, v=v, out=outs[0], k_cache=caches[0][0], mxfp4=True, rotary_dim=64, norm_eps=1e-6)

    def call(i, stream=None):
        B.critiprefill_norm_rope_write(p, q, k, v, w, w, freq, pos, slots, outs[i], *caches[i], stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(0)
    torch.cuda.current_stream().wait_stream(side)
    for c in caches[0]:
        c.fill_(7)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(0)
    for step in range(4):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=gen))
        pos.copy_(torch.randint(0, 1 << 20, (9,), generator=gen))
        slots.copy_(torch.cat([torch.randperm(48, generator=gen)[:7], torch.tensor([-1, 48])]))
        graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        call(1, side)
        side.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(*outs) and all(torch.equal(a, b) for a, b in zip(*caches)), step
