"""CPU-side checks of the cache operators: the oracle's own format, the refusals of the library before any launch, and of the binding."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2409_12490_amd import binding as B

OK, ODD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10004)      # never dereferenced: the checks come first


def _params(**kw):
    p = B.CacheParams()
    p.n_q_heads, p.n_kv_heads, p.head_dim, p.dtype, p.tokens = 8, 2, 128, B.CP_DTYPE_BF16, 10
    p.cache_format, p.page_size, p.n_pages, p.n_seqs, p.max_pages, p.max_q_len = B.CP_CACHE_MXFP8, 64, 100, 3, 20, 4
    p.rotary_dim, p.norm_eps = 128, 1e-5
    for name, heads in (("q", 8), ("k", 2), ("v", 2), ("o", 8), ("ko", 2)):
        s = getattr(p, name + "_stride")
        s[0], s[1] = heads * 128, 128
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _strided(name, token, head, **kw):
    p = _params(**kw)
    s = getattr(p, name + "_stride")
    s[0], s[1] = token, head
    return p


def rope(p, q=OK, k=OK, qw=OK, kw=OK, f=OK, pos=OK, qo=OK, ko=OK):
    return B.load().critiprefill_norm_rope(ctypes.byref(p) if p else None, q, k, qw, kw, f, pos, qo, ko, None)


def rope_write(p, q=OK, k=OK, v=OK, qw=OK, kw=OK, f=OK, pos=OK, slots=OK, qo=OK, kc=OK, vc=OK, ks=OK, vs=OK):
    return B.load().critiprefill_norm_rope_write(ctypes.byref(p) if p else None, q, k, v, qw, kw, f, pos, slots, qo, kc, vc, ks, vs, None)


def write(p, k=OK, v=OK, slots=OK, kc=OK, vc=OK, ks=OK, vs=OK):
    return B.load().critiprefill_cache_write(ctypes.byref(p) if p else None, k, v, slots, kc, vc, ks, vs, None)


def read(p, k=OK, v=OK, slots=OK, kc=OK, vc=OK, ks=OK, vs=OK):
    return B.load().critiprefill_cache_read(ctypes.byref(p) if p else None, slots, kc, vc, ks, vs, k, v, None)


def attn(p, q=OK, kc=OK, vc=OK, ks=OK, vs=OK, table=OK, start=OK, kv=OK, out=OK, lse=OK, ws=OK, ws_bytes=1 << 40):
    return B.load().critiprefill_paged_attn(ctypes.byref(p) if p else None, q, kc, vc, ks, vs, table, start, kv, out, lse, ws, ws_bytes, None)


EVERY = [rope, rope_write, write, read, attn]


@pytest.mark.parametrize("kw,code,of", [
    (dict(n_kv_heads=0), -2, EVERY), (dict(tokens=-1), -2, EVERY), (dict(head_dim=64), -3, EVERY), (dict(dtype=2), -3, EVERY), (dict(dtype=-1), -3, EVERY),
    (dict(n_kv_heads=65536), -3, [write, read]),
    (dict(n_q_heads=7), -2, [rope, rope_write, attn]), (dict(n_q_heads=0), -2, [rope, rope_write, attn]),
    (dict(page_size=0), -2, [rope_write, write, read, attn]), (dict(page_size=8), -3, [rope_write, write, read, attn]),
    (dict(page_size=48), -3, [rope_write, write, read, attn]), (dict(n_pages=0), -2, [rope_write, write, read, attn]),
    (dict(n_pages=1 << 25), -3, [rope_write, write, read, attn]), (dict(cache_format=2), -3, [rope_write, write, read, attn]),
    (dict(rotary_dim=-16), -2, [rope, rope_write]), (dict(rotary_dim=144), -2, [rope, rope_write]), (dict(rotary_dim=24), -3, [rope, rope_write]),
    (dict(norm_eps=-1.0), -2, [rope, rope_write]), (dict(norm_eps=float("nan")), -2, [rope, rope_write]),
    (dict(n_seqs=-1), -2, [attn]), (dict(max_pages=-1), -2, [attn]), (dict(max_q_len=-1), -2, [attn]), (dict(max_kv_len=-1), -2, [attn]), (dict(attn_scale=-1.0), -2, [attn]),
    (dict(attn_scale=float("nan")), -2, [attn]), (dict(n_q_heads=130), -3, [attn]), (dict(max_pages=1 << 24), -3, [attn]),
    (dict(tokens=1 << 30, max_pages=1 << 20), -3, [attn]),
])
def test_bad_sizes_are_refused_before_launch(kw, code, of):
    for f in of:
        assert f(_params(**kw)) == code, f.__name__
    if attn in of:
        assert B.critiprefill_paged_workspace_bytes(_params(**kw)) == 0


@pytest.mark.parametrize("heads", [70000, 2 ** 31 - 1, -1, 0, 7])
def test_write_and_read_do_not_look_at_the_query_heads(heads):
    for f in (write, read):
        assert f(_params(n_q_heads=heads), slots=None) == -1                             # past the checks of sizes: the next refusal is another one


@pytest.mark.parametrize("f", EVERY, ids=lambda f: f.__name__)
def test_null_and_misaligned_arguments(f):
    assert f(None) == -1
    optional = {"qw", "kw", "lse"}
    names = [n for n in f.__code__.co_varnames[1:f.__code__.co_argcount] if n != "ws_bytes"]
    for name in names:
        assert f(_params(), **{name: None}) == -1 if name not in optional else True, name
        byte = ctypes.c_void_p(0x10001)
        assert f(_params(), **{name: byte}) == -4, name
    for name in set(names) - {"slots", "pos", "table", "start", "kv", "lse"}:            # these need 4 bytes, f 8, tensors 16
        assert f(_params(), **{name: ODD}) == -4, name


def test_strides():
    for f, tensors in ((rope, "q k o ko"), (rope_write, "q k v o"), (write, "k v"), (read, "k v"), (attn, "q o")):
        for t in tensors.split():
            assert f(_strided(t, 1028, 128)) == -4 and f(_strided(t, 1024, 132)) == -4 and f(_strided(t, -1024, 128)) == -4
            if t in ("o", "ko") or f is read:
                assert f(_strided(t, 0, 128)) == -2 and f(_strided(t, 1024, 64)) == -2
                heads = 8 if t == "o" else 2
                assert f(_strided(t, heads * 128 - 8, 128)) == -2 and f(_strided(t, 128, 10 * 128 - 8)) == -2      # rows that share elements
                past = {rope: dict(q=ODD), rope_write: dict(slots=None), read: dict(slots=None), attn: dict(ws_bytes=16)}[f]
                assert f(_strided(t, 128, 10 * 128), **past) != -2 and f(_strided(t, heads * 128 + 8, 128), **past) != -2


def test_plain_pages_need_no_scales_and_no_rotation_needs_no_angles():
    # past the checks of these, the next refusal is another one
    assert write(_params(cache_format=B.CP_CACHE_PLAIN), ks=None, vs=None, slots=None) == -1
    assert attn(_params(cache_format=B.CP_CACHE_PLAIN), ks=None, vs=None, ws_bytes=16) == -5
    assert rope(_params(rotary_dim=0), f=None, pos=None, ko=ODD) == -4


def test_nothing_to_do_is_no_error():
    nothing = _params(tokens=0)
    assert rope(nothing, *[None] * 8) == rope_write(nothing, *[None] * 13) == write(nothing, *[None] * 7) == read(nothing, *[None] * 7) == 0
    assert attn(nothing, *[None] * 11, 0) == 0 and attn(_params(n_seqs=0), *[None] * 11, 0) == 0


def test_workspace():
    p = _params()
    need = B.critiprefill_paged_workspace_bytes(p)
    assert need > 0 and attn(p, ws_bytes=need - 1) == -5
    # sizes of the lengths do not move it
    assert B.critiprefill_paged_workspace_bytes(_params(n_seqs=100, max_pages=1000)) == need
    for dtype, fmt in ((d, f) for d in (B.CP_DTYPE_FP32, B.CP_DTYPE_BF16) for f in (B.CP_CACHE_PLAIN, B.CP_CACHE_MXFP8)):
        for heads in (2, 8, 40, 128):
            for longest in (1, 7, 300):
                sizes = {B.critiprefill_paged_workspace_bytes(_params(dtype=dtype, cache_format=fmt, n_q_heads=heads, max_q_len=longest, n_seqs=n, max_pages=m, max_kv_len=v))
                         for n in (1, 9, 500) for m in (1, 30, 1000) for v in (0, 50, 3000)}
                assert len(sizes) == 1 and min(sizes) > 0


def test_binding_refuses_what_the_parameter_block_does_not_fit():
    q, k = torch.zeros(5, 8, 128, dtype=torch.bfloat16), torch.zeros(5, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        B.make_cache_params(8, 2, torch.bfloat16, q=q, k=k[:4])
    with pytest.raises(ValueError):
        B.make_cache_params(4, 2, torch.bfloat16, q=q)
    with pytest.raises(TypeError):
        B.make_cache_params(8, 2, torch.float32, q=q)
    with pytest.raises(TypeError):
        B.make_cache_params(8, 2, torch.float16, q=q.half())
    with pytest.raises(ValueError):
        B.make_cache_params(8, 2, torch.bfloat16, q=q.transpose(1, 2).contiguous().transpose(1, 2))
    with pytest.raises(ValueError):
        B.make_cache_params(8, 2, torch.bfloat16, k_cache=torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        B.make_cache_params(8, 2, torch.bfloat16, k_cache=torch.zeros(3, 2, 16, 128, dtype=torch.bfloat16), mxfp8=True)
    p = B.make_cache_params(8, 2, torch.bfloat16, q=q, k=k, rotary_dim=64)
    with pytest.raises(ValueError):                                 # fp32 frequencies lose the turns of far positions
        B.critiprefill_norm_rope(p, q, k, None, None, torch.zeros(32), torch.zeros(5, dtype=torch.int32), q, k)
    with pytest.raises(ValueError):
        B.critiprefill_norm_rope(p, q, k, None, None, torch.zeros(32, dtype=torch.float64), torch.zeros(4, dtype=torch.int32), q, k)


@pytest.mark.parametrize("mxfp8", [False, True], ids=["plain", "mxfp8"])
def test_binding_refuses_tensors_of_which_the_library_sees_an_address(mxfp8):
    """Pages, scales and weights of another type, too small or not contiguous, and q, k, v and outputs of fewer rows than the block says.  The library must not be reached:
    nothing here is on a GPU."""
    bf16, n = torch.bfloat16, 5
    q, k, ints = torch.zeros(n, 8, 128, dtype=bf16), torch.zeros(n, 2, 128, dtype=bf16), torch.zeros(n + 1, dtype=torch.int32)
    table, ws, w, freq = torch.zeros(n, 3, dtype=torch.int32), torch.zeros(1 << 20, dtype=torch.uint8), torch.ones(128, dtype=bf16), B.rotary_frequencies(64, device="cpu")
    cache = B.alloc_cache(3, 2, 16, mxfp8=mxfp8, device="cpu")
    p = B.make_cache_params(8, 2, bf16, q=q, k=k, v=k, out=q, k_out=k, k_cache=cache[0], mxfp8=mxfp8, page_table=table, rotary_dim=64)
    names = dict(q=q, k=k, v=k, qw=w, kw=w, q_out=q, k_out=k, kc=cache[0], vc=cache[1], ks=cache[2], vs=cache[3])

    def calls(t):
        pool = (t["kc"], t["vc"], t["ks"], t["vs"])
        return {"rope": lambda: B.critiprefill_norm_rope(p, t["q"], t["k"], t["qw"], t["kw"], freq, ints, t["q_out"], t["k_out"]),
                "rope_write": lambda: B.critiprefill_norm_rope_write(p, t["q"], t["k"], t["v"], t["qw"], t["kw"], freq, ints, ints, t["q_out"], *pool),
                "write": lambda: B.critiprefill_cache_write(p, t["k"], t["v"], ints, *pool),
                "read": lambda: B.critiprefill_cache_read(p, ints, *pool, t["k"], t["v"]),
                "attn": lambda: B.critiprefill_paged_attn(p, t["q"], *pool, table, ints, ints, t["q_out"], None, ws)}

    takes = {"rope": "q k qw kw q_out k_out", "rope_write": "q k v qw kw q_out kc vc ks vs", "write": "k v kc vc ks vs", "read": "k v kc vc ks vs", "attn": "q q_out kc vc ks vs"}
    for call, args in takes.items():
        for name in args.split():
            good = names[name]
            if good is None:
                continue
            bad = [good[:-1]]                                                            # a page, a row or a channel less
            if name in ("qw", "kw", "kc", "vc", "ks", "vs"):
                bad += [good.to(torch.float16), good.to(torch.float32), torch.stack([good, good], -1)[..., 0]]
            for b in bad:
                with pytest.raises(ValueError):
                    calls(dict(names, **{name: b}))[call]()


def test_the_oracles_format_against_torch():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 128)) * 2.0 ** rng.integers(-20, 20, (50, 1))
    x[0] = 0.0
    x[1, :32] = [448.0] + [0.0] * 31
    x[2, :32] = [448.5] + [1.0] * 31
    codes, e = O.mx_quantise(x)
    assert (e[0] == 1).all() and e[1, 0] == 127 and e[2, 0] == 128
    units = torch.from_numpy(x.reshape(50, 4, 32) * 2.0 ** (127.0 - e.astype(np.float64))[..., None]).float()
    assert (torch.from_numpy(x).float().double() == torch.from_numpy(x)).float().mean() < 1         # doubles: round once in both
    x32 = units.to(torch.float8_e4m3fn)
    mine = torch.from_numpy(codes.reshape(50, 4, 32)).view(torch.float8_e4m3fn).float()
    assert ((mine - x32.float()).abs() <= x32.float().abs() * 2.0 ** -3).all() and (mine == x32.float()).float().mean() > 0.9999
    back = O.mx_values(codes, e)
    block = np.abs(x).reshape(50, 4, 32).max(-1, keepdims=True) * np.ones(32)
    assert (np.abs(back - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -17 * block.reshape(x.shape)).all()
