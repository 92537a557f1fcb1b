"""CPU-side checks of the cache of 4 bits: the oracle's own format, the refusals of the library before any launch, and of the binding."""
import ctypes
import re
import types

import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2409_12490_amd import binding as B
from tests import test_cache_abi as A


def _params(**kw):
    return A._params(**dict({"cache_format": B.CP_CACHE_MXFP4}, **kw))


HELD = [A.rope_write, A.write, A.read, A.attn]


def test_the_oracles_format_by_enumeration():
    """Every multiple of 1/16 of a unit within the range of a block, and its neighbours, against the nearest value by brute force."""
    levels = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    grid = np.arange(0, 7 * 16 + 1) / 16
    points = np.unique(np.concatenate([grid, grid * (1 + 2.0 ** -20), grid * (1 - 2.0 ** -20)]))
    points = np.concatenate([points[points <= 7.0], -points[points <= 7.0]])
    for x in points:
        row = np.zeros((1, 128))
        row[0, 0], row[0, 1] = 7.0, x
        held, e = O.mx4_quantise(row)
        best = min(range(8), key=lambda c: (abs(levels[c] - abs(x)), c % 2))
        assert e[0, 0] == 127 and held[0, 0] & 15 == 7 and held[0, 0] >> 4 == best + (8 if np.signbit(x) else 0), x
        assert O.mx4_values(held, e)[0, 1] == np.copysign(levels[best], x)
        # the next scale would not be nearer, in the worst case of its steps: half of one is 1 unit from 4 on and 0.5 and 0.25 below
        assert abs(levels[best] - abs(x)) <= (0.25 if abs(x) <= 2 else 0.5 if abs(x) <= 4 else 1.0)


def test_the_oracles_scales():
    x = np.zeros((9, 128))
    x[0, 0], x[1, 0], x[2, 0], x[3, 0] = 7.0, np.nextafter(7.0, 8), 3.5, 2.0 ** -126
    x[4, 0], x[5, 0], x[6, 5], x[7, 70] = 3.4e38, 2.0 ** -149, np.inf, np.nan
    e = O.mx4_scale(x)
    assert e[:, 0].tolist() == [127, 128, 126, 2, 252, 2, 255, 2, 2] and e[7].tolist() == [2, 2, 255, 2]
    held, e = O.mx4_quantise(x)
    v = O.mx4_values(held, e)
    assert v[4, 0] == 6 * 2.0 ** 125 and v[4, 0] < np.finfo(np.float32).max and v[3, 0] == 2.0 ** -126 and v[5, 0] == 0
    assert np.isnan(v[6, :32]).all() and not held[6].any() and np.isnan(v[7, 64:96]).all() and np.isfinite(v[7, :64]).all()


@pytest.mark.parametrize("fmt", [2, 3, 5, -1, 8])
def test_other_formats_are_refused(fmt):
    for f in HELD:
        assert f(_params(cache_format=fmt)) == -3


@pytest.mark.parametrize("kw,code", [(dict(page_size=8), -3), (dict(page_size=48), -3), (dict(n_pages=0), -2), (dict(n_pages=1 << 25), -3), (dict(head_dim=64), -3), (dict(dtype=2), -3),
                                     (dict(tokens=-1), -2), (dict(n_kv_heads=0), -2)])
def test_bad_sizes_are_refused_before_launch(kw, code):
    for f in HELD:
        assert f(_params(**kw)) == code, f.__name__
    assert B.critiprefill_paged_workspace_bytes(_params(**kw)) == 0


def test_pages_and_scales_are_needed_and_aligned():
    for f in HELD:
        for name in ("kc", "vc", "ks", "vs"):
            assert f(_params(), **{name: None}) == -1 and f(_params(), **{name: A.ODD}) == -4, (f.__name__, name)


def test_nothing_to_do_is_no_error():
    nothing = _params(tokens=0)
    assert A.rope_write(nothing, *[None] * 13) == A.write(nothing, *[None] * 7) == A.read(nothing, *[None] * 7) == 0
    assert A.attn(nothing, *[None] * 11, 0) == 0 and A.attn(_params(n_seqs=0), *[None] * 11, 0) == 0


def test_workspace_goes_by_heads_type_and_the_longest_chunk():
    for dtype in (B.CP_DTYPE_FP32, B.CP_DTYPE_BF16):
        for heads in (2, 8, 40, 128):
            for longest in (1, 7, 300):
                sizes = {B.critiprefill_paged_workspace_bytes(_params(dtype=dtype, n_q_heads=heads, max_q_len=longest, n_seqs=n, max_pages=m, max_kv_len=v))
                         for n in (1, 9, 500) for m in (1, 30, 1000) for v in (0, 50, 3000)}
                assert len(sizes) == 1 and min(sizes) > 0
                p = _params(dtype=dtype, n_q_heads=heads, max_q_len=longest)
                s = p.q_stride
                s[0] = p.o_stride[0] = heads * 128
                assert A.attn(p, ws_bytes=min(sizes) - 1) == -5


def test_binding_refuses_pages_that_do_not_fit():
    bf16, n = torch.bfloat16, 5
    q, k, ints = torch.zeros(n, 8, 128, dtype=bf16), torch.zeros(n, 2, 128, dtype=bf16), torch.zeros(n + 1, dtype=torch.int32)
    table, ws, w, freq = torch.zeros(n, 3, dtype=torch.int32), torch.zeros(1 << 20, dtype=torch.uint8), torch.ones(128, dtype=bf16), B.rotary_frequencies(64, device="cpu")
    cache = B.alloc_cache(3, 2, 16, mxfp4=True, device="cpu")
    assert [tuple(c.shape) for c in cache] == [(3, 2, 16, 64)] * 2 + [(3, 2, 16, 4)] * 2 and all(c.dtype == torch.uint8 for c in cache)
    with pytest.raises(ValueError):
        B.alloc_cache(3, 2, 16, mxfp8=True, mxfp4=True, device="cpu")
    with pytest.raises(ValueError):
        B.make_cache_params(8, 2, bf16, k_cache=cache[0], mxfp8=True, mxfp4=True)
    with pytest.raises(ValueError):
        B.make_cache_params(8, 2, bf16, k_cache=cache[0], mxfp8=True)
    with pytest.raises(ValueError):
        B.make_cache_params(8, 2, bf16, k_cache=torch.zeros(3, 2, 16, 128, dtype=torch.uint8), mxfp4=True)
    with pytest.raises(TypeError):
        B.make_cache_params(8, 2, bf16, k_cache=torch.zeros(3, 2, 16, 64, dtype=bf16), mxfp4=True)
    p = B.make_cache_params(8, 2, bf16, q=q, k=k, v=k, out=q, k_out=k, k_cache=cache[0], mxfp4=True, page_table=table, rotary_dim=64)
    st = types.SimpleNamespace(cuda_stream=None)                    # nothing here is on a GPU, and the library is not to get as far as a launch
    calls = {"rope_write": lambda t: B.critiprefill_norm_rope_write(p, q, k, k, w, w, freq, ints, ints, q, *t, stream=st), "write": lambda t: B.critiprefill_cache_write(p, k, k, ints, *t, stream=st),
             "read": lambda t: B.critiprefill_cache_read(p, ints, *t, k, k, stream=st), "attn": lambda t: B.critiprefill_paged_attn(p, q, *t, table, ints, ints, q, None, ws, stream=st)}
    for call in calls.values():
        for i, good in enumerate(cache):
            for bad in (good[:-1], good.to(torch.float16), good.to(bf16), torch.stack([good, good], -1)[..., 0]):
                with pytest.raises(ValueError):
                    call([bad if j == i else c for j, c in enumerate(cache)])
        with pytest.raises(B.CritiPrefillError) as e:
            call([cache[0], cache[1], None, cache[3]])
        assert e.value.status == -1


def test_no_two_kernels_that_differ_in_nothing():
    """The last argument of both kernels says whether tensors go past the caches.  fp32 written into 4 bits never does, what is read back from there always; the other forms are not built."""
    with open(B.lib_path(), "rb") as f:
        built = f.read()
    # a kernel's name in the library: <element type, TURN_NONE, TO_MXFP4, past the caches>, <element type, HELD_MXFP4, past the caches>
    forms = lambda name: {m.group(1).decode() for m in re.finditer(name.encode() + rb"ELb([01])EEE", built)}                                                       # noqa: E731
    assert forms("norm_rope_kernelIfLi0ELi3") == {"0"} and forms("norm_rope_kernelIDF16bLi0ELi3") == {"0", "1"}
    assert forms("cache_read_kernelIfLi2") == {"1"} and forms("cache_read_kernelIDF16bLi2") == {"1"}
