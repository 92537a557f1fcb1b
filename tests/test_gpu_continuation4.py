"""The operators on a cache of 4 bits together: a layer's prefill written into it, a follow-up and captured single tokens appended and attended to."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2409_12490_amd import binding as B
from paper_2409_12490_amd import continuation as C
from tests.cache_helpers import DEV, f64

pytestmark = pytest.mark.gpu


def _held(layer):
    return [O.mx4_values(f64(c).astype(np.uint8), f64(s).astype(np.uint8)) for c, s in zip(layer.cache[:2], layer.cache[2:])]


def test_a_layer_past_its_prefill():
    """What attention gives is fp64's over the values that the cache holds: P and the output rounded to bf16, half a step each, 2^-8, and K rounded to bf16 nowhere.  What the cache holds is the
    follow-up's keys and values after norm and rotation, to half a step of e2m1: within a quarter of the value (0.25 of 1, 0.5 of 2, 1 of 4, the largest ratios) or of a unit below 1."""
    gen = torch.Generator(device=DEV).manual_seed(7)
    heads = C.HQ + 2 * C.HKV
    prompt, follow, tokens = ((torch.randn((n, heads, 128), generator=gen, device=DEV)).bfloat16() for n in (700, 90, 5))
    layer = C.Layer(900, mxfp4=True)
    layer.prefill(prompt)
    s = layer.plan(follow)
    layer.place(s)
    out = layer.extend(s).clone()
    steps, _ = C.decode(layer, tokens)
    assert layer.held == 795
    held_k, held_v = _held(layer)
    table = layer.table.cpu().numpy()
    q = torch.empty((95, C.HQ, 128), dtype=torch.bfloat16, device=DEV)
    kn = torch.empty((95, C.HKV, 128), dtype=torch.bfloat16, device=DEV)
    more = torch.cat([follow, tokens])
    p = B.make_cache_params(C.HQ, C.HKV, q.dtype, q=more[:, :C.HQ], k=more[:, C.HQ:C.HQ + C.HKV], out=q, k_out=kn, rotary_dim=128, norm_eps=1e-5)
    pos = torch.arange(700, 795, dtype=torch.int32, device=DEV)
    B.critiprefill_norm_rope(p, more[:, :C.HQ], more[:, C.HQ:C.HQ + C.HKV], *layer.weights, layer.freq, pos, q, kn)
    at = (table[0][np.arange(700, 795) // C.PAGE], slice(None), np.arange(700, 795) % C.PAGE)
    for held, x, rounded in ((held_k[at], f64(kn), 2.0 ** -8), (held_v[at], f64(more[:, C.HQ + C.HKV:]), 0.0)):
        unit = 2.0 ** (O.mx4_scale(x * (1 + 2.0 ** -7)).astype(np.float64) - 127)[..., None] * np.ones(32)
        assert (np.abs(held - x) <= np.maximum(0.25 * np.abs(x), 0.25 * unit.reshape(x.shape)) * (1 + 2.0 ** -6) + rounded * np.abs(x)).all()
    for got, rows, n in ((out, slice(0, 90), 790), *((steps[i:i + 1], slice(90 + i, 91 + i), 791 + i) for i in range(5))):
        want, _, size, _ = O.paged_attention(f64(q[rows]), held_k, held_v, C.PAGE, table, [0, got.shape[0]], [n], 128 ** -0.5)
        assert (np.abs(f64(got) - want) <= 2.0 ** -8 * (size + np.abs(want)) * 1.01 + 2.0 ** -18 * size.max()).all()


def test_the_example_runs_on_4_bits():
    found = C.run(prompt=700, follow=40, steps=4, verbose=False, mxfp4=True)
    # e2m1's half steps are a sixth to a quarter of a value, in the mean square a tenth, of K and of V each: of a row's 2-norm well below a half
    assert found["finite"] and found["held"] == 744 and found["off"] <= 0.5 and max(found["step_off"]) <= 0.5
