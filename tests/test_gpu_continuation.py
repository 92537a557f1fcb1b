"""The example that takes a layer from its prefill through a follow-up to single tokens: its rows over the cache against dense attention over what went into it."""
import pytest
import torch

from paper_2409_12490_amd import continuation

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mxfp8,bound", [(False, 8e-3), (True, 8e-2)])
def test_a_layer_past_its_prefill(mxfp8, bound):
    # Relative, 2-norm.  bf16: P and O rounded in both, 2^-8 / sqrt(3) each at most.  8 bits: values of e4m3, half a step is 2^-4 relative at most and 2^-5 in the mean square
    # over keys and values each, smaller in the sums over keys
    found = continuation.run(prompt=1500, follow=130, steps=3, mxfp8=mxfp8, verbose=False)
    assert found["finite"] and found["held"] == 1500 + 130 + 3 and found["off"] <= bound


@pytest.mark.parametrize("mxfp8,bound", [(False, 8e-3), (True, 8e-2)])
def test_every_captured_step_is_at_its_own_place(mxfp8, bound):
    """Tokens whose values are a hundred times those of the prompt: of 300 to 340 keys, each of a weight of its own order, theirs are most of the sum, so that a step that does not see its own or an
    earlier one, or sees one twice, is off by about 1 / sqrt(40) and more.  Bounds as above: 8 bits, half a step of e4m3 in the mean square is 2^-5 of a value at most, of K likewise."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    heads = continuation.HQ + 2 * continuation.HKV
    qkv = torch.randn((300, heads, 128), generator=gen, device="cuda").bfloat16()
    tokens = torch.randn((40, heads, 128), generator=gen, device="cuda")
    tokens[:, -continuation.HKV:] *= 100.0
    tokens = tokens.bfloat16()
    layer = continuation.Layer(340, mxfp8)
    _, kr = layer.prefill(qkv)
    outs, us = continuation.decode(layer, tokens)
    want = continuation._dense_rows(layer, kr, qkv, tokens).float()
    assert layer.held == 340 and len(us) == 40 and outs.shape == want.shape
    for i, (got, w) in enumerate(zip(outs.float(), want)):
        assert float((got - w).norm() / w.norm()) <= bound, i
    blind = tokens.clone()
    blind[:, -continuation.HKV:] = 0
    missed = (continuation._dense_rows(layer, kr, qkv, blind).float() - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)
    assert (missed > 0.5).all()                                     # what the tokens behind the prompt are of a row


def test_the_example_says_how_far_its_steps_are_off():
    found = continuation.run(prompt=700, follow=40, steps=4, verbose=False)
    assert len(found["step_off"]) == 4 and max(found["step_off"]) <= 8e-2
