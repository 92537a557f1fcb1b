"""The example that takes a layer from its prefill through a follow-up to single tokens: its rows over the cache against dense attention over what went into it."""
import pytest

from paper_2409_12490_amd import continuation

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mxfp8,bound", [(False, 8e-3), (True, 8e-2)])
def test_a_layer_past_its_prefill(mxfp8, bound):
    # Relative, 2-norm.  bf16: P and O rounded in both, 2^-8 / sqrt(3) each at most.  8 bits: values of e4m3, half a step is 2^-4 relative at most and 2^-5 in the mean square
    # over keys and values each, smaller in the sums over keys
    found = continuation.run(prompt=1500, follow=130, steps=3, mxfp8=mxfp8, verbose=False)
    assert found["finite"] and found["held"] == 1500 + 130 + 3 and found["off"] <= bound
