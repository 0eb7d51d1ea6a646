"""LayerFew's refusals that need no device: tensors that do not belong together."""
import pytest
import torch

from paper_2608_28511_amd import _lib as L
from paper_2608_28511_amd import layer


@pytest.fixture(scope="module", autouse=True)
def lib():
    return L.load(build_if_missing=True)


def bf(*s):
    return torch.zeros(s, dtype=torch.bfloat16)


def f32(*s):
    return torch.zeros(s)


OK = dict(S=4, Wr=f32(32, 8), W1=bf(8, 32, 48), W2=bf(8, 48, 32), K=2)
SHARED = dict(Ws1=bf(32, 16), Ws2=bf(16, 32))


@pytest.mark.parametrize("bad", [
    dict(SHARED, ss1=f32(16)), dict(SHARED, ss2=f32(32)), dict(SHARED, ss1=f32(16), ss2=f32(32)), dict(s2=f32(8, 32)),
    dict(ss2=f32(32)), dict(Ws1=bf(32, 16))])
def test_scales_without_8_bit_weights(bad):
    """At the layer's construction, not at its first call."""
    with pytest.raises(ValueError, match="must be given together"):
        layer.LayerFew(**{**OK, **bad})
