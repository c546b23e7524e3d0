"""A decoder's rotated layers on the GPU: refusals before anything is written, and layers against their operators."""
import math

import pytest
import torch

from .test_gpu_decoder_fp4 import BF16, DEV, build

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [-1.0, -1e-30, math.nan, -math.inf])
@pytest.mark.parametrize("cache_bits", [4, 8])
def test_a_later_layers_eps_is_refused_before_a_cache_is_written(eps, cache_bits):
    make, _, _, _, rng = build(4, 2, 64, 4, 2, 16, 128, BF16, 2, 40, 16, 0, cache_bits=cache_bits)
    model = make()
    x = torch.randn(2, 3, 64, generator=torch.Generator().manual_seed(1)).to(DEV, BF16)
    model(x)
    kept = [t.view(torch.uint8).clone() for c in model.caches for t in c]
    model.layers[1].rotary.eps = eps
    with pytest.raises(ValueError):
        model(x * 100)
    assert model.length.tolist() == [3, 3]
    assert all(torch.equal(a, b.view(torch.uint8)) for a, b in zip(kept, (t for c in model.caches for t in c)))
