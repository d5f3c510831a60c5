"""Attention over pages of 8 bits where sizes are far from one: queries, keys and scales near the ends of fp32."""
import math

import pytest

from tests.test_gpu_pages8 import _cache, _check, _reference

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("kv", ["i8", "e4m3"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("keys,queries,scale", [
    (3e-36, 6e37, 0.0), (1e-35, 6e37, 1e-2), (3e-36, 1.0, 3e36),         # q . K' over codes is too large, the score is not
    (3e36, 1e-37, 0.0), (7e37, 1.4e-38, 0.0), (7e37, 1e-40, 0.0),       # the power of two that brings q to 2^14 is larger than a normal number's inverse
    (1e-25, 1e-14, 3e38), (1e-30, 1e-9, 3e38),                          # scale log2(e) is larger than fp32 holds
    (7e37, 1e0, 1e-38), (1e30, 1e15, -1e-45)])                          # ... smaller than a normal number
def test_scores_that_fp32_holds_are_right_whatever_they_are_made_of(kv, hd, keys, queries, scale):
    """Scores of 1e-3 to 2e2 in size from factors whose products, taken in some order, are too large or too small for fp32.  The bound is the suite's for ordinary ones: every factor is exact or rounds once.
    (The ones in front of the weights, q in two halves, have 22 bits where q is a normal number; below that q has fewer, and is taken as it is.)"""
    import torch
    lens = [70, 300, 1000]
    cache, g = _cache(lens, 2, 2, hd, kv, 16, seed=19, garbage=True)
    cache.k_scales.mul_(keys)
    q = (torch.empty(3, 4, hd, dtype=torch.float64, device=DEV).normal_(generator=g) * queries).float()
    out = cache.attend(0, q, scale=scale)
    used = torch.tensor(scale, dtype=torch.float32).double().item() or 1 / math.sqrt(hd)
    _check(out, *_reference(cache, q.double(), lens, scale=used))
