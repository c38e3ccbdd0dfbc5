"""Temperatures as large as there are: every finite one has a distribution (all tokens about as likely in the end)."""
import math

import pytest
import torch

from paper_2605_13907_amd import binding as B
from tests.test_gpu_sample import check, logits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.AisContext()
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [9, 3001, 40_000])
@pytest.mark.parametrize("temperature", [1e10, 2.9e38, 3.2e38, torch.finfo(torch.float32).max])
def test_large_temperatures(ctx, dtype, vocab, temperature):
    z, e = logits(5, vocab, dtype, 97)
    for limits in (dict(), dict(top_k=5), dict(top_p=0.9), dict(min_p=0.1), dict(top_k=4500, top_p=0.7), dict(top_p=0.6, min_p=0.5)):
        got = check(ctx, z, e, temperature=temperature, **limits)
        assert (got >= 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("limits", [dict(top_k=19_999, top_p=0.9), dict(top_p=0.97), dict(top_k=9_000, top_p=0.5), dict(top_k=16_000),
                                    dict(top_k=19_999, top_p=0.6, min_p=0.3), dict(top_p=0.3)])
@pytest.mark.parametrize("temperature", [3e7, 1e8, 1e9, 1e12, 1e25, 1e35])
def test_masks_of_several_sizes_at_large_temperatures(ctx, dtype, limits, temperature):
    """Masks that the temperature makes likely tokens, each in its own measure, whatever they have in common as numbers."""
    z, e = logits(4, 20_000, dtype, 101)
    z[0, 8_000:] = -1e10
    z[0, 14_000:] = -1e20
    z[1, ::2] = -5e9
    z[1, ::3] = -1e12
    z[1, ::5] = -1e30
    z[2, 3_000:] = -1e30
    z[2, 9_000:] = torch.finfo(dtype).min
    z[3, ::3] = -4.5e9
    z[3, 1::3] = -math.inf
    check(ctx, z, e, temperature=temperature, **limits)
