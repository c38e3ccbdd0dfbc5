"""Temperatures as large as there are: every finite one has a distribution (all tokens about as likely in the end)."""
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
