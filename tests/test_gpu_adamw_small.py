"""Steps along gradients whose squares are fp32's subnormal numbers when the root is taken, beside an eps that is smaller still.  Tolerances
are those of the AdamW tests: scaling by powers of two adds no rounding."""
import pytest
import torch

from paper_2605_13907_amd import binding as B
from tests.test_gpu_adamw import Twin, tensor

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.AisContext()
    yield c
    c.close()


@pytest.mark.parametrize("param", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("step", [0, 10 ** 6])
@pytest.mark.parametrize("size", [2e-14, 1e-15, 1e-18, 1.2e-18, 3e-19, 1.1e-19, 5e-20, 1e-20, 1e-21, 4e-22, 1e-22, 1e-23])
def test_small_gradients(ctx, size, step, bits, param):
    """Step 1, whose correction brings v back up, and the millionth, where it is nothing."""
    twin = Twin([tensor(n, param, n) for n in (256, 77)], bits, step=step)
    for sign in (1.0, -0.75, 0.5):
        twin.check_step(ctx, [torch.full((n,), sign * size, device="cuda") for n in (256, 77)], eps=1e-30)


@pytest.mark.parametrize("bits", [32, 8])
def test_magnitudes_side_by_side(ctx, bits):
    """From where squares are normal numbers to where they are 0."""
    twin = Twin([tensor(512, torch.float32, 1)], bits, step=10 ** 6)
    g = 10.0 ** torch.linspace(-24.0, -12.0, 512, dtype=torch.float64, device="cuda")
    for k in range(3):
        twin.check_step(ctx, [(g if k % 2 == 0 else -0.5 * g).float()], eps=1e-30)


def test_a_constant_gradient_steps_by_the_rate(ctx):
    p = torch.zeros(64, device="cuda")
    state = B.AdamWState([p])
    ctx.adamw_step(state, [torch.full((64,), 5e-20, device="cuda")], lr=0.125, beta1=0.0, beta2=0.0, eps=1e-30, weight_decay=0.0)
    # g^2 is 2.5e-39, held to 2^-150 in 2^-128: 2^-22 of the square, half of that of its root
    assert torch.allclose(p, torch.full_like(p, -0.125), rtol=2.0 ** -20, atol=0.0)
