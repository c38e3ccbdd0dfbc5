"""Which of its two forms a call of the preference loss through logits takes, and what it hands on: decided on the host, without a GPU."""
import torch
import pytest

from paper_2605_13907_amd import binding as B

Z, IDS, VALID, CU = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32), torch.ones(4, dtype=torch.uint8), torch.tensor([0, 2, 4])
LOGP, LSE, REF, WEIGHT = (torch.full((n,), float(n)) for n in (4, 4, 4, 1))


@pytest.fixture
def ctx(monkeypatch):
    c = object.__new__(B.AisContext)
    c.device = torch.device("cpu")
    monkeypatch.setattr(B, "_logits_geometry", lambda z, device=None, name="logits": (z.shape[0], z.shape[1], z.stride(0)))
    seen = []

    def through(logits, token_ids, valid, cu_rows, logp_ref, params=None, weight=None, want_grad=True, dlogits=None):
        seen[:] = [logits, token_ids, valid, cu_rows, logp_ref, params, weight, want_grad, dlogits]
        return "loss", "reward", "logp", "dlogits"

    c._preference_through_logits = through
    c.seen = seen
    return c


def alike(a, b):
    return len(a) == len(b) and all(x is y for x, y in zip(a, b))


def test_without_log_probs(ctx):
    p = B.AisPreferenceParams()
    four = ("loss", "reward", "logp", "dlogits")
    assert ctx.preference_loss_grad(Z, IDS, VALID, CU, REF) == four and alike(ctx.seen, [Z, IDS, VALID, CU, REF, None, None, True, None])
    assert ctx.preference_loss_grad(Z, IDS, VALID, CU, None, p, WEIGHT, False, Z) == four
    assert alike(ctx.seen, [Z, IDS, VALID, CU, None, p, WEIGHT, False, Z])
    assert ctx.preference_loss_grad(Z, IDS, None, CU, logp_ref=REF, params=p, weight=WEIGHT, want_grad=False) == four
    assert alike(ctx.seen, [Z, IDS, None, CU, REF, p, WEIGHT, False, None])


def test_with_log_probs(ctx):
    p = B.AisPreferenceParams()
    three = ("loss", "reward", "dlogits")
    assert ctx.preference_loss_grad(Z, IDS, VALID, CU, LOGP, LSE, REF) == three
    assert alike(ctx.seen, [Z, IDS, VALID, CU, REF, None, None, True, None])
    assert ctx.preference_loss_grad(Z, IDS, VALID, CU, LOGP, LSE, REF, p, weight=WEIGHT) == three
    assert alike(ctx.seen, [Z, IDS, VALID, CU, REF, p, WEIGHT, True, None])
    assert ctx.preference_loss_grad(Z, IDS, VALID, CU, LOGP, LSE, None, p, WEIGHT, Z) == three
    assert alike(ctx.seen, [Z, IDS, VALID, CU, None, p, WEIGHT, True, Z])
    assert ctx.preference_loss_grad(Z, IDS, VALID, CU, logp_train=LOGP, lse=LSE, logp_ref=REF) == three


@pytest.mark.parametrize("wrong", [LOGP.double(), LOGP[:3], torch.stack((LOGP, LOGP), 1)[:, 0], None, 1.0])
def test_their_form_is_checked(ctx, wrong):
    for args in (dict(logp_train=wrong, lse=LSE), dict(logp_train=LOGP, lse=wrong)):
        with pytest.raises((TypeError, ValueError), match="logp_train" if args["lse"] is LSE else "lse"):
            ctx.preference_loss_grad(Z, IDS, VALID, CU, **args, logp_ref=REF)
    assert not ctx.seen
