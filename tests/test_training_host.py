"""The differentiable router's calls (CPU only): what its backward pass hands to `route_backward`, with both calls replaced by stand-ins
that note their arguments and compute gate = logits of the first k experts, balance and z = sums of logits."""
import numpy as np
import pytest
import torch

from paper_2606_01007_amd import training


@pytest.fixture
def calls(monkeypatch):
    seen = []

    def route(x, k, fam_off=None, score="softmax", **kw):
        L, N, E = x.shape
        F = 1 if fam_off is None else len(fam_off) - 1
        zero = torch.zeros((F, L))
        out = dict(trace=torch.arange(k, dtype=torch.int16).expand(L, N, k).contiguous(), gate=x[:, :, :k].clone(),
                   norm=x.sum(2), D=torch.zeros((F, L, E), dtype=torch.int32), tokens=zero.int(), balance=zero + x.sum((1, 2)))
        if score == "softmax":
            out["z"] = zero + 2 * x.sum((1, 2))
        return out

    def route_backward(x, trace, norm, fam_off=None, **kw):
        seen.append(dict(kw, fam_off=fam_off))
        return torch.ones_like(x)

    monkeypatch.setattr(training, "route", route)
    monkeypatch.setattr(training, "route_backward", route_backward)
    return seen


def _logits():
    return torch.randn((2, 6, 5), generator=torch.Generator().manual_seed(1)).requires_grad_(True)


@pytest.mark.parametrize("used", ["gate", "balance", "z"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_outputs_that_no_loss_uses_have_no_gradient(calls, score, used):
    x = _logits()
    gate, balance, z, _ = training.balanced_route(x, 2, [0, 6], score=score)
    dict(gate=gate, balance=balance, z=z)[used].sum().backward()
    assert len(calls) == 1
    given = {n for n in ("gate", "balance", "z") if calls[0]["grad_" + n] is not None}
    assert given == ({used} if (score, used) != ("sigmoid", "z") else set())
    assert torch.equal(x.grad, torch.ones_like(x))


def test_a_second_derivative_is_refused(calls):
    """The backward pass runs outside automatic differentiation: a second derivative through it would lack the router's part."""
    x = _logits()
    gate, balance, _, _ = training.balanced_route(x, 2, [0, 6])
    (first,) = torch.autograd.grad((gate * x[:, :, :2]).sum() + balance.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        first.sum().backward()


@pytest.mark.parametrize("make", [list, np.array, torch.tensor])
def test_the_families_are_those_of_the_forward_call(calls, make):
    x = _logits()
    off = make([0, 2, 6])
    gate, balance, z, _ = training.balanced_route(x, 2, off)
    off[1] = 5
    (balance.sum() + z.sum()).backward()
    assert [int(v) for v in calls[0]["fam_off"]] == [0, 2, 6]
