"""GPU: the autograd functions under create_graph, and graphs that keep tensors which a later call writes."""
import pytest
import torch

from paper_2606_15682_amd import reqat

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _cases():
    g = torch.Generator().manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=g)
    y = torch.tensor([1, 0, 7, 3], dtype=torch.int32, device=DEV)
    f = torch.full((4,), -2.0, device=DEV)
    return {"policy": ([rand(4, 40)], lambda z: reqat.PolicyLoss.apply(z, y, f, f)),
            "sem": ([rand(4, 4096).bfloat16()], lambda z: reqat.SemLoss.apply(z, y, 0.1)),
            "norm": ([rand(4, 40), rand(40), rand(40)], lambda x, w, b: reqat.LayerNorm.apply(x, w, b)),
            "embedding": ([rand(9, 40)], lambda t: reqat.Embedding.apply(y, t, 2.0))}


@pytest.mark.parametrize("name", ["policy", "sem", "norm", "embedding"])
def test_create_graph(name):
    values, f = _cases()[name]
    leaves = [v.to(DEV).requires_grad_() for v in values]
    out = f(*leaves)
    loss = (out * out).sum()
    first = torch.autograd.grad(loss, leaves, retain_graph=True)
    again = torch.autograd.grad(loss, leaves, create_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    with pytest.raises(RuntimeError, match="no second derivative"):
        sum((g.float() ** 2).sum() for g in again).backward()


def test_a_step_between_forward_and_backward():
    w = torch.ones(64, device=DEV, requires_grad=True)
    x = torch.randn((5, 64), generator=torch.Generator().manual_seed(2)).to(DEV).requires_grad_()
    opt = reqat.AdamW([w], 1e-3)
    kept = reqat.LayerNorm.apply(x, w).sum()
    opt.step([torch.ones(64, device=DEV)])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        kept.backward()
    reqat.LayerNorm.apply(x, w).sum().backward()          # a graph made after the step
    assert w.grad is not None and x.grad is not None
