"""The autograd functions have a first derivative: a second one is refused, whatever the incoming gradient depends on.  On CPU
tensors, with plain forms in the kernels' place."""
import pytest
import torch

from paper_2606_15682_amd import reqat


@pytest.fixture(autouse=True)
def plain_forms(monkeypatch):
    def loss(logits, targets, *rest):
        lse = torch.logsumexp(logits.float(), 1)
        lp = logits.float().gather(1, targets[:, None].long())[:, 0] - lse
        return -lp.sum().reshape(1), torch.stack([lp, lse, -torch.ones_like(lp), lp], 1)

    def slope(logits, targets, factor):
        p = torch.softmax(logits.detach().float(), 1)
        p[torch.arange(len(p)), targets.long()] -= 1.0
        return (p * factor).to(logits.dtype)

    def layer_norm(x, w, b, eps, center):
        return x.detach() * w.detach(), torch.zeros(x.shape[0], 2)

    monkeypatch.setattr(reqat, "policy_loss", loss)
    monkeypatch.setattr(reqat, "policy_loss_backward", lambda z, y, stats, temp, g: slope(z, y, g.detach()))
    monkeypatch.setattr(reqat, "sem_loss", lambda z, y, lam, eps: loss(z, y) + (torch.zeros(len(y)),))
    monkeypatch.setattr(reqat, "sem_loss_backward", lambda z, y, s, w, lam, scale, out_dtype: slope(z, y, scale))
    monkeypatch.setattr(reqat, "layer_norm", layer_norm)
    monkeypatch.setattr(reqat, "layer_norm_backward", lambda dy, x, w, stats, center, bias: (
        dy.detach() * w.detach(), (dy * x).detach().sum(0), dy.detach().sum(0) if bias else None))
    monkeypatch.setattr(reqat, "embedding", lambda ids, table, scale: table.detach()[ids.long()] * scale)
    monkeypatch.setattr(reqat, "embedding_backward", lambda dy, ids, rows, scale: torch.zeros(rows, dy.shape[1]).index_add_(
        0, ids.long(), dy.detach() * scale))


Y = torch.tensor([1, 0, 2], dtype=torch.int32)


def _leaf(*shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(1)).requires_grad_()


def _policy():
    z, f = _leaf(3, 5), torch.zeros(3)
    return [z], lambda z: reqat.PolicyLoss.apply(z, Y, f, f)


def _sem():
    return [_leaf(3, 5)], lambda z: reqat.SemLoss.apply(z, Y, 0.1)


def _norm(bias):
    return [_leaf(3, 5), _leaf(5)] + [_leaf(5)] * bias, lambda x, w, b=None: reqat.LayerNorm.apply(x, w, b)


def _embedding():
    return [_leaf(4, 5)], lambda t: reqat.Embedding.apply(Y, t, 2.0)


CASES = {"policy": _policy, "sem": _sem, "norm": lambda: _norm(0), "norm with bias": lambda: _norm(1), "embedding": _embedding}


@pytest.mark.parametrize("linear", [True, False])
@pytest.mark.parametrize("name", list(CASES))
def test_refused(name, linear):
    """linear: the incoming gradient is a constant, and the gradients still depend on the saved inputs."""
    leaves, f = CASES[name]()
    out = f(*leaves)
    loss = out.sum() if linear else (out * out).sum()
    first = torch.autograd.grad(loss, leaves, retain_graph=True)
    again = torch.autograd.grad(loss, leaves, create_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    if name == "embedding" and linear:
        assert not again[0].requires_grad                 # a constant gradient of a lookup is a constant
        return
    for g in again:
        with pytest.raises(RuntimeError, match="no second derivative"):
            # other operations have a second derivative, which alone would be the wrong answer
            torch.autograd.grad((g * g).sum() + sum((x ** 3).sum() for x in leaves), leaves, retain_graph=True)


def test_backward_without_a_graph_is_as_before():
    leaves, f = CASES["norm with bias"]()
    f(*leaves).sum().backward()
    assert all(x.grad is not None and not x.grad.requires_grad for x in leaves)
