"""Tensors of the caller's that a call writes: autograd has to know, or a graph that keeps one runs backward with other
values.  On CPU tensors, with the C calls left out."""
import contextlib

import pytest
import torch

from paper_2606_15682_amd import reqat

BF = torch.bfloat16


@pytest.fixture(autouse=True)
def no_calls(monkeypatch):
    monkeypatch.setattr(reqat, "_call", lambda *a: None)
    monkeypatch.setattr(reqat, "_require_cuda", lambda *a: None)


def _given_outputs():
    z, y, f = torch.zeros(3, 8), torch.zeros(3, dtype=torch.int32), torch.zeros(3)
    x, w, s2, s4 = torch.zeros(3, 8), torch.zeros(8), torch.zeros(3, 2), torch.zeros(3, 4)
    table = torch.zeros(5, 8)
    return {"policy_loss_grad": lambda out: reqat.policy_loss_grad(z, y, f, f, out=out),
            "policy_loss_backward": lambda out: reqat.policy_loss_backward(z, y, s4, out=out),
            "layer_norm": lambda out: reqat.layer_norm(x, w, out=out),
            "layer_norm_backward": lambda out: reqat.layer_norm_backward(x, x, w, s2, out=out, ws=torch.zeros(10 ** 6, dtype=torch.uint8)),
            "embedding": lambda out: reqat.embedding(y, table, out=out),
            "embedding_backward": lambda out: reqat.embedding_backward(x, y, 3, out=out),
            "embedding_backward, added": lambda out: reqat.embedding_backward(x, y, 3, out=out, accumulate=True)}


@pytest.mark.parametrize("name", list(_given_outputs()))
def test_given_outputs(name):
    out = torch.ones(3, 8)
    a = torch.ones(3, 8, requires_grad=True)
    kept = (a * out).sum()                                # keeps out for a's gradient
    before = out._version
    _given_outputs()[name](out)
    assert out._version > before
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        kept.backward()
    with torch.inference_mode():                          # tensors without a counter are taken as before
        _given_outputs()[name](torch.ones(3, 8))


@pytest.mark.parametrize("captured", [False, True])
def test_adamw(captured, monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    p = [torch.nn.Parameter(torch.ones(8)), torch.ones(8), torch.ones(8)]
    copies = [None, torch.ones(8, dtype=BF, requires_grad=True), torch.ones(8, dtype=BF)]
    opt = reqat.AdamW(p, 1e-3, copies=[c if c is None else c.detach() for c in copies], captured=captured)
    x = torch.ones(8, requires_grad=True)
    graphs = [(x * t).sum() for t in (p[0], copies[1], p[2], copies[2])]
    opt.step([torch.ones(8), torch.ones(8), None])
    for i, graph in enumerate(graphs):
        if i < 2:                                         # the copy shares its counter with the leaf it was detached from
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                graph.backward()
        else:
            graph.backward()                              # left out: not written
    if not captured:
        opt.step([None] * 3)
