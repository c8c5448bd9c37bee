"""GPU: a whole training step of a small quantized layer: embedding, norm, fake-quantized products, policy loss, backward,
AdamW on master weights; against plain torch operations, captured in a graph, and on another stream."""
import pytest
import torch

from paper_2606_15682_amd import reqat

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
T, V, D, H = 96, 515, 256, 384
SHAPES = {"table": (V, D), "norm1": (D,), "up": (H, D), "down": (D, H), "norm2": (D,), "bias2": (D,), "head": (V, D)}


def _masters():
    g = torch.Generator().manual_seed(11)
    out = {}
    for name, shape in SHAPES.items():
        x = torch.randn(shape, generator=g) * (0.1 if len(shape) == 1 else shape[1] ** -0.5)
        out[name] = (x + 1.0 if name.startswith("norm") else x).to(DEV)
    return out


def _batch():
    g = torch.Generator().manual_seed(12)
    ids = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    ids[-3:] = -1                                          # a padded batch
    targets = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    weights = torch.full((T,), 1.0 / 60)
    weights[:30] = 0.0
    weights[-3:] = 0.0
    return dict(ids=ids.to(DEV), targets=targets.to(DEV), old=torch.full((T,), -6.3, device=DEV),
                adv=torch.randn(T, generator=g).to(DEV), ref=torch.full((T,), -6.2, device=DEV), weights=weights.to(DEV))


def _loss(w, b, norm, embed, policy):
    x = embed(b["ids"], w["table"])
    h = reqat.FakeQuantSTE.apply(norm(x, w["norm1"], None, 1e-6, False))
    a = torch.nn.functional.silu(h @ reqat.FakeQuantSTE.apply(w["up"]).t())
    y = x + reqat.FakeQuantSTE.apply(a) @ reqat.FakeQuantSTE.apply(w["down"]).t()
    z = norm(y, w["norm2"], w["bias2"], 1e-6, True) @ w["head"].t()
    return policy(z, b["targets"], b["old"], b["adv"], b["ref"], b["weights"], 0.2, 0.2, 0.05, 1.0)


def _own(w, b):
    return _loss(w, b, reqat.LayerNorm.apply, lambda i, t: reqat.Embedding.apply(i, t, 2.0), reqat.PolicyLoss.apply)


def _plain(w, b):
    def norm(x, weight, bias, eps, center):
        z = x.float()
        if center:
            z = z - z.mean(1, keepdim=True)
        y = z * torch.rsqrt((z * z).mean(1, keepdim=True) + eps) * weight.float()
        return (y if bias is None else y + bias.float()).bfloat16()

    def embed(ids, table):
        return torch.where(ids[:, None] >= 0, table[ids.clamp(min=0).long()] * 2.0, 0.0)

    def policy(z, targets, old, adv, ref, weights, low, high, kl, temp):
        lp = torch.log_softmax(z.float() / temp, 1).gather(1, targets[:, None].long())[:, 0]
        r, x = torch.exp(lp - old), ref - lp
        return (weights * (-torch.minimum(r * adv, r.clamp(1 - low, 1 + high) * adv) + kl * (torch.expm1(x) - x))).sum()

    return _loss(w, b, norm, embed, policy)


class Trainer:
    def __init__(self, bits=32, captured=False):
        self.names = list(SHAPES)
        masters = _masters()
        self.masters = [masters[n] for n in self.names]
        self.copies = [m.to(torch.bfloat16).requires_grad_() for m in self.masters]
        self.opt = reqat.AdamW(self.masters, 1e-2, (0.9, 0.95), 1e-8, 0.01, state_bits=bits,
                               copies=[c.detach() for c in self.copies], captured=captured)

    def step(self, b):
        loss = _own(dict(zip(self.names, self.copies)), b)
        grads = torch.autograd.grad(loss, self.copies)
        self.opt.step(grads)
        return loss


def test_gradients_of_the_step():
    b, t = _batch(), Trainer()
    w = dict(zip(t.names, t.copies))
    one, two = _own(w, b), _plain(w, b)
    # both round activations to bfloat16 at the same places; a value that lands on the other side of a rounding moves a
    # quantized block by a step of the 4-bit grid, an eighth of it at most, in few places
    assert abs(float(one) - float(two)) <= 2e-2 * abs(float(two)) + 1e-3
    for n, a, c in zip(t.names, torch.autograd.grad(one, t.copies), torch.autograd.grad(two, t.copies)):
        assert torch.isfinite(a).all()
        assert float((a.float() - c.float()).norm()) <= 0.05 * float(c.float().norm()), n
    unused = torch.ones(V, dtype=torch.bool, device=DEV)
    unused[b["ids"][b["ids"] >= 0].long()] = False
    assert not torch.autograd.grad(_own(w, b), t.copies)[0][unused].any()


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_step_replays_the_eager_one(bits):
    b = _batch()
    eager, graph = Trainer(bits, True), Trainer(bits, True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph.step(b)
    torch.cuda.current_stream().wait_stream(side)
    eager.step(b)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        loss = graph.step(b)
    for k in range(4):
        if k == 2:                                         # another batch in the same buffers
            b["ids"].copy_(b["ids"].roll(5))
            b["adv"].mul_(-1.0)
        want = eager.step(b)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want), k
        for n, p, q, c in zip(eager.names, eager.masters, graph.masters, graph.copies):
            assert torch.equal(p, q) and torch.equal(c, q.to(torch.bfloat16)), (n, k)
        assert torch.equal(eager.opt.m, graph.opt.m) and torch.equal(eager.opt.v, graph.opt.v)


def test_on_another_stream():
    b, one, two = _batch(), Trainer(), Trainer()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(3):
            two.step(b)
    for _ in range(3):
        one.step(b)
    torch.cuda.synchronize()
    for p, q in zip(one.masters, two.masters):
        assert torch.equal(p, q)


def test_two_graphs_at_once():
    """Two captured calls of each operator that takes a workspace, replayed on two streams: each has its own."""
    g0 = torch.Generator().manual_seed(5)
    x = torch.randn((700, 1000), generator=g0).to(DEV)
    dys = [torch.randn((700, 1000), generator=g0).to(DEV) for _ in range(2)]
    ids = torch.randint(0, 300, (700,), generator=g0, dtype=torch.int32).to(DEV)
    ids[:200] = 7
    w = torch.ones(1000, device=DEV)
    stats = reqat.layer_norm(x, w)[1]
    run = lambda dy: reqat.layer_norm_backward(dy, x, w, stats, bias=True) + (reqat.embedding_backward(dy, ids, 300),)
    want = [run(dy) for dy in dys]
    graphs, got = [], []
    for dy in dys:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(run(dy))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in dys]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(p, q) for p, q in zip(a, b))
