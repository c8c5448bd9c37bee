"""GPU: the policy loss's kernels for more than 128 rows, against 64 bits with bounds relative for every element: rows of 256 and of
1024 threads with every number of vectors a thread, several rows a workgroup, masked rows among them, in place, both types; the
loss alone; the gradient from statistics."""
import pytest
import torch

from paper_2606_15682_amd import reqat
from tests import policy_ref as pr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
TYPES = [(BF, 8), (F32, 4)]


def _grad(c, kl=0.05, temp=1.0, **kw):
    return reqat.policy_loss_grad(c["logits"], c["targets"], c["old"], c["adv"], ref_logp=c["ref"], weights=c["weights"],
                                  kl_coef=kl, temperature=temp, **kw)


def _both(T, V, dtype, pad=0, masked=0.25, temp=1.0, kl=0.05):
    """A call beside its logits and one in their place, both against 64 bits, the memory between rows as it was."""
    print("policy rows", T, V, dtype, pad, flush=True)
    c = pr.case(T, V, dtype, DEV, pad=pad, masked=masked, temp=temp)
    c["weights"][0], c["weights"][-1] = 0.0, 1.0 / T      # a workgroup whose first row has no weight, a last one that has
    e = pr.exact(c, temp, kl)
    got = _grad(c, kl, temp)
    pr.check(got, e, dtype)
    assert not got[1][~e.live].any() and not got[2][~e.live].any()
    c["logits"][~e.live] = float("nan")                   # not read
    if pad:
        wide = c["logits"].as_strided((T, V + pad), (V + pad, 1))
        kept = wide[:, V:].clone()
    again = _grad(c, kl, temp, out=c["logits"])
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    if pad:
        assert torch.equal(wide[:, V:], kept)


# more rows than the 1024 workgroups of 256 threads: 0 to 4 vectors a thread, rests of every kind
@pytest.mark.parametrize("dtype,n", TYPES)
@pytest.mark.parametrize("T,vectors,rest", [(1500, 0, 3), (1025, 0, 1), (2049, 1, 0), (1500, 200, 1), (1100, 256, 0), (1300, 257, 2),
                                            (1100, 512, 1), (1100, 600, 0), (1030, 768, 3), (1100, 769, 0), (1030, 1024, 0),
                                            (1030, 1023, 3)])
def test_rows_of_256_threads(T, vectors, rest, dtype, n):
    _both(T, vectors * n + rest, dtype, pad=vectors % 3)


# more rows than the 256 workgroups of 1024 threads: 2 to 18 vectors a thread held, and rows that do not fit
@pytest.mark.parametrize("dtype,n", TYPES)
@pytest.mark.parametrize("steps", range(1, 21))
def test_rows_of_1024_threads(steps, dtype, n):
    # the last step just begun, half full, full; with and without a partial vector
    V = (steps * 1024 + (1, 512, 1024)[steps % 3]) * n + (0, 1, n - 1)[steps % 3]
    _both(257 + 130 * (steps % 2), V, dtype, pad=(0, 5, 0, 2)[steps % 4])


@pytest.mark.parametrize("dtype,V", [(BF, 152064), (F32, 152064), (F32, 75001)])
def test_vocabulary_of_a_model(dtype, V):
    _both(300, V, dtype)


@pytest.mark.parametrize("dtype,n", TYPES)
def test_masks_over_many_rows(dtype, n):
    """Runs without weight longer than the grid, a single row with weight, none."""
    for V in (40 * n + 1, 1500 * n):
        T = 1400
        c = pr.case(T, V, dtype, DEV)
        weights = c["weights"].clone()
        for first, last in ((0, 1100), (300, 1400), (1, 1400), (0, 1399), (0, 1400)):
            c["weights"] = weights.clone()
            c["weights"][first:last] = 0.0
            e = pr.exact(c, 1.0, 0.05)
            got = _grad(c)
            pr.check(got, e, dtype)
            assert not got[1][~e.live].any() and not got[2][~e.live].any()


# above 128 rows a workgroup reads a row once: its loop of four vectors a thread, its single ones, and a partial one
@pytest.mark.parametrize("dtype,n", TYPES)
@pytest.mark.parametrize("T,vectors,rest", [(129, 511, 1), (130, 2047, 0), (130, 2048, 0), (200, 2049, 3), (131, 5000, 1),
                                            (300, 10240, 0), (150, 19008, 0), (1001, 2500, 2)])
def test_loss_alone(T, vectors, rest, dtype, n):
    V = vectors * n + rest
    print("policy loss", T, V, dtype, flush=True)
    c = pr.case(T, V, dtype, DEV, pad=T % 3, masked=0.25, temp=0.8)
    e = pr.exact(c, 0.8, 0.05)
    loss, stats = reqat.policy_loss(c["logits"], c["targets"], c["old"], c["adv"], ref_logp=c["ref"], weights=c["weights"],
                                    kl_coef=0.05, temperature=0.8)
    pr.check((loss, stats, None), e, dtype)
    assert not stats[~e.live].any()


# one workgroup a row, two, many; in place the target's element comes later
@pytest.mark.parametrize("dtype,n", TYPES)
@pytest.mark.parametrize("T,V", [(1, 1), (1, 3), (7, 4096), (1, 4097), (3, 152064), (129, 30001), (1024, 9000), (2047, 8200), (2048, 8200),
                                 (2500, 777)])
def test_gradient_from_statistics(T, V, dtype, n):
    print("policy gradient from statistics", T, V, dtype, flush=True)
    pad = T % 4
    c = pr.case(T, V, dtype, DEV, pad=pad, masked=0.2 if T > 2 else 0.0, temp=0.7)
    e = pr.exact(c, 0.7, 0.05)
    stats = reqat.policy_loss(c["logits"], c["targets"], c["old"], c["adv"], ref_logp=c["ref"], weights=c["weights"],
                              kl_coef=0.05, temperature=0.7)[1]
    up = torch.tensor([3.0], device=DEV)
    grad = reqat.policy_loss_backward(c["logits"], c["targets"], stats, temperature=0.7, grad_loss=up)
    want, room = pr.gradient_from(e, stats, 3.0, dtype)
    assert torch.all((grad.double() - want).abs() <= room)
    assert not grad[~e.live].any()
    wide = torch.full((T, V + 3), 7.0, dtype=dtype, device=DEV)
    beside = reqat.policy_loss_backward(c["logits"], c["targets"], stats, temperature=0.7, grad_loss=up, out=wide[:, 2:2 + V])
    assert torch.equal(beside, grad) and (wide[:, :2] == 7.0).all() and (wide[:, 2 + V:] == 7.0).all()
    for _ in range(3):
        logits = c["logits"].clone()
        reqat.policy_loss_backward(logits, c["targets"], stats, temperature=0.7, grad_loss=up, out=logits)
        assert torch.equal(logits, grad)


def test_captured_beside_eager():
    """Loss, gradient and the gradient in the logits' place in one graph, replayed over new logits."""
    T, V = 300, 20001
    cases = [pr.case(T, V, BF, DEV, seed=s, masked=0.25) for s in range(3)]
    c = {k: v.clone() for k, v in cases[0].items()}

    def step():
        loss, stats, grad = _grad(c)
        alone, given = reqat.policy_loss(c["logits"], c["targets"], c["old"], c["adv"], ref_logp=c["ref"], weights=c["weights"],
                                         kl_coef=0.05)
        few = c["logits"][:5].clone()
        reqat.policy_loss_backward(few, c["targets"][:5], given[:5], out=few)
        return loss, stats, grad, alone, given, few

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for k in (1, 2, 0, 1):
        for name, value in cases[k].items():
            c[name].copy_(value)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        assert all(torch.equal(a, b) for a, b in zip(got, step())), k
        pr.check(got[:3], pr.exact(cases[k], 1.0, 0.05), BF)
