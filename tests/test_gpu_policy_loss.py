"""GPU: the policy loss against its formula in 64 bits, at sizes, strides, masks and values where it can go wrong."""
import math

import pytest
import torch

from paper_2606_15682_amd import reqat
from tests import train_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _case(T, V, dtype, seed=0, pad=0, std=2.0):
    g = torch.Generator().manual_seed(1000 * T + V + seed)
    wide = (torch.randn((T, V + pad), generator=g) * std).to(dtype)
    targets = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    z = wide[:, :V].double()
    lp = z.gather(1, targets[:, None].long())[:, 0] - torch.logsumexp(z, 1)
    delta = 0.3 * torch.randn(T, generator=g)
    for border in (math.log(0.8), math.log(1.2)):          # off the borders, where the gradient jumps
        delta = torch.where((delta - border).abs() < 1e-3, torch.tensor(border + 2e-3), delta)
    old = (lp - delta).float()
    return dict(logits=wide.to(DEV)[:, :V], targets=targets.to(DEV), old=old.to(DEV),
                adv=torch.randn(T, generator=g).to(DEV), ref=(lp + 0.2 * torch.randn(T, generator=g)).float().to(DEV),
                weights=(torch.rand(T, generator=g) + 0.1).to(DEV) / T)


def _bounds(c, temp):
    """Bound on the error of lp: products c z of up to 8 half steps each (the factor, the product's rounding, the maximum's
    product, both sides) and a sum of V terms, at most V / 2048 + 32 additions deep, each term 2^t off by 2 steps and |t|
    half steps."""
    finite = torch.where(torch.isfinite(c["logits"]), c["logits"], torch.zeros_like(c["logits"]))
    top = 1.45 * float(finite.float().abs().max()) / temp
    V = c["logits"].shape[1]
    return ref.EPS32 * (16 * top + V / 2048 + 64)


def _check(c, got, temp=1.0, kl=0.05, low=0.2, high=0.2, with_ref=True, weights="weights"):
    w = None if weights is None else c[weights]
    loss, stats, grad = (t.double().cpu() for t in got)
    eloss, estats, egrad = ref.policy(c["logits"], c["targets"], c["old"], c["adv"], c["ref"] if with_ref else None, w,
                                      low, high, kl, temp)
    d = _bounds(c, temp)
    T = c["targets"].shape[0]
    w = torch.full((T,), 1.0 / T, dtype=torch.float64) if w is None else w.double().cpu()
    nan = torch.isnan(estats[:, 0])
    assert torch.equal(torch.isnan(stats[:, 0]), nan)
    s, e = stats[~nan], estats[~nan]
    assert torch.all((s[:, :2] - e[:, :2]).abs() <= d + ref.EPS32 * e[:, :2].abs())
    assert torch.all((s[:, 3] - e[:, 3]).abs() <= e[:, 3] * (2 * d + 8 * ref.EPS32))
    # dL/dlp moves by r |A| d and kl exp(x) d
    a = c["adv"].double().cpu()[~nan].abs()
    ex = torch.exp(c["ref"].double().cpu()[~nan] - e[:, 0]) if with_ref else torch.zeros_like(a)
    live = w[~nan] != 0
    room = w[~nan] * (a * e[:, 3] + kl * (ex + 1)) * (2 * d + 16 * ref.EPS32) * live
    assert torch.all((s[:, 2] - e[:, 2]).abs() <= room)
    # p is off by 2 d relative, the factor by `room`, and the result is rounded once
    slope = (room / temp)[:, None]
    p = egrad[~nan].abs()
    dt = c["logits"].dtype
    tol = slope + p * (ref.half_step(dt) * 1.01 + 4 * d) + 1e-37
    assert torch.all((grad[~nan] - egrad[~nan]).abs() <= tol)
    assert torch.isnan(grad[nan]).all()
    if nan.any():
        assert torch.isnan(loss[0])
        return
    each = w * (c["adv"].double().cpu().abs() * torch.maximum(estats[:, 3], torch.ones(T, dtype=torch.float64)) + 1.0)
    tol = float(each.sum()) * (4 * d + 32 * ref.EPS32) * 2
    if with_ref:                                          # exp(x) - x - 1 moves by |exp(x) - 1| d
        x = c["ref"].double().cpu() - estats[:, 0]
        tol += float((w * torch.expm1(x).abs() * (w != 0)).sum()) * 4 * d
    assert torch.all((loss[:3] - eloss[:3]).abs() <= tol), (loss, eloss)
    assert abs(float(loss[3] - eloss[3])) <= 1e-6


def _run(c, temp=1.0, kl=0.05, low=0.2, high=0.2, with_ref=True, weights="weights", **kw):
    return reqat.policy_loss_grad(c["logits"], c["targets"], c["old"], c["adv"], ref_logp=c["ref"] if with_ref else None,
                                  weights=None if weights is None else c[weights], clip_low=low, clip_high=high,
                                  kl_coef=kl, temperature=temp, **kw)


SIZES = [(1, 1), (1, 2), (2, 7), (3, 8), (5, 33), (17, 1000), (2, 4097), (300, 129), (3, 16384), (6, 65537)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V", SIZES)
def test_loss_and_gradient(T, V, dtype):
    print("policy", T, V, dtype, flush=True)
    c = _case(T, V, dtype)
    _check(c, _run(c))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_full_vocabulary_and_temperature(dtype):
    c = _case(5, 152064, dtype, std=3.0)
    _check(c, _run(c), kl=0.05)
    z = (c["logits"].double() / 0.6)
    lp = z.gather(1, c["targets"][:, None].long())[:, 0] - torch.logsumexp(z, 1)
    c["old"], c["ref"] = (lp - 0.05).float(), (lp + 0.1).float()
    _check(c, _run(c, temp=0.6), temp=0.6)


@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_and_places(pad, dtype):
    c = _case(9, 777, dtype, pad=pad)
    wide = torch.full((9, 777 + pad + 2), 5.0, dtype=dtype, device=DEV)
    out = wide[:, 1:778]                                  # an odd place beside the logits' stride
    got = _run(c, out=out)
    assert got[2].data_ptr() == out.data_ptr()
    _check(c, got)
    assert torch.all(wide[:, 0] == 5.0) and torch.all(wide[:, 778:] == 5.0)


def test_in_place_and_without_terms():
    c = _case(33, 1003, torch.bfloat16, pad=5)
    first = _run(c, kl=0.0, with_ref=False, weights=None)
    _check(c, first, kl=0.0, with_ref=False, weights=None)
    keep = c["logits"].clone()
    again = _run(c, kl=0.0, with_ref=False, weights=None, out=c["logits"])
    for a, b in zip(first, again):
        assert torch.equal(a, b)
    assert not torch.equal(keep, c["logits"])


def test_masked_rows_are_not_read():
    c = _case(40, 515, torch.float32)
    plain = _run(c)
    mask = torch.zeros(40, dtype=torch.bool, device=DEV)
    mask[[0, 3, 17, 38, 39]] = True
    c["weights"] = torch.where(mask, 0.0, c["weights"])
    want = ref.policy(c["logits"], c["targets"], c["old"], c["adv"], c["ref"], c["weights"], kl=0.05)[0]
    c["logits"][mask] = math.nan
    c["adv"][mask] = math.inf
    c["targets"][mask] = -100
    loss, stats, grad = _run(c)
    assert torch.all(stats[mask] == 0) and torch.all(grad[mask] == 0)
    assert torch.equal(stats[~mask], plain[1][~mask]) and torch.equal(grad[~mask], plain[2][~mask])
    assert torch.all((loss.double().cpu() - want).abs() <= 1e-5)
    all_masked = torch.zeros_like(c["weights"])
    loss, stats, grad = reqat.policy_loss_grad(c["logits"], c["targets"], c["old"], c["adv"], weights=all_masked)
    assert not loss.any() and not stats.any() and not grad.any()


def test_special_logits_and_targets():
    c = _case(8, 130, torch.float32)
    c["logits"][0, 3:] = -math.inf                        # most of the vocabulary masked out
    c["targets"][0] = 1
    c["logits"][1, :129] = -math.inf                      # one token left
    c["targets"][1] = 129
    c["logits"][2, 5] = math.nan
    c["logits"][3, 5] = math.inf
    c["targets"][4], c["targets"][5] = 130, -1
    c["logits"][6] = -math.inf                            # nothing left
    for t in (0, 1):
        c["old"][t] = c["ref"][t] = 0.0
    c["ref"][0] = -1.0
    c["old"][0] = -1.0
    loss, stats, grad = _run(c)
    assert torch.isnan(stats[[2, 3, 4, 5, 6], 0]).all() and torch.isnan(grad[[2, 3, 4, 5, 6]]).all()
    assert math.isnan(float(loss[0]))
    keep = [0, 1, 7]
    d = {k: v[keep].contiguous() for k, v in c.items()}
    got = (ref.policy(d["logits"], d["targets"], d["old"], d["adv"], d["ref"], d["weights"], kl=0.05))
    assert torch.allclose(stats[keep].double().cpu(), got[1], atol=1e-5)
    assert torch.allclose(grad[keep].double().cpu(), got[2], atol=1e-6)


def test_large_logits():
    c = _case(6, 300, torch.float32, std=1.0)
    for shift in (0.0, 1e3, -1e3):
        d = dict(c, logits=c["logits"] + shift)
        z = d["logits"].double()
        lp = z.gather(1, d["targets"][:, None].long())[:, 0] - torch.logsumexp(z, 1)
        d["old"], d["ref"] = (lp - 0.05).float(), (lp + 0.1).float()
        _check(d, _run(d))


def test_clipping_borders_and_signs():
    """Every branch: ratios on both sides of both borders, advantages of both signs and zero."""
    ratios = torch.tensor([0.5, 0.79, 0.81, 1.0, 1.19, 1.21, 3.0])
    advs = torch.tensor([-1.5, 0.0, 2.0])
    T = len(ratios) * len(advs)
    c = _case(T, 50, torch.float32)
    z = c["logits"].double()
    lp = z.gather(1, c["targets"][:, None].long())[:, 0] - torch.logsumexp(z, 1)
    c["old"] = (lp - torch.log(ratios.repeat_interleave(len(advs))).double().to(DEV)).float()
    c["adv"] = advs.repeat(len(ratios)).to(DEV)
    for kl, with_ref in ((0.0, False), (0.1, True)):
        got = _run(c, kl=kl, with_ref=with_ref)
        _check(c, got, kl=kl, with_ref=with_ref)
    assert (got[0][3] > 0).item()


def test_small_kl_differences():
    """exp(x) - x - 1 for x from 1e-3 on: its square law, not the rounding of close numbers."""
    c = _case(64, 40, torch.float32)
    c["logits"].zero_()
    c["targets"].zero_()
    lp = -math.log(40)
    lp32 = float(torch.tensor(lp, dtype=torch.float32))
    x = torch.logspace(-3, 1, 64, dtype=torch.float64) * torch.where(torch.arange(64) % 2 == 0, 1.0, -1.0)
    c["ref"] = (lp32 + x).float().to(DEV)
    c["adv"].zero_()
    c["old"] = torch.full((64,), lp32, device=DEV)
    w = torch.zeros(64, device=DEV)
    for t in range(64):
        w.zero_()
        w[t] = 1.0
        loss = reqat.policy_loss(c["logits"], c["targets"], c["old"], c["adv"], ref_logp=c["ref"], weights=w)[0]
        d = float(c["ref"][t].double()) - lp
        want = math.expm1(d) - d
        # lp is off by up to 8 half steps of its size 3.7
        assert abs(float(loss[2]) - want) <= abs(math.expm1(d)) * 8 * 3.7 * ref.EPS32 + 1e-6 * want


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V", [(1, 5), (3, 4099), (260, 513), (2, 152064)])
def test_backward_from_statistics(T, V, dtype):
    c = _case(T, V, dtype)
    c["weights"][0] = 0.0 if T > 1 else c["weights"][0]
    loss, stats = reqat.policy_loss(c["logits"], c["targets"], c["old"], c["adv"], ref_logp=c["ref"], weights=c["weights"],
                                    kl_coef=0.05, temperature=0.7)
    both = reqat.policy_loss_grad(c["logits"], c["targets"], c["old"], c["adv"], ref_logp=c["ref"], weights=c["weights"],
                                  kl_coef=0.05, temperature=0.7)
    # two workgroup sizes add the same terms in two orders: each is within its bound
    d = _bounds(c, 0.7)
    assert torch.all((stats[:, :2] - both[1][:, :2]).abs() <= 2 * d + 2 * ref.EPS32 * stats[:, :2].abs())
    assert torch.all((stats[:, 3] - both[1][:, 3]).abs() <= stats[:, 3] * (4 * d + 16 * ref.EPS32))
    assert torch.allclose(loss, both[0], rtol=1e-4, atol=1e-6)
    up = torch.tensor([3.0], device=DEV)
    grad = reqat.policy_loss_backward(c["logits"], c["targets"], stats, temperature=0.7, grad_loss=up)
    lse, slope = stats[:, 1:2].double(), stats[:, 2:3].double()
    want = -torch.exp(c["logits"].double() / 0.7 - lse)
    want[torch.arange(T), c["targets"].long()] += 1.0
    scale = 3.0 * slope / 0.7
    top = 1.45 * float(c["logits"].float().abs().max()) / 0.7
    tol = ref.half_step(dtype) * 1.01 * (want * scale).abs() + scale.abs() * ref.EPS32 * (8 * top + 64) + 1e-37
    assert torch.all((grad.double() - want * scale).abs() <= tol)
    # in place
    reqat.policy_loss_backward(c["logits"], c["targets"], stats, temperature=0.7, grad_loss=up, out=c["logits"])
    assert torch.equal(c["logits"], grad)


def test_against_differences_and_autograd():
    """Central differences of the loss: h^2 times a third derivative of at most a few, and FP32's 2^-24 of the loss over h."""
    c = _case(4, 9, torch.float32)
    args = (c["targets"], c["old"], c["adv"], c["ref"], c["weights"], 0.2, 0.2, 0.05, 0.8)
    z = c["logits"].clone().requires_grad_()
    (reqat.PolicyLoss.apply(z, *args) * 2.0).backward()
    h = 2.0 ** -7
    for t in range(4):
        for j in range(9):
            up, down = c["logits"].clone(), c["logits"].clone()
            up[t, j] += h
            down[t, j] -= h
            f = [float(reqat.PolicyLoss.apply(x, *args)) for x in (up, down)]
            # a row may cross a clipping border: those of this seed are further than h away
            assert abs((f[0] - f[1]) / (2 * h) * 2.0 - float(z.grad[t, j])) <= 2e-4


def test_deterministic_and_empty():
    c = _case(77, 5001, torch.bfloat16)
    a, b = _run(c), _run(c)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    e = {k: v[:0] for k, v in c.items()}
    loss, stats, grad = _run(e)
    assert not loss.any() and stats.shape == (0, 4) and grad.shape == (0, 5001)


def test_reference_without_weight():
    """With kl_coef 0 a reference, however far, is reported and reaches neither loss nor gradient."""
    for T in (3, 200):                                     # cut into slices, whole rows
        c = _case(T, 9000, torch.float32)
        want = reqat.policy_loss_grad(c["logits"], c["targets"], c["old"], c["adv"])
        far = torch.full((T,), 300.0, device=DEV)
        loss, stats, grad = reqat.policy_loss_grad(c["logits"], c["targets"], c["old"], c["adv"], ref_logp=far)
        assert torch.equal(loss[:2], want[0][:2]) and torch.equal(stats, want[1]) and torch.equal(grad, want[2])
        assert torch.isinf(loss[2])
