"""GPU: the policy loss of logits far from zero, up to the type's largest and lowest values, through each of its kernels."""
import math

import pytest
import torch

from paper_2606_15682_amd import reqat
from tests import policy_ref as pr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
# few rows whole and in slices, rows of 256 and of 1024 threads, several rows a workgroup
SIZES = [(7, 33), (14, 40000), (133, 5000), (301, 9001), (1101, 515)]


def _edit(dtype):
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max

    def edit(z, y):
        V = z.shape[1]
        half = V // 2
        kind = torch.arange(z.shape[0], device=z.device) % 7
        for k, (fill, part) in enumerate(((low, slice(0, half)), (low, slice(half, V)), (-math.inf, slice(0, half)),
                                          (low, slice(0, V)), (high, slice(0, V)), (0.5 * low, slice(0, half)))):
            z[kind == k, part] = fill
        y[(kind == 0) | (kind == 2) | (kind == 5)] = V - 1
        y[kind == 1] = 0
        z[kind == 6, y[kind == 6].long()] = high          # one token has it all
    return edit


def _run(c, temp, kl, **kw):
    return reqat.policy_loss_grad(c["logits"], c["targets"], c["old"], c["adv"], ref_logp=c["ref"], weights=c["weights"],
                                  kl_coef=kl, temperature=temp, **kw)


@pytest.mark.parametrize("temp", [1.0, 0.6, 2.5])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V", SIZES)
def test_lowest_and_largest(T, V, dtype, temp):
    print("policy values", T, V, dtype, temp, flush=True)
    c = pr.case(T, V, dtype, DEV, temp=temp, edit=_edit(dtype))
    e = pr.exact(c, temp, 0.05)
    got = _run(c, temp, 0.05)
    pr.check(got, e, dtype)
    loss, stats = reqat.policy_loss(c["logits"], c["targets"], c["old"], c["adv"], ref_logp=c["ref"], weights=c["weights"],
                                    kl_coef=0.05, temperature=temp)
    pr.check((loss, stats, None), e, dtype)
    up = torch.tensor([2.0], device=DEV)
    grad = reqat.policy_loss_backward(c["logits"], c["targets"], stats, temperature=temp, grad_loss=up)
    want, room = pr.gradient_from(e, stats, 2.0, dtype)
    assert torch.all((grad.double() - want).abs() <= room)
    reqat.policy_loss_backward(c["logits"], c["targets"], stats, temperature=temp, grad_loss=up, out=c["logits"])
    assert torch.equal(c["logits"], grad)


@pytest.mark.parametrize("shift", [50.0, -1000.0, 1e5])
@pytest.mark.parametrize("T,V", SIZES)
def test_far_from_zero(T, V, shift):
    """A common shift costs the probabilities nothing, at temperatures whose reciprocal is rounded."""
    c = pr.case(T, V, F32, DEV, temp=0.6, edit=lambda z, y: z.add_(shift))
    e = pr.exact(c, 0.6, 0.05)
    pr.check(_run(c, 0.6, 0.05), e, F32)
    stats = reqat.policy_loss(c["logits"], c["targets"], c["old"], c["adv"], ref_logp=c["ref"], weights=c["weights"],
                              kl_coef=0.05, temperature=0.6)[1]
    grad = reqat.policy_loss_backward(c["logits"], c["targets"], stats, temperature=0.6)
    want, room = pr.gradient_from(e, stats, 1.0, F32)
    assert torch.all((grad.double() - want).abs() <= room)


@pytest.mark.parametrize("T,V", [(5, 5001), (2, 152064), (2100, 700)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_masked_and_missing_targets_from_statistics(T, V, dtype):
    """A target of probability 0 or outside the vocabulary, where the gradient comes from the log-sum-exp."""
    c = pr.case(T, V, dtype, DEV)
    stats = torch.zeros((T, 4), device=DEV)
    e = pr.exact(c)
    stats[:, 0], stats[:, 1], stats[:, 2] = e.lp, e.lse, 0.5
    c["logits"][0, c["targets"][0].long()] = -math.inf
    stats[0, 0], stats[0, 1] = -math.inf, torch.logsumexp(c["logits"][0].double(), 0)
    for out in (None, c["logits"].clone()):
        got = reqat.policy_loss_backward(c["logits"] if out is None else out, c["targets"], stats, out=out)
        p = torch.exp(c["logits"][0].double() - stats[0, 1].double())
        want = -0.5 * p
        want[c["targets"][0].long()] += 0.5
        assert torch.all((got[0].double() - want).abs() <= 1.01 * pr.half_step(dtype) * want.abs() + 40 * pr.E * want.abs() + 1e-37)
    c["targets"][1] = V
    stats[1, 0] = stats[1, 2] = math.nan
    for out in (None, c["logits"].clone()):
        got = reqat.policy_loss_backward(c["logits"] if out is None else out, c["targets"], stats, out=out)
        assert torch.isnan(got[1]).all() and torch.isfinite(got[0]).all()


def _worst_temperature():
    """The temperature whose scale log2(e) / temperature is rounded most."""
    def off(t):
        c = math.log2(math.e) / pr.f32(t)
        return abs(pr.f32(c) - c) / c
    return max((0.4 + 0.01 * k for k in range(200)), key=off)


@pytest.mark.parametrize("T,V", [(1040, 4000), (3, 40000), (300, 9001)])
def test_probabilities_of_far_tokens(T, V):
    """FP32: tokens 60 below the first one.  Each exponent's own roundings (2^-24 of 60) average out over thousands of tokens;
    what the scale's rounding adds is the same in all, 54 half steps here, and does not."""
    temp = _worst_temperature()
    c = pr.case(T, V, F32, DEV, temp=temp, edit=lambda z, y: (z.uniform_(-64 * temp, -56 * temp), z[:, 0].zero_(), y.zero_()))
    e = pr.exact(c, temp)
    loss, stats, grad = _run(c, temp, 0.0)
    back = reqat.policy_loss_backward(c["logits"], c["targets"], stats, temperature=temp)
    live = stats[:, 2] != 0
    assert live.any()
    want = -(stats[:, 2:3].double() / e.temp) * e.p
    for got in (grad, back):
        rel = (got.double() / want - 1)[live, 1:].mean()
        # the factor and its two divisions 3, the exponential 2; log p (0 here) and the averages 1
        assert float(rel.abs()) <= 6 * pr.E, float(rel) / pr.E


@pytest.mark.parametrize("dtype,vector", [(F32, 4), (BF, 8)])
def test_many_small_terms_beside_a_large_one(dtype, vector):
    """The thread that has a row's first token adds up some 297 terms of 2^-25 beside its 1.  One after the other they are lost, half
    of 2^-24 each; by vectors every addition rounds once, and so does each join."""
    T, V = 130, 152064
    z = torch.full((T, V), -25 * math.log(2.0), dtype=dtype, device=DEV)
    z[:, 0] = 0.0
    zeros = torch.zeros(T, device=DEV)
    stats = reqat.policy_loss(z, torch.zeros(T, dtype=torch.int32, device=DEV), zeros, zeros)[1]
    want = -math.log1p((V - 1) * math.exp(float(z[0, 1])))
    # additions of a thread, 14 joins, exponentials and the logarithm (of 0.0045)
    room = pr.E * (-(-V // (512 * vector)) + 14 + 4)
    assert torch.all((stats[:, 0].double() - want).abs() <= room)
