"""The policy loss's reference and bounds by themselves, on the CPU: against another form, against differences, and that they
notice what a wrong kernel would write."""
import math

import pytest
import torch

from tests import policy_ref as pr
from tests import train_ref

SIZES = [(6, 4001), (3, 65537), (5, 152064), (40, 129)]


def _rounded(e, dtype):
    """What a right kernel gives, as far as its outputs' types can hold it."""
    stats = torch.stack([e.lp, e.lse, e.slope, e.r], 1).float()
    return e.loss.float(), stats, pr.gradient(e, dtype)[0].to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V", SIZES)
def test_a_missing_vector_is_noticed(T, V, dtype):
    c = pr.case(T, V, dtype, "cpu", masked=0.2)
    e = pr.exact(c, 0.7, 0.05)
    loss, stats, grad = _rounded(e, dtype)
    pr.check((loss, stats, grad), e, dtype)
    n = 16 // grad.element_size()
    t = int(torch.nonzero((e.slope != 0)).flatten()[0])
    wrongs = []
    for j in (0, n * (V // (2 * n)), n * ((V - 1) // n)):
        wrongs.append(grad.clone())
        wrongs[-1][t, j:j + n] = 0                        # not written
        wrongs.append(grad.clone())
        wrongs[-1][t, j:j + n] *= 1.02                    # another factor
    wrongs.append(grad.clone())
    wrongs[-1][t, n:2 * n] = grad[t, :n]                  # another place
    for wrong in wrongs:
        with pytest.raises(AssertionError, match="gradient"):
            pr.check((loss, stats, wrong), e, dtype)
    given, room = pr.gradient_from(e, stats, 3.0, dtype)
    assert torch.all((given.to(dtype).double() - given).abs() <= room)
    live = given[t].abs() > 1e-30
    assert torch.all(room[t][live] < 0.02 * given[t][live].abs())


@pytest.mark.parametrize("temp,kl", [(1.0, 0.0), (0.6, 0.05), (1.7, 0.3)])
def test_against_the_other_form(temp, kl):
    c = pr.case(30, 77, torch.float32, "cpu", masked=0.3, temp=temp)
    e = pr.exact(c, temp, kl)
    loss, stats, grad = train_ref.policy(c["logits"], c["targets"], c["old"], c["adv"], c["ref"], c["weights"], pr.f32(0.2), pr.f32(0.2),
                                         pr.f32(kl), pr.f32(temp))
    assert torch.allclose(e.loss, loss, rtol=1e-12, atol=1e-14)
    assert torch.allclose(torch.stack([e.lp, e.lse, e.slope, e.r], 1), stats, rtol=1e-12, atol=1e-14)
    assert torch.allclose(pr.gradient(e, torch.float32)[0], grad, rtol=1e-10, atol=1e-16)


def test_rows_of_the_lowest_values():
    """Equal logits, whatever they are, have probability 1 / V; one that is higher has all of it."""
    for value in (torch.finfo(torch.bfloat16).min, -1e30, 0.0, torch.finfo(torch.bfloat16).max):
        c = pr.case(2, 50, torch.bfloat16, "cpu", edit=lambda z, y: z.fill_(value))
        e = pr.exact(c)
        assert torch.allclose(e.lp, torch.full((2,), -math.log(50), dtype=torch.float64))
        assert torch.allclose(e.p, torch.full((2, 50), 0.02, dtype=torch.float64))
