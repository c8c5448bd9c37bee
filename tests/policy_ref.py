"""The policy loss in 64 bits, row-wise vectors on any device, with bounds for FP32 arithmetic that are relative for every element:
an element of the gradient that is missing, shifted or mis-scaled is outside of them, however small it is.

Logits enter relative to their largest one, so that rows of the type's largest and lowest values have their definition too."""
import math
from types import SimpleNamespace

import torch

E = 2.0 ** -24                                            # half a step of FP32, relative


def f32(x):
    return float(torch.tensor(x, dtype=torch.float32))


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def exact(c, temp=1.0, kl=0.0, low=0.2, high=0.2):
    """Everything of a call in float64, with bounds d_* on what FP32 arithmetic adds; c: logits, targets, old, adv, ref (or
    None) and weights.  Rows of weight 0 are zeros."""
    temp, kl, low, high = f32(temp), f32(kl), f32(low), f32(high)
    z, y = c["logits"].double(), c["targets"].long()
    T, V = z.shape
    w, old, adv = c["weights"].double(), c["old"].double(), c["adv"].double()
    top = z.amax(1, keepdim=True)
    x = (z - top) / temp                                  # at most 0
    known = (y >= 0) & (y < V)
    at = torch.where(known, y, 0)[:, None]
    dy = torch.where(known, x.gather(1, at)[:, 0], math.nan)
    lnS = torch.logsumexp(x, 1)
    lp, lse = dy - lnS, top[:, 0] / temp + lnS
    p = torch.exp(x - lnS[:, None])
    # S: terms off by 3 half steps of the exponent (difference, factor, product) and 2 of the exponential, and a chain of
    # additions: up to V / 256 in a thread, the joins, and the corrections when a larger maximum comes
    spread = torch.where(p > 0, p * x.clamp(min=-1e30).abs(), 0.0).sum(1)
    d_S = E * (3 * spread + V / 256 + 128)
    d_lp = E * (2 * dy.abs() + 4 * lnS + lp.abs() + 4) + d_S
    d_lse = E * (2 * top[:, 0].abs() / temp + 4 * lnS + lse.abs() + 4) + d_S
    r = torch.exp(lp - old)
    outside = ((adv > 0) & (r > 1 + high)) | ((adv < 0) & (r < 1 - low))
    surrogate = -torch.minimum(r * adv, r.clamp(1 - low, 1 + high) * adv)
    slope = torch.where(outside, 0.0, -adv * r)
    d_r = r * (d_lp + E * ((lp - old).abs() + 4))
    d_slope = torch.where(outside, 0.0, adv.abs() * (d_r + 2 * E * r))
    d_surrogate = adv.abs() * (d_r + 2 * E * (r + 1 + high))
    term = d_term = torch.zeros_like(w)
    if c["ref"] is not None:
        u = c["ref"].double() - lp
        grow = torch.expm1(u)
        term = grow - u
        d_u = d_lp + E * u.abs()
        d_term = grow.abs() * d_u + 4 * E * (grow.abs() + u.abs())
        if kl != 0.0:
            slope = slope - kl * grow
            d_slope = d_slope + kl * ((grow + 1) * d_u + 5 * E * grow.abs())
    live = w != 0
    zero = lambda t: torch.where(live, t, 0.0)
    d_slope = zero(w.abs() * (d_slope + 2 * E * slope.abs()))
    slope = zero(w * slope)
    q = torch.where(torch.arange(V, device=z.device) == y[:, None], 1.0 - p, -p)
    out = SimpleNamespace(lp=zero(lp), lse=zero(lse), slope=slope, r=zero(r), d_lp=zero(d_lp), d_lse=zero(d_lse), d_slope=d_slope,
                          d_r=zero(d_r), temp=temp, x=x, p=p, q=q, y=y, lnS=lnS, d_S=d_S, live=live, z=z)
    parts = [zero(w * surrogate), zero(w * term), zero(w * outside)]
    sums = [t.sum() for t in parts]
    out.loss = torch.stack([sums[0] + kl * sums[1]] + sums)
    rooms = [zero(w.abs() * d_surrogate).sum(), zero(w.abs() * d_term).sum()]
    out.d_loss = torch.stack([rooms[0] + kl * rooms[1], rooms[0], rooms[1], torch.zeros_like(rooms[0])])
    out.d_loss = out.d_loss + 2 * E * torch.stack([sums[0].abs() + kl * sums[1].abs()] + [s.abs() for s in sums])
    return out


def gradient(e, dtype):
    """(dL/dlogits, bound) of loss and gradient in one call."""
    s, d_s = (e.slope / e.temp)[:, None], (e.d_slope / e.temp)[:, None]
    rel = E * (3 * e.x.abs() + 8) + e.d_S[:, None]        # of p, and of the factor's divisions
    hot = torch.arange(e.p.shape[1], device=e.p.device) == e.y[:, None]
    return _bounded(s * e.q, d_s * e.q.abs() + s.abs() * (torch.where(e.p > 0, e.p * rel, 0.0) + hot * 4 * E), s, dtype)


def gradient_from(e, stats, factor, dtype):
    """(dL/dlogits, bound) from statistics that are within their own bounds; their dL/dlp is taken as it is."""
    s = (factor * stats[:, 2].double() / e.temp)[:, None]
    z_y = e.z.gather(1, e.y[:, None])
    by_target = (e.lp.abs() < e.lse.abs())[:, None]
    either = lambda a, b: torch.where(by_target, a, b)
    # whichever form is taken where |lp| and |lse| are as good as equal, both are as exact
    rel = either(e.d_lp[:, None], e.d_lse[:, None]) + E * (either(3 * (e.z - z_y).abs() / e.temp + 3 * e.lp.abs()[:, None],
                                                                  3 * e.z.abs() / e.temp + 3 * e.lse.abs()[:, None]) + 8)
    hot = torch.arange(e.p.shape[1], device=e.p.device) == e.y[:, None]
    rel = torch.where(hot, e.d_lp[:, None] + 8 * E, rel)
    room = s.abs() * (torch.where(e.p > 0, e.p * rel, 0.0) + hot * e.q.abs() * 8 * E)
    return _bounded(s * e.q, room, s, dtype)


def _bounded(g, room, s, dtype):
    """A result rounded once; exponentials below FP32's smallest normal number may be 0."""
    return g, room + 1.01 * half_step(dtype) * g.abs() + (s.abs() + 1) * 1e-37


def check(got, e, dtype):
    """(loss, stats, gradient or None) of a call against exact()."""
    loss, stats, grad = got
    stats = stats.double()
    assert torch.all((stats[:, 0] - e.lp).abs() <= e.d_lp), "log p"
    beyond = torch.isinf(e.lse.float())                   # FP32 does not hold it
    assert torch.all(torch.where(beyond, stats[:, 1] == e.lse.float(), (stats[:, 1] - e.lse).abs() <= e.d_lse)), "log-sum-exp"
    assert torch.all((stats[:, 2] - e.slope).abs() <= e.d_slope), "slope"
    assert torch.all((stats[:, 3] - e.r).abs() <= e.d_r), "ratio"
    assert torch.all((loss.double() - e.loss).abs() <= e.d_loss), (loss.double() - e.loss, e.d_loss)
    if grad is not None:
        want, room = gradient(e, dtype)
        assert torch.all((grad.double() - want).abs() <= room), "gradient"


def case(T, V, dtype, device, seed=0, pad=0, std=2.0, temp=1.0, masked=0.0, edit=None):
    """Inputs of a call off the clipping borders; edit: changes the logits and targets before the rest follows from them."""
    g = torch.Generator(device=device).manual_seed(1000 * T + V + seed)
    rand = lambda *s: torch.randn(s, generator=g, device=device)
    logits = (std * rand(T, V + pad)).to(dtype)[:, :V]
    targets = torch.randint(0, V, (T,), generator=g, device=device, dtype=torch.int32)
    if edit is not None:
        edit(logits, targets)
    c = dict(logits=logits, targets=targets, old=torch.zeros(T, device=device), adv=rand(T), ref=None,
             weights=(torch.rand(T, generator=g, device=device) + 0.1) / T)
    lp = exact(c, temp).lp
    delta = 0.3 * rand(T).double()
    for border in (math.log(0.8), math.log(1.2)):         # where the gradient jumps
        delta = torch.where((delta - border).abs() < 2e-3, border + 4e-3, delta)
    c["old"], c["ref"] = (lp - delta).float(), (lp + 0.2 * rand(T).double()).float()
    if masked:
        c["weights"] = torch.where(torch.rand(T, generator=g, device=device) < masked, 0.0, c["weights"])
    return c
