"""Plain 64-bit forms of the operators around the quantized layers (policy loss, norm, embedding, AdamW), on the CPU."""
import math

import torch

EPS32 = 2.0 ** -24                                  # half a step of FP32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def policy(logits, targets, old, adv, ref=None, weights=None, low=0.2, high=0.2, kl=0.0, temp=1.0):
    """(loss[4], stats [T, 4], grad [T, V]) in float64, rows of weight 0 as zeros."""
    z = logits.double().cpu() / temp
    T, V = z.shape
    w = torch.full((T,), 1.0 / max(T, 1), dtype=torch.float64) if weights is None else weights.double().cpu()
    old, adv = old.double().cpu(), adv.double().cpu()
    loss, stats, grad = torch.zeros(4, dtype=torch.float64), torch.zeros((T, 4), dtype=torch.float64), torch.zeros((T, V), dtype=torch.float64)
    for t in range(T):
        if w[t] == 0:
            continue
        y = int(targets[t])
        lse = torch.logsumexp(z[t], 0)
        lp = (z[t, y] if 0 <= y < V else torch.tensor(math.nan, dtype=torch.float64)) - lse
        r, a = torch.exp(lp - old[t]), adv[t]
        outside = bool((a > 0 and r > 1 + high) or (a < 0 and r < 1 - low))
        surr = -torch.minimum(r * a, r.clamp(1 - low, 1 + high) * a)
        slope = torch.zeros((), dtype=torch.float64) if outside else -a * r
        k = torch.zeros((), dtype=torch.float64)
        if ref is not None:
            x = ref.double().cpu()[t] - lp
            k = torch.expm1(x) - x
            slope = slope - kl * torch.expm1(x)
        loss += w[t] * torch.stack([surr + kl * k, surr, k, torch.tensor(float(outside), dtype=torch.float64)])
        stats[t] = torch.stack([lp, lse, w[t] * slope, r])
        g = -torch.exp(z[t] - lse)
        if 0 <= y < V:
            g[y] += 1
        grad[t] = g * w[t] * slope / temp
    return loss, stats, grad


def norm(x, w, b=None, eps=1e-6, center=True):
    x, w = x.double().cpu(), w.double().cpu()
    mu = x.mean(1) if center else torch.zeros(x.shape[0], dtype=torch.float64)
    rstd = (((x - mu[:, None]) ** 2).mean(1) + eps) ** -0.5
    y = (x - mu[:, None]) * rstd[:, None] * w
    return y if b is None else y + b.double().cpu(), torch.stack([mu, rstd], 1)


def norm_backward(dy, x, w, stats, center=True):
    dy, x, w, stats = (t.double().cpu() for t in (dy, x, w, stats))
    mu, rstd = stats[:, :1], stats[:, 1:]
    h, g = (x - mu) * rstd, dy * w
    dx = g - h * (g * h).mean(1, keepdim=True)
    if center:
        dx = dx - g.mean(1, keepdim=True)
    return dx * rstd, (dy * h).sum(0), dy.sum(0)


def embedding_backward(dy, ids, rows, scale=1.0):
    """(gradient, sum of the magnitudes added to it)."""
    dy, ids = dy.double().cpu(), ids.long().cpu()
    keep = (ids >= 0) & (ids < rows)
    out = torch.zeros((rows, dy.shape[1]), dtype=torch.float64)
    mag = out.clone()
    out.index_add_(0, ids[keep], dy[keep])
    mag.index_add_(0, ids[keep], dy[keep].abs())
    return out * scale, mag * abs(scale)


# ------------------------------------------------------------------ AdamW: FP32 steps exactly, by rounding 64-bit results

def f32(x):
    """Rounds float64 to FP32 (products, sums, quotients and roots of FP32 numbers are rounded right this way)."""
    return x.float().double()


def number(x):
    return float(torch.tensor(x, dtype=torch.float32))


def states(m, v, g, betas, scale=None):
    """m', v' and sqrt(v') as FP32 steps give them (float64 tensors of FP32 numbers in and out)."""
    b1, b2 = (number(b) for b in betas)
    c1, c2 = (number(1.0 - b) for b in betas)
    if scale is not None:
        g = f32(g * scale)
    m = f32(f32(b1 * m) + f32(c1 * g))
    v = f32(f32(b2 * v) + f32(c2 * f32(g * g)))
    return m, v, f32(torch.sqrt(v))


def updated(p, m, u, step, lr, betas, eps, decay):
    """p' in 64 bits, and a bound on the FP32 form's distance from it."""
    move = lr / (1 - betas[0] ** step) * m / (u * (1 - betas[1] ** step) ** -0.5 + eps)
    # decay and its product 2 roundings of p, the step's 7 (two factors, root * u, + eps, quotient, product, root), the difference 1
    return p * (1 - lr * decay) - move, EPS32 * (3 * p.abs() + 9 * move.abs()) + 1e-45


def _blocks(x):
    return torch.nn.functional.pad(x, (0, -x.numel() % 128)).view(-1, 128)


E4M3 = torch.tensor(sorted({(m / 8 + (1 if e else 0)) * 2.0 ** (max(e, 1) - 7) for e in range(16) for m in range(8)
                            if (e, m) != (15, 7)}), dtype=torch.float64)
Q = torch.tensor([0.0] + [(1 + (c % 16) / 16) * 2.0 ** ((c + 1792) // 16 - 127) for c in range(1, 256)], dtype=torch.float64)


def _nearest(x, grid):
    """Index of the nearest number of a grid, ties to the even index; x >= 0."""
    hi = torch.searchsorted(grid, x).clamp(1, len(grid) - 1)
    lo = hi - 1
    below, above = x - grid[lo], grid[hi] - x
    return torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)


def hold(m, u):
    """8-bit form of m and u (float64 tensors of FP32 numbers): codes and scales of each, blocks of 128."""
    n = m.numel()
    b = _blocks(m)
    top = b.abs().amax(1)
    sm = torch.where(torch.isfinite(b).all(1), f32(top / 448.0), math.nan)
    x = torch.where(sm[:, None] > 0, f32(b / sm[:, None]), 0.0).clamp(-448, 448)
    k = _nearest(x.abs(), E4M3)                    # grid index = code of the magnitude
    mc = torch.where(sm[:, None] > 0, k + 128 * torch.signbit(x).long(), 0).flatten()[:n]
    b = _blocks(u)
    su = torch.where(torch.isfinite(b).all(1), f32(b.amax(1) / 1.9375), math.nan)
    x = torch.where(su[:, None] > 0, f32(b / su[:, None]), 0.0)
    k = torch.where(x > 0, _nearest(x, Q).clamp(1, 255), 0)      # grid index = code
    return mc.to(torch.uint8), sm, k.flatten()[:n].to(torch.uint8), su


def values(mc, sm, uc, su):
    n = mc.numel()
    m = E4M3[(mc & 127).clamp(max=126).long()] * torch.where(mc >= 128, -1.0, 1.0) * sm.repeat_interleave(128)[:n]
    u = f32(Q[uc.long()] * su.repeat_interleave(128)[:n])
    return f32(m), f32(u * u), u
