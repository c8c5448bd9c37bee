"""Timing cases of the operators that surround the quantized linear layers in a
training step: the embedding and its gradient, the norm before each product, the
policy loss over the logits, and the AdamW step on the master weights, through the
calls of ``paper_2606_15682_amd.reqat``.

Hidden sizes, MLP widths and the vocabulary are those of the layers that the
library's benchmark names.  Each case has a ``kind``:
  ``policy``   the clipped policy loss with a KL term over bfloat16 or 32-bit logits.
               ``mode`` loss: the loss and the per-token statistics; grad: those and
               the gradient in one pass; backward: the gradient from the statistics.
  ``norm``     layer norm (centred) or root-mean-square norm (not centred).
               ``mode`` forward, or backward with the gradients of weight and bias.
  ``embed``    ``mode`` forward: rows of the table times a factor; fresh: the gradient
               of the whole table; add: the gradient added to one that is there (a
               table that is also the output layer's).  Token ids are spread evenly over
               their logarithm, as words are, and a few positions are padding.
  ``adamw``    one step over a list of tensors, states in 32 or in 8 bits, with a
               factor on the gradients (clipping) and bfloat16 copies of 32-bit weights.

Where ``own`` is false everything is elementary torch operations in 32 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
VOCAB = 152064
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ELT = {"bf16": 2, "f32": 4}

# policy loss
CLIP_LOW, CLIP_HIGH = 0.2, 0.28
# norm
EPS = 1e-6
# AdamW
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-4, 0.9, 0.95, 1e-8, 0.1
STEP = 37                    # the step that is taken
BLOCK = 128                  # elements to a scale of the 8-bit states


def listed():
    return [
        # one short answer under a small vocabulary of odd size: launches and latency count
        {"name": "policy_grad_t24_v32003", "kind": "policy", "mode": "grad", "T": 24, "V": 32003, "dtype": "bf16",
         "kl": 0.04, "temp": 1.0, "prompt": 0.0},
        # a training batch: answers behind prompts, which carry no weight; loss and gradient
        {"name": "policy_grad_t4096_v152064", "kind": "policy", "mode": "grad", "T": 4096, "V": VOCAB, "dtype": "bf16",
         "kl": 0.04, "temp": 1.0, "prompt": 0.25},
        # the loss alone, on 32-bit logits sampled at a temperature: a validation batch
        {"name": "policy_loss_t1001_v152064_f32", "kind": "policy", "mode": "loss", "T": 1001, "V": VOCAB, "dtype": "f32",
         "kl": 0.0, "temp": 0.6, "prompt": 0.0},
        # a few rows of the smallest model
        {"name": "norm_fwd_m16_k1536", "kind": "norm", "mode": "forward", "M": 16, "K": 1536, "dtype": "bf16",
         "wdtype": "bf16", "center": False, "bias": False},
        # a ragged batch of the 7B-like size, centred, with a bias
        {"name": "norm_fwd_m9001_k3584", "kind": "norm", "mode": "forward", "M": 9001, "K": 3584, "dtype": "bf16",
         "wdtype": "f32", "center": True, "bias": True},
        # the backward pass of a 14B-like training batch
        {"name": "norm_bwd_m8192_k5120", "kind": "norm", "mode": "backward", "M": 8192, "K": 5120, "dtype": "bf16",
         "wdtype": "f32", "center": True, "bias": True},
        # lookup of a batch of the 7B-like size
        {"name": "embed_fwd_t8192_k3584", "kind": "embed", "mode": "forward", "T": 8192, "K": 3584, "V": VOCAB,
         "dtype": "bf16", "gdtype": "bf16", "scale": 1.0},
        # a short sequence's gradient, added to the one that the output layer left
        {"name": "embed_add_t333_k1536", "kind": "embed", "mode": "add", "T": 333, "K": 1536, "V": VOCAB,
         "dtype": "bf16", "gdtype": "bf16", "scale": 1.0},
        # a batch's gradient of the 14B-like table, in 32 bits, from nothing
        {"name": "embed_fresh_t8192_k5120", "kind": "embed", "mode": "fresh", "T": 8192, "K": 5120, "V": VOCAB,
         "dtype": "bf16", "gdtype": "f32", "scale": 2.0},
        # norm weights and biases of a few layers: many small tensors, latency
        {"name": "adamw32_norms", "kind": "adamw", "set": "norms", "count": 60, "total": 0, "bits": 32, "pdtype": "f32",
         "gdtype": "bf16", "copy": True, "clip": False},
        # a 14B-like layer with its master weights and the copies that the quantizer reads
        {"name": "adamw32_14b_layer", "kind": "adamw", "set": "14b", "count": 0, "total": 0, "bits": 32, "pdtype": "f32",
         "gdtype": "bf16", "copy": True, "clip": True},
        # two 1.5B-like layers with 8-bit states
        {"name": "adamw8_1.5b_layers", "kind": "adamw", "set": "1.5b", "count": 2, "total": 0, "bits": 8, "pdtype": "f32",
         "gdtype": "bf16", "copy": True, "clip": True},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    """Seconds a pass needs at a rate near this card's."""
    return work(case)["bytes"] / 4e12


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["policy", "policy", "norm", "norm", "embed", "embed", "adamw", "adamw"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        case = {"kind": kind}
        if kind == "policy":
            case.update(mode=rng.choice(["loss", "grad", "grad", "backward"]), T=_log_uniform(rng, 1, 8192),
                        V=rng.choice([VOCAB, _log_uniform(rng, 500, VOCAB)]), dtype=dtype,
                        kl=rng.choice([0.0, 0.04]), temp=rng.choice([1.0, 0.6]), prompt=rng.choice([0.0, 0.25, 0.5]))
        elif kind == "norm":
            case.update(mode=rng.choice(["forward", "backward"]), M=_log_uniform(rng, 1, 16384),
                        K=rng.choice([1536, 3584, 5120, _log_uniform(rng, 64, 27648)]), dtype=dtype,
                        wdtype=rng.choice(["bf16", "f32"]), center=rng.random() < 0.5, bias=rng.random() < 0.5)
        elif kind == "embed":
            case.update(mode=rng.choice(["forward", "fresh", "add"]), T=_log_uniform(rng, 1, 32768),
                        K=rng.choice([1536, 3584, 5120, _log_uniform(rng, 64, 8192)]),
                        V=rng.choice([VOCAB, _log_uniform(rng, 500, VOCAB)]), dtype=dtype,
                        gdtype=rng.choice([dtype, "f32"]), scale=rng.choice([1.0, 2.0]))
        else:
            pdtype = rng.choice(["f32", "f32", "bf16"])
            count = _log_uniform(rng, 1, 200)
            case.update(set="random", count=count, total=max(count, _log_uniform(rng, 1000, 1.5e8)),
                        bits=rng.choice([32, 8]), pdtype=pdtype, gdtype=rng.choice(["bf16", "f32"]),
                        copy=pdtype == "f32" and rng.random() < 0.75, clip=rng.random() < 0.5)
        if _cost(case) <= most:
            return case


# ------------------------------------------------------------------ shapes and work

def _rng(case):
    return random.Random("%s" % sorted((k, v) for k, v in case.items() if k != "name"))


def _masked(case):
    """Rows of a policy case without weight: the prompts' tokens, at the start of each of a few sequences."""
    r, T = _rng(case), case["T"]
    count = min(T, 1 + T // 512)
    cuts = [0] + sorted(r.sample(range(1, T), count - 1)) + [T]
    out = torch.zeros(T, dtype=torch.bool)
    for a, b in zip(cuts, cuts[1:]):
        n = int((b - a) * case["prompt"] * r.uniform(0.8, 1.2))
        out[a:a + min(n, b - a - 1)] = True
    return out


def _sizes(case):
    """Elements of the tensors of an AdamW case."""
    if case["set"] == "norms":
        widths = [1536, 1536, 2048, 257, 8960]
        return [widths[i % len(widths)] for i in range(case["count"])]
    if case["set"] == "14b":
        return [7168 * 5120, 7168, 5120 * 5120, 27648 * 5120, 13824 * 5120, 5120, 5120]
    if case["set"] == "1.5b":
        return [2048 * 1536, 2048, 1536 * 1536, 17920 * 1536, 8960 * 1536, 1536, 1536, 1537 * 3] * case["count"]
    r = _rng(case)
    shares = [r.expovariate(1.0) ** 2 + 1e-9 for _ in range(case["count"])]
    return [max(1, int(case["total"] * s / sum(shares))) for s in shares]


def _layout(case):
    """Where the tensors of an AdamW case begin in one buffer (at multiples of BLOCK), and the buffer's size."""
    at, out = 0, []
    for n in _sizes(case):
        out.append((at, n))
        at += -(-n // BLOCK) * BLOCK
    return out, at


def _ids(case, seed):
    """Token ids, evenly spread over their logarithm; about one in a hundred positions is padding."""
    gen = _generator(seed, 11)
    u = torch.rand(case["T"], generator=gen, device=DEV, dtype=torch.float64)
    ids = (torch.exp(u * math.log(case["V"] + 1.0)) - 1.0).to(torch.int32).clamp(0, case["V"] - 1)
    ids[torch.rand(case["T"], generator=gen, device=DEV) < 0.01] = -1
    return ids


def _distinct(case):
    """About how many different ids an embedding case has (the draw above, in expectation)."""
    T, top = case["T"], math.log(case["V"] + 1.0)
    edges = sorted({0, *(int(1.1 ** i) for i in range(200) if 1.1 ** i < case["V"]), case["V"]})
    total = 0.0
    for a, b in zip(edges, edges[1:]):
        p = (math.log(b + 1.0) - math.log(a + 1.0)) / top / (b - a)
        total += (b - a) * -math.expm1(T * 0.99 * math.log1p(-min(p, 1 - 1e-12)))
    return total


def work(case):
    """Bytes and operations of one pass: every input read once, every output written once."""
    kind = case["kind"]
    if kind == "policy":
        T, row = case["T"], case["V"] * ELT[case["dtype"]]
        seen = T - int(_masked(case).sum())
        moved = seen * row + 32 * T + (T * row if case["mode"] != "loss" else 0)
        return {"bytes": moved, "flops": seen * case["V"] * (6 if case["mode"] == "loss" else 9)}
    if kind == "norm":
        n, e, w = case["M"] * case["K"], ELT[case["dtype"]], case["K"] * ELT[case["wdtype"]]
        if case["mode"] == "forward":
            return {"bytes": 2 * n * e + w * (1 + case["bias"]) + 8 * case["M"], "flops": 8 * n}
        return {"bytes": 3 * n * e + w * (2 + case["bias"]) + 8 * case["M"], "flops": 14 * n}
    if kind == "embed":
        n, e, g = case["T"] * case["K"], ELT[case["dtype"]], ELT[case["gdtype"]]
        rows = _distinct(case)
        if case["mode"] == "forward":
            return {"bytes": n * e + rows * case["K"] * e + 4 * case["T"], "flops": n}
        if case["mode"] == "fresh":
            return {"bytes": n * e + case["V"] * case["K"] * g + 4 * case["T"], "flops": 2 * n}
        return {"bytes": n * e + 2 * rows * case["K"] * g + 4 * case["T"], "flops": 2 * n}
    n = sum(_sizes(case))           # without what lies between the tensors
    state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK + 8     # 8 bits: the states' values are returned too
    return {"bytes": int(n * (2 * ELT[case["pdtype"]] + ELT[case["gdtype"]] + (2 if case["copy"] else 0) + state)),
            "flops": 20 * n}


# ------------------------------------------------------------------ inputs

def _generator(seed, stream):
    return torch.Generator(device=DEV).manual_seed(1000003 * (seed % (1 << 40)) + stream)


def _normal(gen, shape, dtype, std=1.0):
    """Normal numbers, made in pieces of rows."""
    out = torch.empty(shape, dtype=DTYPES[dtype], device=DEV)
    flat = out.view(shape[0], -1)
    piece = max(1, (1 << 27) // max(1, flat.shape[1]))
    for i in range(0, shape[0], piece):
        x = torch.randn((min(piece, shape[0] - i), flat.shape[1]), generator=gen, device=DEV)
        flat[i:i + piece] = (x * std).to(out.dtype)
    return out


def _policy_inputs(case, seed):
    """Logits and what a policy's step holds beside them.  No ratio lies within a thousandth of a clipping border,
    where the gradient jumps."""
    T, V = case["T"], case["V"]
    gen = _generator(seed, 1)
    logits = _normal(gen, (T, V), case["dtype"], 2.0)
    targets = torch.randint(0, V, (T,), generator=gen, device=DEV, dtype=torch.int32)
    at = torch.arange(T, device=DEV)
    lift = 12.0 + 3.0 * torch.randn(T, generator=gen, device=DEV)
    logits[at, targets.long()] = lift.to(logits.dtype)          # sampled tokens are likely ones
    delta = 0.15 * torch.randn(T, generator=gen, device=DEV)
    for border in (math.log1p(-CLIP_LOW), math.log1p(CLIP_HIGH)):
        delta = torch.where((delta - border).abs() < 1e-3, delta.new_tensor(border + 2e-3), delta)
    lp = torch.empty(T, device=DEV)
    for i in range(0, T, 512):
        z = logits[i:i + 512].float() / case["temp"]
        lp[i:i + 512] = z.gather(1, targets[i:i + 512, None].long())[:, 0] - torch.logsumexp(z, 1)
    out = {"logits": logits, "targets": targets, "old": lp - delta,
           "adv": torch.randn(T, generator=gen, device=DEV),
           "ref": lp + 0.2 * torch.randn(T, generator=gen, device=DEV) if case["kl"] else None}
    seen = ~_masked(case).to(DEV)
    out["weights"] = seen.float() / seen.sum()
    return out


def _norm_inputs(case, seed):
    """Activations with a few channels of twenty times the size, and means off zero."""
    M, K = case["M"], case["K"]
    gen = _generator(seed, 2)
    wide = torch.where(torch.rand(K, generator=gen, device=DEV) < 0.01, 20.0, 1.0)
    x = torch.randn((M, K), generator=gen, device=DEV) * wide + 0.5 * torch.randn((M, 1), generator=gen, device=DEV)
    out = {"x": x.to(DTYPES[case["dtype"]]),
           "w": (1.0 + 0.2 * torch.randn(K, generator=gen, device=DEV)).to(DTYPES[case["wdtype"]]),
           "b": (0.1 * torch.randn(K, generator=gen, device=DEV)).to(DTYPES[case["wdtype"]]) if case["bias"] else None}
    if case["mode"] == "backward":
        out["dy"] = _normal(gen, (M, K), case["dtype"], 1e-2)
        x = out["x"].double()
        mu = x.mean(1) if case["center"] else x.new_zeros(M)
        rstd = (((x - mu[:, None]) ** 2).mean(1) + EPS) ** -0.5
        out["stats"] = torch.stack([mu, rstd], 1).float()
    return out


def _embed_inputs(case, seed):
    gen = _generator(seed, 3)
    out = {"ids": _ids(case, seed)}
    if case["mode"] == "forward":
        out["table"] = _normal(gen, (case["V"], case["K"]), case["dtype"], 0.02)
    else:
        out["dy"] = _normal(gen, (case["T"], case["K"]), case["dtype"], 1e-2)
        if case["mode"] == "add":
            out["base"] = _normal(gen, (case["V"], case["K"]), case["gdtype"], 1e-2)
    return out


def _adamw_inputs(case, seed):
    """Weights, gradients and states of a run that has gone on for a while: the tensors one after the other in a buffer
    for each (u holds the square roots of the second moments); 8-bit states as codes and scales."""
    gen = _generator(seed, 4)
    layout, size = _layout(case)
    out = {"p": torch.zeros(size, dtype=DTYPES[case["pdtype"]], device=DEV),
           "g": torch.zeros(size, dtype=DTYPES[case["gdtype"]], device=DEV),
           "m": torch.zeros(size, device=DEV), "u": torch.zeros(size, device=DEV)}
    spread = random.Random(seed)
    for at, n in layout:
        std = math.exp(spread.gauss(-7.0, 1.0))
        here = slice(at, at + n)
        out["p"][here] = 0.02 * torch.randn(n, generator=gen, device=DEV)
        out["g"][here] = std * torch.randn(n, generator=gen, device=DEV)
        out["m"][here] = 0.3 * std * torch.randn(n, generator=gen, device=DEV)
        out["u"][here] = (0.3 + torch.rand(n, generator=gen, device=DEV)) * std
    if case["bits"] == 8:
        out["m"], out["u"] = _hold_m(out["m"]), _hold_u(out["u"])
    out["scale"] = torch.full((1,), 0.83, device=DEV) if case["clip"] else None
    return out


def prepare(case, seed):
    state = {"case": case}
    state.update({"policy": _policy_inputs, "norm": _norm_inputs, "embed": _embed_inputs,
                  "adamw": _adamw_inputs}[case["kind"]](case, seed))
    if case["kind"] == "policy" and case["mode"] == "backward":
        state["stats"] = _plain_policy(state, False)[1]
    if own:
        from paper_2606_15682_amd import reqat
        state["reqat"] = reqat
    if case["kind"] == "adamw":
        state["copies"] = state["p"].to(torch.bfloat16) if case["copy"] else None
        if own:
            split = lambda t: [t[at:at + n] for at, n in _layout(case)[0]]
            opt = reqat.AdamW(split(state["p"]), lr=LR, betas=(BETA1, BETA2), eps=ADAM_EPS, weight_decay=DECAY,
                              state_bits=case["bits"], copies=split(state["copies"]) if case["copy"] else None)
            if case["bits"] == 32:
                held, new = (opt.m, opt.v), (state.pop("m"), state.pop("u").square_())
            else:
                held, new = (opt.m, opt.m_scale, opt.v, opt.v_scale), state.pop("m") + state.pop("u")
            for a, b in zip(held, new):
                a.copy_(b)
            opt.steps = STEP - 1
            state.update(opt=opt, grads=split(state["g"]))
        elif case["bits"] == 32:
            state["v"] = state.pop("u").square_()
    return state


# ------------------------------------------------------------------ plain forms

def _plain_policy(state, gradient):
    case, V = state["case"], state["case"]["V"]
    logits, weights, T = state["logits"], state["weights"], state["logits"].shape[0]
    stats = torch.zeros((T, 4), device=DEV)
    parts = torch.zeros((T, 4), dtype=torch.float64, device=DEV)
    grad = torch.empty_like(logits) if gradient else None
    for i in range(0, T, 512):
        rows = slice(i, min(T, i + 512))
        w = weights[rows]
        z = logits[rows].float() / case["temp"]
        hot = state["targets"][rows].long()[:, None]
        top = z.amax(1, keepdim=True)
        e = torch.exp(z - top)
        total = e.sum(1, keepdim=True)
        lp = ((z.gather(1, hot) - top) - torch.log(total))[:, 0]
        r = torch.exp(lp - state["old"][rows])
        adv = state["adv"][rows]
        surr = -torch.minimum(r * adv, r.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * adv)
        out = ((adv > 0) & (r > 1.0 + CLIP_HIGH)) | ((adv < 0) & (r < 1.0 - CLIP_LOW))
        d = torch.where(out, torch.zeros_like(r), -adv * r)
        kl = torch.zeros_like(r, dtype=torch.float64)
        if case["kl"]:
            x = state["ref"][rows] - lp
            kl = torch.expm1(x.double()) - x.double()        # a difference of close numbers: in 64 bits
            d = d - case["kl"] * torch.expm1(x)
        seen = w != 0
        row = torch.stack([lp, (top + torch.log(total))[:, 0], w * d, r], 1)
        stats[rows] = torch.where(seen[:, None], row, torch.zeros_like(row))
        part = w.double()[:, None] * torch.stack([surr.double() + case["kl"] * kl, surr.double(), kl, out.double()], 1)
        parts[rows] = torch.where(seen[:, None], part, torch.zeros_like(part))
        if gradient:
            g = (e / total).neg_()
            g.scatter_add_(1, hot, torch.ones_like(g[:, :1]))
            grad[rows] = torch.where(seen[:, None], g * (stats[rows, 2:3] / case["temp"]), 0.0).to(grad.dtype)
    return parts.sum(0).float(), stats, grad


def _plain_policy_backward(state):
    case, logits, stats = state["case"], state["logits"], state["stats"]
    grad = torch.empty_like(logits)
    for i in range(0, logits.shape[0], 512):
        z = logits[i:i + 512].float() / case["temp"]
        g = torch.exp(z - stats[i:i + 512, 1:2]).neg_()
        g.scatter_add_(1, state["targets"][i:i + 512, None].long(), torch.ones_like(g[:, :1]))
        d = stats[i:i + 512, 2:3] / case["temp"]
        grad[i:i + 512] = torch.where(d != 0, g * d, 0.0).to(grad.dtype)
    return grad


def _plain_norm(state):
    case, x, w = state["case"], state["x"].float(), state["w"].float()
    if case["mode"] == "forward":
        mu = x.mean(1, keepdim=True) if case["center"] else x.new_zeros((x.shape[0], 1))
        xc = x - mu
        rstd = 1.0 / torch.sqrt((xc * xc).mean(1, keepdim=True) + EPS)
        y = xc * rstd * w
        if case["bias"]:
            y = y + state["b"].float()
        return y.to(state["x"].dtype), torch.cat([mu, rstd], 1)
    mu, rstd = state["stats"][:, :1], state["stats"][:, 1:]
    dy = state["dy"].float()
    xh = (x - mu) * rstd
    g = dy * w
    dx = g - xh * (g * xh).mean(1, keepdim=True)
    if case["center"]:
        dx = dx - g.mean(1, keepdim=True)
    dw = (dy * xh).sum(0).to(state["w"].dtype)
    return (rstd * dx).to(state["x"].dtype), dw, dy.sum(0).to(state["w"].dtype) if case["bias"] else None


def _plain_embed(state):
    case, ids = state["case"], state["ids"].long()
    valid = ids >= 0
    if case["mode"] == "forward":
        out = state["table"][ids.clamp(min=0)].float() * case["scale"]
        return torch.where(valid[:, None], out, 0.0).to(state["table"].dtype)
    total = torch.zeros((case["V"], case["K"]), device=DEV)
    total.index_add_(0, ids[valid], state["dy"][valid].float())
    total *= case["scale"]
    if case["mode"] == "add":
        state["base"].copy_((state["base"].float() + total).to(state["base"].dtype))
        return state["base"]
    return total.to(DTYPES[case["gdtype"]])


def _over(x, y):
    """x / y rounded once; by a number, torch multiplies with its rounded reciprocal."""
    return x / torch.full_like(x, y)


def _hold_m(m):
    """First moments in 8 bits: E4M3 codes of m / s, s = (largest of the block) / 448."""
    b = m.view(-1, BLOCK)
    s = _over(b.abs().amax(1), 448.0)
    x = torch.where(s[:, None] > 0, b / s[:, None], 0.0)
    return x.to(torch.float8_e4m3fn).view(torch.uint8).flatten(), s


def _hold_u(u):
    """Square roots of second moments in 8 bits: value 2^-15 (1 + 1/16) .. 1.9375, four bits behind the binary point,
    times s = (largest of the block) / 1.9375; code 0 is zero, and no other number becomes zero."""
    b = u.view(-1, BLOCK)
    s = _over(b.amax(1), 1.9375)
    x = torch.where(s[:, None] > 0, b / s[:, None], 0.0)
    bits = x.view(torch.int32)
    code = ((bits + 0x3FFFF + ((bits >> 19) & 1)) >> 19) - 0x700
    code = torch.where(x > 0, code.clamp(1, 255), 0)
    return code.to(torch.uint8).flatten(), s


def _value_m(codes, s):
    return codes.view(torch.float8_e4m3fn).float() * s.repeat_interleave(BLOCK)


def _value_u(codes, s):
    value = ((codes.to(torch.int32) + 0x700) << 19).view(torch.float32)
    return torch.where(codes > 0, value, 0.0) * s.repeat_interleave(BLOCK)


def _plain_adamw(state):
    case = state["case"]
    b1, b2, c1, c2 = (torch.tensor(x, dtype=torch.float32, device=DEV) for x in (BETA1, BETA2, 1 - BETA1, 1 - BETA2))
    step = LR / (1 - BETA1 ** STEP)
    root = (1 - BETA2 ** STEP) ** -0.5
    g = state["g"].float()
    if state["scale"] is not None:
        g = g * state["scale"]
    if case["bits"] == 32:
        m, v = state["m"], state["v"]
    else:
        m, v = _value_m(*state["m"]), _value_u(*state["u"])
        v = v * v
    m = b1 * m + c1 * g                         # every product and sum rounded
    v = b2 * v + c2 * (g * g)
    u = torch.sqrt(v.double()).float()          # rounded once, which decides 8-bit codes
    x = state["p"].float()
    x = x * (1 - LR * DECAY) - step * (m / (u * root + ADAM_EPS))
    state["p"].copy_(x.to(state["p"].dtype))
    if case["copy"]:
        state["copies"].copy_(x.to(torch.bfloat16))
    if case["bits"] == 32:
        state["m"], state["v"] = m, v
    else:
        state["m"], state["u"] = _hold_m(m), _hold_u(u)
        m, v = _value_m(*state["m"]), _value_u(*state["u"])
        v = v * v
    return state["p"], m, v, state["copies"]


# ------------------------------------------------------------------ one pass

def run(state):
    case = state["case"]
    kind, mode = case["kind"], case.get("mode")
    if not own:
        if kind == "policy":
            if mode == "backward":
                return _plain_policy_backward(state)
            loss, stats, grad = _plain_policy(state, mode == "grad")
            return (loss, stats) if mode == "loss" else (loss, stats, grad)
        return {"norm": _plain_norm, "embed": _plain_embed, "adamw": _plain_adamw}[kind](state)
    reqat = state["reqat"]
    if kind == "policy":
        if mode == "backward":
            return reqat.policy_loss_backward(state["logits"], state["targets"], state["stats"],
                                              temperature=case["temp"])
        call = reqat.policy_loss if mode == "loss" else reqat.policy_loss_grad
        return call(state["logits"], state["targets"], state["old"], state["adv"], ref_logp=state["ref"],
                    weights=state["weights"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=case["kl"],
                    temperature=case["temp"])
    if kind == "norm":
        if mode == "forward":
            return reqat.layer_norm(state["x"], state["w"], state["b"], eps=EPS, center=case["center"])
        return reqat.layer_norm_backward(state["dy"], state["x"], state["w"], state["stats"], center=case["center"],
                                         bias=case["bias"])
    if kind == "embed":
        if mode == "forward":
            return reqat.embedding(state["ids"], state["table"], scale=case["scale"])
        if mode == "add":
            return reqat.embedding_backward(state["dy"], state["ids"], case["V"], scale=case["scale"],
                                            out=state["base"], accumulate=True)
        return reqat.embedding_backward(state["dy"], state["ids"], case["V"], scale=case["scale"],
                                        out_dtype=DTYPES[case["gdtype"]])
    opt = state["opt"]
    opt.steps = STEP - 1                        # every pass is that step, as in the plain form
    opt.step(state["grads"], grad_scale=state["scale"])
    m, v = (opt.m, opt.v) if case["bits"] == 32 else opt.moments()
    return state["p"], m, v, state["copies"]


# ------------------------------------------------------------------ the definition in 64 bits

def _exact_policy(case, seed):
    inp = _policy_inputs(case, seed)
    T, V = inp["logits"].shape
    w = inp["weights"].double()
    stats = torch.zeros((T, 4), dtype=torch.float64, device=DEV)
    terms = torch.zeros((T, 4), dtype=torch.float64, device=DEV)
    grad = torch.zeros((T, V), dtype=torch.float64, device=DEV) if case["mode"] != "loss" else None
    given = _plain_policy(dict(inp, case=case), False)[1].double() if case["mode"] == "backward" else None
    for t0 in range(0, T, 128):
        idx = torch.arange(t0, min(T, t0 + 128), device=DEV)
        idx = idx[w[idx] != 0]
        if not len(idx):
            continue
        z = inp["logits"][idx].double().div_(case["temp"])
        y = inp["targets"][idx].long()
        lse = torch.logsumexp(z, dim=1)
        lp = z[torch.arange(len(idx), device=DEV), y] - lse
        ratio, a = (lp - inp["old"][idx].double()).exp(), inp["adv"][idx].double()
        low, high = 1.0 - CLIP_LOW, 1.0 + CLIP_HIGH
        gain = torch.where(a >= 0, ratio.clamp(max=high), ratio.clamp(min=low)) * a
        stuck = torch.where(a >= 0, ratio > high, ratio < low) & (a != 0)
        slope = torch.where(stuck, 0.0, -ratio * a)
        penalty = torch.zeros_like(lp)
        if case["kl"]:
            gap = inp["ref"][idx].double() - lp
            penalty = gap.expm1() - gap
            slope = slope - case["kl"] * gap.expm1()
        terms[idx] = w[idx, None] * torch.stack([case["kl"] * penalty - gain, -gain, penalty, stuck.double()], dim=1)
        stats[idx] = torch.stack([lp, lse, w[idx] * slope, ratio], dim=1)
        if grad is not None:
            # the backward pass alone starts from 32-bit statistics, which are its inputs
            lse, slope = (lse, w[idx] * slope) if given is None else (given[idx, 1], given[idx, 2])
            p = z.sub_(lse[:, None]).exp_().neg_()
            p[torch.arange(len(idx), device=DEV), y] += 1.0
            grad[idx] = p.mul_((slope / case["temp"])[:, None])
    if case["mode"] == "backward":
        return grad
    return (terms.sum(dim=0), stats) + ((grad,) if case["mode"] == "grad" else ())


def _exact_norm(case, seed):
    inp = _norm_inputs(case, seed)
    x, w = inp["x"].double(), inp["w"].double()
    if case["mode"] == "forward":
        mean = x.sum(1) / case["K"] if case["center"] else torch.zeros(case["M"], dtype=torch.float64, device=DEV)
        x = x - mean[:, None]
        scale = torch.rsqrt(x.square().sum(1) / case["K"] + EPS)
        y = x * scale[:, None] * w[None, :]
        return (y if inp["b"] is None else y + inp["b"].double()), torch.stack([mean, scale], dim=1)
    mean, scale = inp["stats"].double().unbind(1)
    hat = (x - mean[:, None]) * scale[:, None]
    up = inp["dy"].double()
    dw, db = (up * hat).sum(0), up.sum(0)
    g = up * w[None, :]
    shared = hat * ((g * hat).sum(1) / case["K"])[:, None]
    if case["center"]:
        shared += (g.sum(1) / case["K"])[:, None]
    return (g - shared) * scale[:, None], dw, db if case["bias"] else None


def _exact_embed(case, seed):
    inp = _embed_inputs(case, seed)
    where = torch.nonzero(inp["ids"] >= 0)[:, 0]
    rows = inp["ids"][where].long()
    if case["mode"] == "forward":
        out = torch.zeros((case["T"], case["K"]), dtype=torch.float64, device=DEV)
        out[where] = inp["table"][rows].double() * case["scale"]
        return out
    out = inp["base"].double() if case["mode"] == "add" else \
        torch.zeros((case["V"], case["K"]), dtype=torch.float64, device=DEV)
    return out.index_add_(0, rows, inp["dy"][where].double(), alpha=case["scale"])


def _single(x):
    return x.to(torch.float32).to(torch.float64)


def _exact_held(x, top, digits, lowest):
    """What a block format holds of x (64 bits, 32-bit values): x / s rounded to `digits` bits behind the binary point,
    in steps that stop shrinking below 2^lowest, times s."""
    rows = x.view(-1, BLOCK)
    s = _single(rows.abs().max(dim=1, keepdim=True).values / top)
    q = _single(torch.where(s > 0, rows / s, 0.0))
    power = torch.where(q == 0, 1.0, 0.5 * q.abs() / torch.frexp(q.abs())[0])       # 2^floor(log2 |q|), exact
    step = power.clamp(min=2.0 ** lowest) * 2.0 ** -digits
    return torch.round(q / step) * step, s


def _exact_adamw(case, seed):
    inp = _adamw_inputs(case, seed)
    b1, b2, c1, c2 = (BETA1, BETA2, 1 - BETA1, 1 - BETA2)
    if case["bits"] == 8:                       # the definition takes every step of the states to 32 bits
        b1, b2, c1, c2 = (float(torch.tensor(x, dtype=torch.float32)) for x in (b1, b2, c1, c2))
    near = _single if case["bits"] == 8 else (lambda x: x)
    p, g, m, u = inp["p"].double(), inp["g"].double(), inp["m"], inp["u"]
    if inp["scale"] is not None:
        g = near(g * inp["scale"].double())
    if case["bits"] == 8:
        u = _value_u(*u).double()
        m, v = _value_m(*m).double(), near(u * u)
    else:
        m, v = m.double(), (u * u).double()
    m = near(near(b1 * m) + near(c1 * g))
    v = near(near(b2 * v) + near(c2 * near(g * g)))
    p = p * (1 - LR * DECAY) - LR / (1 - BETA1 ** STEP) * m / (torch.sqrt(v / (1 - BETA2 ** STEP)) + ADAM_EPS)
    if case["bits"] == 8:
        root = near(torch.sqrt(v)).view(-1, BLOCK)
        q, s = _exact_held(m, 448.0, 3, -6)
        m = _single(q * s).flatten()
        q, s = _exact_held(root, 1.9375, 4, -1000)
        q = torch.where(root > 0, q.clamp(min=1.0625 * 2.0 ** -15), 0.0)
        v = _single(_single(q * s) ** 2).flatten()
    return p, m, v, p if case["copy"] else None


def exact(case, seed):
    kinds = {"policy": _exact_policy, "norm": _exact_norm, "embed": _exact_embed, "adamw": _exact_adamw}
    return kinds[case["kind"]](case, seed)
