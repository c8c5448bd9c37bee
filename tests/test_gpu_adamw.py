"""GPU: AdamW steps against their formulas: states and codes exactly, parameters within FP32's rounding."""
import copy
import math

import pytest
import torch

from paper_2606_15682_amd import reqat
from tests import train_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
SIZES = [1, 2, 3, 4, 5, 127, 128, 129, 1023, 4096, 4097, 10007, 0, 33000]


def _make(sizes, dtype, std=1.0, seed=0):
    g = torch.Generator().manual_seed(len(sizes) + seed)
    return [(torch.randn(n, generator=g) * std).to(dtype).to(DEV) for n in sizes]


class Model:
    """The same steps in 64 bits, states by FP32's rounding."""

    def __init__(self, params, bits, lr, betas, eps, decay):
        self.bits, self.lr, self.betas, self.eps, self.decay, self.t = bits, lr, betas, eps, decay, 0
        self.m = [torch.zeros(p.numel(), dtype=torch.float64) for p in params]
        self.v = [torch.zeros(p.numel(), dtype=torch.float64) for p in params]
        self.codes = [None] * len(params)

    def step(self, i, p, g, scale=None):
        """(p', bound) of parameter i (64 bits), states moved on."""
        m, v, u = ref.states(self.m[i], self.v[i], g, self.betas, scale)
        out = ref.updated(p, m, u, self.t, self.lr, self.betas, self.eps, self.decay)
        if self.bits == 8:
            self.codes[i] = ref.hold(m, u)
            m, v, _ = ref.values(*self.codes[i])
        self.m[i], self.v[i] = m, v
        return out


def _state(opt, i, which):
    at, n = opt.offsets[i], opt.params[i].numel()
    return which[at:at + n].double().cpu()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("pdtype,gdtype", [(F32, BF), (F32, F32), (BF, BF), (BF, F32)])
def test_steps(bits, pdtype, gdtype):
    params = _make(SIZES, pdtype, 0.05)
    copies = [torch.empty_like(p, dtype=BF) if i % 3 else None for i, p in enumerate(params)]
    lr, betas, eps, decay = 3e-3, (0.9, 0.98), 1e-8, 0.1
    opt = reqat.AdamW(params, lr, betas, eps, decay, state_bits=bits, copies=copies)
    model = Model(params, bits, lr, betas, eps, decay)
    for step in range(4):
        print("adamw", bits, pdtype, gdtype, "step", step, flush=True)
        grads = _make(SIZES, gdtype, 10.0 ** (step - 3), seed=10 + step)
        scale = None if step % 2 else torch.tensor([0.37], device=DEV)
        before = [p.double().cpu() for p in params]
        opt.step(grads, grad_scale=scale)
        model.t += 1
        mv, vv = opt.moments()
        for i, n in enumerate(SIZES):
            want, room = model.step(i, before[i], grads[i].double().cpu(), None if scale is None else float(scale))
            assert torch.equal(_state(opt, i, mv), model.m[i]), (i, n)
            assert torch.equal(_state(opt, i, vv), model.v[i]), (i, n)
            got = params[i].double().cpu()
            assert torch.all((got - want).abs() <= room + (1.01 * ref.half_step(BF) * want.abs() if pdtype == BF else 0)), (i, n)
            if bits == 8:
                at, blocks = opt.offsets[i], -(-n // 128)
                mc, ms, vc, vs = model.codes[i]
                assert torch.equal(opt.m[at:at + n].cpu(), mc) and torch.equal(opt.v[at:at + n].cpu(), vc)
                assert torch.equal(opt.m_scale[at // 128:at // 128 + blocks].double().cpu(), ms)
                assert torch.equal(opt.v_scale[at // 128:at // 128 + blocks].double().cpu(), vs)
            if copies[i] is not None:
                if pdtype == F32:
                    assert torch.equal(copies[i], params[i].to(BF))
                else:
                    assert torch.equal(copies[i], params[i])
    assert opt.steps == 4


def test_many_tensors_take_several_launches():
    sizes = [1 + (i * 37) % 300 for i in range(150)]
    params, grads = _make(sizes, F32), _make(sizes, F32, seed=1)
    opt = reqat.AdamW(params, 1e-2, state_bits=8)
    model = Model(params, 8, 1e-2, (0.9, 0.999), 1e-8, 0.01)
    before = [p.double().cpu() for p in params]
    opt.step(grads)
    model.t = 1
    for i in range(150):
        want, room = model.step(i, before[i], grads[i].double().cpu())
        assert torch.all((params[i].double().cpu() - want).abs() <= room), i


def test_left_out_parameters_and_odd_places():
    whole = torch.randn(1000, generator=torch.Generator().manual_seed(2)).to(DEV)
    params = [whole[1:300], whole[300:301], whole[303:999]]          # not on 16-byte boundaries
    kept = whole.clone()
    grads = [torch.ones(600, device=DEV)[1:300], None, torch.full((999,), 2.0, dtype=F32, device=DEV)[303:999]]
    opt = reqat.AdamW(params, 1e-2, weight_decay=0.0)
    opt.step(grads)
    assert torch.equal(whole[[0, 300, 301, 302, 999]], kept[[0, 300, 301, 302, 999]])
    for p, k in ((params[0], kept[1:300]), (params[2], kept[303:999])):
        assert torch.allclose(p, k - 1e-2, atol=1e-6)                # the first step of a constant gradient is lr
    assert not opt.m[opt.offsets[1]:opt.offsets[1] + 128].any()


@pytest.mark.parametrize("bits", [32, 8])
def test_bad_and_extreme_gradients(bits):
    """NaN and Inf stay in their element (32 bits) or block of 128 (8 bits); zeros, tiny and huge gradients."""
    n = 128 * 6
    p, g = torch.ones(n, device=DEV), torch.ones(n, device=DEV)
    g[5], g[130] = math.nan, math.inf
    g[256:384] = 0.0
    g[384:512] = 1e-22                                     # its square is below FP32's smallest number
    g[512:640] = 1e18
    opt = reqat.AdamW([p], 1e-3, eps=1e-8, weight_decay=0.0, state_bits=bits)
    opt.step([g])
    bad = torch.zeros(n, dtype=torch.bool, device=DEV)
    bad[5] = bad[130] = True
    assert torch.equal(torch.isnan(p), bad)
    assert torch.equal(p[256:384], torch.ones(128, device=DEV))
    assert torch.isfinite(p[384:]).all() and torch.allclose(p[512:640], torch.full((128,), 0.999, device=DEV))
    m, v = opt.moments()
    if bits == 8:
        assert torch.isnan(m[:256]).all() and torch.isnan(v[:256]).all() and not opt.m[:256].any()
        assert torch.isfinite(m[256:]).all() and torch.isfinite(v[256:]).all()
    else:
        assert int((~torch.isfinite(m)).sum()) == 2
    opt.step([torch.zeros(n, device=DEV)])
    assert torch.isfinite(p[256:]).all()


def test_wide_range_inside_a_block():
    """Gradients over twelve decades in one block: codes as the rule says, no second moment becomes zero."""
    g = torch.logspace(-12, 0, 128, dtype=torch.float64).float().to(DEV)
    p = torch.zeros(128, device=DEV)
    opt = reqat.AdamW([p], 1e-3, (0.9, 0.999), 1e-8, 0.0, state_bits=8)
    model = Model([p], 8, 1e-3, (0.9, 0.999), 1e-8, 0.0)
    for step in range(3):
        before = p.double().cpu()
        opt.step([g])
        model.t += 1
        want, room = model.step(0, before, g.double().cpu())
        assert torch.all((p.double().cpu() - want).abs() <= room)
        assert torch.equal(opt.m.cpu(), model.codes[0][0]) and torch.equal(opt.v.cpu(), model.codes[0][2])
    assert (opt.v > 0).all()


def test_all_codes_are_read_back():
    opt = reqat.AdamW([torch.zeros(256, device=DEV)], 1e-3, state_bits=8)
    opt.m.copy_(torch.arange(256) % 128 + 128 * (torch.arange(256) // 128))
    opt.m[127], opt.m[255] = 0, 0                          # the format's NaN, which is never written
    opt.v.copy_(torch.arange(256))
    opt.m_scale.copy_(torch.tensor([0.3, 7.0]))
    opt.v_scale.copy_(torch.tensor([1e-4, 5.0]))
    m, v = opt.moments()
    em, ev, _ = ref.values(opt.m.cpu(), opt.m_scale.double().cpu(), opt.v.cpu(), opt.v_scale.double().cpu())
    assert torch.equal(m.double().cpu(), em) and torch.equal(v.double().cpu(), ev)


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps(bits):
    """Replays count on: parameters as eager steps make them, with the rate changed on the device between two."""
    sizes = [1000, 77, 4096]
    eager, graph = _make(sizes, F32), _make(sizes, F32)
    grads = _make(sizes, F32, 0.1, seed=5)
    a = reqat.AdamW(eager, 1e-2, (0.9, 0.95), state_bits=bits)
    b = reqat.AdamW(graph, 1e-2, (0.9, 0.95), state_bits=bits, captured=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.step(grads)
    torch.cuda.current_stream().wait_stream(side)
    a.step(grads)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.step(grads)
    for k in range(4):
        if k == 2:
            a.lr = 3e-3
            b.lr_tensor.fill_(3e-3)
        for x in grads:
            x.mul_(-1.5)
        a.step(grads)
        g.replay()
        torch.cuda.synchronize()
        for p, q in zip(eager, graph):
            # the rate as an FP32 number, and logarithms on the device: the factors may differ by two half steps
            assert torch.all((p - q).abs() <= 4e-7 * p.abs() + 1e-8), k
        assert torch.equal(a.m, b.m) and torch.equal(a.v, b.v)
    assert int(b.step_tensor) == 5


def test_against_plain_recurrence():
    """Ten steps of one number in Python's floats."""
    p = torch.tensor([0.5], device=DEV)
    opt = reqat.AdamW([p], 0.1, (0.9, 0.99), 1e-6, 0.05)
    x, m, v = 0.5, 0.0, 0.0
    for t in range(1, 11):
        grad = math.sin(t)
        opt.step([torch.tensor([grad], device=DEV)])
        m, v = 0.9 * m + 0.1 * grad, 0.99 * v + 0.01 * grad * grad
        x = x * (1 - 0.1 * 0.05) - 0.1 * (m / (1 - 0.9 ** t)) / (math.sqrt(v / (1 - 0.99 ** t)) + 1e-6)
        # each step: 3 half steps of x and some 20 of its move of at most 0.3, over ten steps
        assert abs(float(p) - x) <= t * ref.EPS32 * (3 + 20 * 0.3)


def test_replaced_memory_is_the_one_used():
    """A parameter that was given other memory is stepped there; one that no longer fits is refused."""
    p = [torch.nn.Parameter(torch.ones(300, device=DEV)), torch.nn.Parameter(torch.ones(50, device=DEV))]
    copies = [torch.empty(300, dtype=BF, device=DEV), None]
    opt = reqat.AdamW(p, 1e-2, weight_decay=0.0, copies=copies)
    g = [torch.ones(300, device=DEV), torch.ones(50, device=DEV)]
    opt.step(g)
    old = p[0].data
    kept = old.clone()
    p[0].data = torch.full((300,), 5.0, device=DEV)
    opt.copies[0] = other = torch.zeros(300, dtype=BF, device=DEV)
    opt.step(g)
    assert torch.equal(old, kept) and torch.allclose(p[0].data, torch.full((300,), 4.99, device=DEV), atol=1e-6)
    assert torch.equal(other, p[0].data.to(BF))
    p[0].data = torch.ones(299, device=DEV)
    with pytest.raises(ValueError):
        opt.step(g)
    p[0].data = p[1].data
    with pytest.raises(ValueError):
        opt.step(g)
    assert opt.steps == 2


def test_gradients_in_odd_places():
    """States lie at multiples of 128; parameters, gradients and copies anywhere: every alignment of them, both state widths."""
    n = 1000
    for bits in (32, 8):
        for off in range(1, 8):
            wide = torch.randn(n + 8, generator=torch.Generator().manual_seed(off)).to(DEV)
            grad = torch.randn(n + 8, generator=torch.Generator().manual_seed(9 + off)).to(BF).to(DEV)
            low = torch.zeros(n + 8, dtype=BF, device=DEV)
            a, b = wide.clone(), wide[off:off + n].clone()
            one = reqat.AdamW([a[off:off + n]], 1e-2, state_bits=bits, copies=[low[off:off + n]])
            two = reqat.AdamW([b], 1e-2, state_bits=bits)
            one.step([grad[off:off + n]])
            two.step([grad[off:off + n].clone()])
            assert torch.equal(a[off:off + n], b) and torch.equal(a[:off], wide[:off]) and torch.equal(a[off + n:], wide[off + n:])
            assert torch.equal(low[off:off + n], b.to(BF)) and not low[:off].any() and not low[off + n:].any()
            assert torch.equal(one.m, two.m) and torch.equal(one.v, two.v)


@pytest.mark.parametrize("bits", [32, 8])
def test_copied_and_assigned_states(bits):
    """A deep copy steps its own parameters and states; assigned buffers are the ones used, ones that do not fit are refused."""
    p = _make([300, 77], F32)
    grads = _make([300, 77], F32, seed=3)
    a = reqat.AdamW(p, 1e-2, state_bits=bits)
    a.step(grads)
    b = copy.deepcopy(a)
    kept = [t.clone() for t in (a.m, a.v, *p)]
    b.step(grads)
    assert all(torch.equal(x, y) for x, y in zip(kept, (a.m, a.v, *p)))
    assert b.steps == 2 and not torch.equal(b.params[0], p[0])
    a.step(grads)
    assert torch.equal(a.m, b.m) and torch.equal(a.v, b.v) and all(torch.equal(x, y) for x, y in zip(p, b.params))
    old = a.m
    before = old.clone()
    a.m = torch.zeros_like(old)
    a.step(grads)
    assert torch.equal(old, before) and a.m.any()
    a.v = a.v[:-128].clone()
    with pytest.raises(ValueError):
        a.step(grads)
    a.v = torch.zeros(a.m.numel(), dtype=torch.float64, device=DEV)
    with pytest.raises(TypeError):
        a.step(grads)
