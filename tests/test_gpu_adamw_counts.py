"""GPU: AdamW with parameters that some steps leave out: each one's bias correction goes by its own number of steps."""
import pytest
import torch

from paper_2606_15682_amd import reqat
from tests import train_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SIZES = [300, 1, 4097, 128]
# which parameters have gradients: one comes late, one rests in between, one step has none at all
STEPS = ["1111", "1011", "1010", "0000", "1110", "0111", "1111"]


@pytest.mark.parametrize("bits", [32, 8])
def test_parameters_left_out_and_stepped_again(bits):
    g = torch.Generator().manual_seed(3)
    params = [(0.1 * torch.randn(n, generator=g)).to(DEV) for n in SIZES]
    lr, betas, eps, decay = 1e-2, (0.9, 0.999), 1e-8, 0.1
    opt = reqat.AdamW(params, lr, betas, eps, decay, state_bits=bits)
    states = [(torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)) for n in SIZES]
    count = [0] * len(SIZES)
    for k, pattern in enumerate(STEPS):
        print("adamw", bits, "step", k, pattern, flush=True)
        grads = [torch.randn(n, generator=g).to(DEV) if on == "1" else None for n, on in zip(SIZES, pattern)]
        before = [p.double().cpu() for p in params]
        opt.step(grads)
        got_m, got_v = opt.moments()
        for i, (n, grad) in enumerate(zip(SIZES, grads)):
            m, v = states[i]
            if grad is None:
                assert torch.equal(params[i].double().cpu(), before[i])
            else:
                count[i] += 1
                m, v, u = ref.states(m, v, grad.double().cpu(), betas)
                want, room = ref.updated(before[i], m, u, count[i], lr, betas, eps, decay)
                assert torch.all((params[i].double().cpu() - want).abs() <= room), (k, i)
                if bits == 8:
                    m, v, _ = ref.values(*ref.hold(m, u))
                states[i] = m, v
            at = opt.offsets[i]
            assert torch.equal(got_m[at:at + n].double().cpu(), m) and torch.equal(got_v[at:at + n].double().cpu(), v)


def test_a_late_parameter_moves_by_the_rate():
    """A constant gradient's first step is lr, whenever it comes."""
    p = [torch.zeros(200, device=DEV), torch.zeros(70, device=DEV)]
    g = [torch.ones(200, device=DEV), torch.ones(70, device=DEV)]
    opt = reqat.AdamW(p, 1e-3, (0.9, 0.999), weight_decay=0.0)
    for _ in range(50):
        opt.step([g[0], None])
    opt.step(g)
    # some ten roundings of FP32, and eps beside 1
    assert torch.allclose(p[1], torch.full((70,), -1e-3, device=DEV), rtol=1e-6)


def test_captured_steps_count_replays():
    p = [torch.zeros(200, device=DEV), torch.zeros(70, device=DEV)]
    g = [torch.ones(200, device=DEV), None]
    opt = reqat.AdamW(p, 1e-3, weight_decay=0.0, captured=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        opt.step(g)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step(g)
    assert opt.steps == 1 and int(opt.step_tensor) == 1
    for k in range(2, 5):
        graph.replay()
        assert int(opt.step_tensor) == k and not p[1].any()
        assert torch.allclose(p[0], torch.full((200,), -1e-3 * k, device=DEV), rtol=1e-4)
    with pytest.raises(ValueError):
        opt.step([g[0], torch.ones(70, device=DEV)])
