"""GPU: the training operators beyond 2^31 elements: what lies behind them is what a small call of the same rows gives, to the bit."""
import pytest
import torch

from paper_2606_15682_amd import reqat

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def room():
    if torch.cuda.get_device_properties(0).total_memory < 100 << 30:
        pytest.skip("needs 100 GiB of memory")
    yield
    torch.cuda.empty_cache()


def _rand(rows, cols, dtype):
    """A row of numbers of its own for each of the first and last thousand rows, and something between."""
    x = torch.empty((rows, cols), dtype=dtype, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(rows)
    part = torch.randn((1000, cols), generator=g, device=DEV).to(dtype)
    for at in range(0, rows, 1000):
        x[at:at + 1000] = part[:min(1000, rows - at)]
    x[-1000:] = torch.randn((1000, cols), generator=g, device=DEV).to(dtype)
    return x


def test_policy_loss():
    T, V, n = 15000, 152064, 300                          # 2.3e9 logits; 300 rows take the same kernels
    z = _rand(T, V, BF)
    g = torch.Generator(device=DEV).manual_seed(1)
    y = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    old, adv = torch.full((T,), -12.0, device=DEV), torch.randn(T, generator=g, device=DEV)
    w = torch.full((T,), 1.0 / T, device=DEV)
    w[-7] = 0.0
    last = lambda t: t[-n:].contiguous()
    few = [last(t) for t in (z, y, old, adv, w)]
    want = reqat.policy_loss_grad(*few[:4], weights=few[4])
    alone = reqat.policy_loss(z, y, old, adv, weights=w)[1]
    alone_few = reqat.policy_loss(*few[:4], weights=few[4])[1]
    assert torch.equal(alone[-n:], alone_few)
    back = reqat.policy_loss_backward(z, y, alone)
    assert torch.equal(back[-n:], reqat.policy_loss_backward(few[0], few[1], alone_few))
    del back
    stats, grad = reqat.policy_loss_grad(z, y, old, adv, weights=w, out=z)[1:]
    assert torch.equal(stats[-n:], want[1]) and torch.equal(grad[-n:], want[2])


@pytest.mark.parametrize("K", [96, 3584, 27648])
def test_layer_norm(K):
    M, n = (1 << 31) // K + 5000, 2000
    x, dy = _rand(M, K, BF), _rand(M, K, BF)
    w, b = torch.rand(K, device=DEV) + 0.5, torch.rand(K, device=DEV)
    y, stats = reqat.layer_norm(x, w, b)
    ey, es = reqat.layer_norm(x[-n:], w, b)
    assert torch.equal(y[-n:], ey) and torch.equal(stats[-n:], es)
    dx, dw, db = reqat.layer_norm_backward(dy, x, w, stats, bias=True, out=y)
    assert torch.equal(dx[-n:], reqat.layer_norm_backward(dy[-n:], x[-n:], w, es)[0])
    # the weights' gradients: all rows' products in 64 bits, in parts
    want_w, want_b, size = (torch.zeros(K, dtype=torch.float64, device=DEV) for _ in range(3))
    for at in range(0, M, 1 << 18):
        part = slice(at, min(M, at + (1 << 18)))
        h, d = (x[part].float() - stats[part, :1]) * stats[part, 1:], dy[part].float()
        want_w += (d * h).sum(0, dtype=torch.float64)
        want_b += d.sum(0, dtype=torch.float64)
        size += (d * h).abs().sum(0, dtype=torch.float64) + d.abs().sum(0, dtype=torch.float64)
    # up to M / 64 additions in a row, whose errors have random signs: eight standard deviations of them
    room = size * 2.0 ** -24 * 8 * (M / 64 + 100) ** 0.5
    assert torch.all((dw.double() - want_w).abs() <= room) and torch.all((db.double() - want_b).abs() <= room)


def test_embedding():
    V, D, T = 450000, 5120, 3000                          # 2.3e9 elements
    table = _rand(V, D, BF)
    g = torch.Generator(device=DEV).manual_seed(2)
    ids = torch.randint(V - 900, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    ids[::10] = torch.arange(T // 10, device=DEV, dtype=torch.int32)
    assert torch.equal(reqat.embedding(ids, table), table[ids.long()])
    dy = _rand(T, D, BF)
    rows = torch.where(ids < 1000, ids, ids - (V - 2000))  # the same order of ids in a table of 2000
    for few in (400, T):
        want = reqat.embedding_backward(dy[:few], rows[:few], 2000)
        got = reqat.embedding_backward(dy[:few], ids[:few], V)
        assert torch.equal(got[-1000:], want[-1000:]) and torch.equal(got[:1000], want[:1000])
        assert not got[1000:-1000].any()
        base = table[-1000:].clone()
        reqat.embedding_backward(dy[:few], ids[:few], V, out=table, accumulate=True)
        touched = (want[-1000:] != 0).any(1)
        assert torch.equal(table[-1000:][~touched], base[~touched])
        assert torch.all((table[-1000:].float() - (base.float() + want[-1000:].float())).abs() <= 2.0 ** -7 * (base.float().abs() + want[-1000:].float().abs()))


def test_embedding_of_many_tokens():
    T, V, D = 262144, 4000, 8200                          # 2.1e9 elements of dy and of the output
    g = torch.Generator(device=DEV).manual_seed(3)
    ids = torch.randint(0, V - 100, (T,), generator=g, device=DEV, dtype=torch.int32)
    ids[-2000:] = torch.randint(V - 100, V, (2000,), generator=g, device=DEV, dtype=torch.int32)
    table = _rand(V, D, BF)
    out = reqat.embedding(ids, table)
    assert torch.equal(out[-2000:], table[ids[-2000:].long()])
    whole = torch.arange(D, device=DEV) % 5
    dy = out
    dy[:] = (whole - 2).to(BF)
    dy[-2000:] = (torch.arange(2000, device=DEV)[:, None] % 7 - 3 + whole).to(BF)
    want = torch.zeros((100, D), dtype=torch.float64, device=DEV)
    want.index_add_(0, ids[-2000:].long() - (V - 100), dy[-2000:].double())
    got = reqat.embedding_backward(dy, ids, V, out_dtype=F32)      # whole numbers: exact in any order
    assert torch.equal(got[-100:].double(), want)
    counts = torch.bincount(ids[:-2000].long(), minlength=V)[:V - 100, None]
    assert torch.equal(got[:V - 100], (counts * (whole - 2)).float())


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw(bits):
    n, last = (1 << 31) + 12800 + 77, 12800 + 77          # the last part begins with a block of 128
    p, g = torch.zeros(n, dtype=BF, device=DEV), torch.zeros(n, dtype=BF, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(4)
    p[-last:], g[-last:] = (torch.randn(last, generator=gen, device=DEV).to(BF) for _ in range(2))
    q = p[-last:].clone()
    opt, few = reqat.AdamW([p], 1e-2, state_bits=bits), reqat.AdamW([q], 1e-2, state_bits=bits)
    for _ in range(2):
        opt.step([g])
        few.step([g[-last:]])
    assert torch.equal(p[-last:], q) and not p[:-last].any()
    at = n - last
    assert torch.equal(opt.m[at:], few.m) and torch.equal(opt.v[at:], few.v)
    assert all(torch.equal(a[at:], b) for a, b in zip(opt.moments(), few.moments()))
