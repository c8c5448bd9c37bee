"""GPU: embedding lookup and its gradient by sorted tokens, against their formulas in 64 bits."""
import pytest
import torch

from paper_2606_15682_amd import reqat
from tests import train_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _ids(T, V, kind, seed=0):
    g = torch.Generator().manual_seed(31 * T + V + seed)
    if kind == "same":
        ids = torch.full((T,), V // 2, dtype=torch.int32)
    elif kind == "falling":
        ids = ((T - 1 - torch.arange(T)) % V).to(torch.int32)
    elif kind == "words":
        ids = (torch.exp(torch.rand(T, generator=g, dtype=torch.float64) * torch.log(torch.tensor(V + 1.0))) - 1).int().clamp(0, V - 1)
    else:
        ids = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    if T > 4:                                              # padding, in the forms that a caller may use
        ids[torch.randint(0, T, (max(1, T // 20),), generator=g)] = -1
        ids[1], ids[3] = V, -2 ** 31
    return ids.to(DEV)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V,D", [(1, 1, 1), (5, 3, 7), (9, 100, 64), (333, 1000, 129), (64, 5000, 3584), (7, 11, 1027)])
def test_lookup(T, V, D, dtype):
    g = torch.Generator().manual_seed(V)
    table = torch.randn((V, D), generator=g).to(dtype).to(DEV)
    ids = _ids(T, V, "any")
    known = (ids >= 0) & (ids < V)
    rows = table[torch.where(known, ids, 0).long()]
    assert torch.equal(reqat.embedding(ids, table), torch.where(known[:, None], rows, 0))
    scaled = reqat.embedding(ids, table, scale=1.7)
    want = torch.where(known[:, None], rows.float() * torch.tensor(1.7, device=DEV), 0).to(dtype)
    assert torch.equal(scaled, want)                       # one product of FP32 numbers, rounded once
    wide = torch.full((T, D + 3), 9.0, dtype=dtype, device=DEV)
    out = reqat.embedding(ids, torch.nn.functional.pad(table, (0, 5))[:, :D], out=wide[:, 1:D + 1])
    assert torch.equal(out, torch.where(known[:, None], rows, 0))
    assert torch.all(wide[:, 0] == 9.0) and torch.all(wide[:, D + 1:] == 9.0)


CASES = [(1, 1, 1, "any"), (3, 2, 5, "any"), (63, 10, 64, "same"), (64, 10, 64, "same"), (65, 10, 33, "same"),
         (129, 3, 257, "same"), (1000, 7, 100, "any"), (1025, 961, 64, "falling"), (2049, 300, 72, "words"), (511, 40, 136, "words"), (512, 9, 100, "same"), (513, 40, 136, "words"),
         (4000, 152064, 40, "words"), (5000, 250000, 9, "any"), (700, 256, 1027, "words"), (66000, 1000, 8, "words")]


@pytest.mark.parametrize("dtype,gdtype", [(BF, BF), (BF, F32), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("T,V,D,kind", CASES)
def test_gradient(T, V, D, kind, dtype, gdtype):
    print("embedding gradient", T, V, D, kind, dtype, gdtype, flush=True)
    g = torch.Generator().manual_seed(T)
    ids = _ids(T, V, kind)
    dy = torch.randn((T, D), generator=g).to(dtype).to(DEV)
    want, mag = ref.embedding_backward(dy, ids, V, 0.5)
    # 16 additions of a piece, and the pieces of the most frequent id; up to 512 tokens one after the other
    most = int(torch.bincount(ids[(ids >= 0) & (ids < V)].long()).max()) if ((ids >= 0) & (ids < V)).any() else 0
    room = mag * ref.EPS32 * ((most if T <= 512 else min(most, 16) + most // 16 + 1) + 3)
    fresh = reqat.embedding_backward(dy, ids, V, scale=0.5, out_dtype=gdtype)
    assert fresh.dtype == gdtype and fresh.shape == (V, D)
    assert torch.all((fresh.double().cpu() - want).abs() <= room + 1.01 * ref.half_step(gdtype) * want.abs())
    assert torch.equal(fresh, reqat.embedding_backward(dy, ids, V, scale=0.5, out_dtype=gdtype))
    base = torch.randn((V, D), generator=g).to(gdtype).to(DEV)
    out = base.clone()
    assert reqat.embedding_backward(dy, ids, V, scale=0.5, out=out, accumulate=True) is out
    total = base.double().cpu() + want
    room = room + ref.EPS32 * (base.double().cpu().abs() + want.abs())
    assert torch.all((out.double().cpu() - total).abs() <= room + 1.01 * ref.half_step(gdtype) * total.abs())
    untouched = torch.ones(V, dtype=torch.bool)
    untouched[ids[(ids >= 0) & (ids < V)].long().cpu()] = False
    assert torch.equal(out.cpu()[untouched], base.cpu()[untouched])


def test_exact_sums_and_order():
    """Whole numbers: every sum is exact, so that a token lost, doubled or in the wrong row shows."""
    T, V, D = 30011, 5000, 24
    for kind in ("any", "words", "falling", "same"):
        ids = _ids(T, V, kind)
        dy = ((torch.arange(T, device=DEV)[:, None] * 7 + torch.arange(D, device=DEV)) % 61 - 30).float()
        want, _ = ref.embedding_backward(dy, ids, V)
        assert torch.equal(reqat.embedding_backward(dy, ids, V).double().cpu(), want)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strides(dtype):
    T, V, D = 300, 40, 77
    ids = _ids(T, V, "words")
    dy = torch.randn((T, D + 3), generator=torch.Generator().manual_seed(1)).to(dtype).to(DEV)
    want = reqat.embedding_backward(dy[:, 2:2 + D].contiguous(), ids, V)
    table = torch.full((V, D + 2), 4.0, dtype=dtype, device=DEV)
    got = reqat.embedding_backward(dy[:, 2:2 + D], ids, V, out=table[:, 1:D + 1])
    assert torch.equal(got, want)
    assert torch.all(table[:, 0] == 4.0) and torch.all(table[:, D + 1] == 4.0)


def test_nan_stays_in_its_row():
    T, V, D = 200, 50, 16
    ids = _ids(T, V, "any")
    dy = torch.ones((T, D), device=DEV)
    ids[10], ids[11] = 7, -1
    dy[10, 3] = float("nan")
    dy[11] = float("nan")                                  # padding
    out = reqat.embedding_backward(dy, ids, V)
    bad = torch.isnan(out)
    assert bad[7, 3] and int(bad.sum()) == 1


def test_nothing_to_do():
    table = torch.ones((5, 8), device=DEV)
    ids = torch.empty(0, dtype=torch.int32, device=DEV)
    dy = torch.empty((0, 8), device=DEV)
    assert reqat.embedding(ids, table).shape == (0, 8)
    assert not reqat.embedding_backward(dy, ids, 5).any()
    kept = table.clone()
    assert torch.equal(reqat.embedding_backward(dy, ids, 5, out=table, accumulate=True), kept)
    ids = torch.full((70,), -1, dtype=torch.int32, device=DEV)
    dy = torch.ones((70, 8), device=DEV)
    assert not reqat.embedding(ids, table).any()
    assert not reqat.embedding_backward(dy, ids, 5).any()
    assert torch.equal(reqat.embedding_backward(dy, ids, 5, out=table, accumulate=True), kept)


def test_autograd():
    table = torch.randn((30, 12), generator=torch.Generator().manual_seed(3)).to(DEV).requires_grad_()
    ids = _ids(50, 30, "any")
    c = torch.randn((50, 12), generator=torch.Generator().manual_seed(4)).to(DEV)
    (reqat.Embedding.apply(ids, table, 3.0) * c).sum().backward()
    want, mag = ref.embedding_backward(c, ids, 30, 3.0)
    assert torch.all((table.grad.double().cpu() - want).abs() <= mag * 60 * ref.EPS32)
    table.grad = None
    reqat.Embedding.apply(ids, table).sum().backward()     # an expanded gradient
    assert torch.equal(table.grad[:, 0], table.grad[:, 11])
