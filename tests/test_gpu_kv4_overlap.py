"""GPU: inputs and outputs of the KV4 cache's calls side by side in the rows of one buffer."""
import pytest
import torch

from paper_2606_15682_amd import reqat
from tests.test_gpu_kv4_attention import Setup

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("nqs", [[1, 1, 1], [6, 2, 3], [70, 40, 1]])
def test_queries_and_outputs_in_one_buffer(nqs):
    s = Setup([100, 77, 300], 2, 128, 32, seed=6)
    q = s.queries(nqs, 5)
    want = s.run(q, nqs)
    n = q.shape[1]
    both = torch.full((len(q), 2 * n + 16), 5.0, dtype=torch.bfloat16, device=DEV)
    both[:, n + 8:2 * n + 8] = q.to(DEV)
    got = s.run(both[:, n + 8:2 * n + 8], nqs, out=both[:, :n])
    assert torch.equal(got[0], want[0]) and torch.equal(both[:, n + 8:2 * n + 8], q.to(DEV))
    assert bool((both[:, n:n + 8] == 5.0).all()) and bool((both[:, 2 * n + 8:] == 5.0).all())
    with pytest.raises(reqat.ReqatError):
        s.run(both[:, n + 8:2 * n + 8], nqs, out=both[:, 16:n + 16])
    if len(q) > 1:
        with pytest.raises(reqat.ReqatError):
            s.run(both[:, n + 8:2 * n + 8], nqs, out=both[:, n + 8:2 * n + 8])


def test_rotated_queries_beside_their_inputs():
    H, group, D, T = 2, 3, 64, 50
    Q, W = H * group * D, H * D
    gen = torch.Generator(device=DEV).manual_seed(3)
    wide = torch.randn((T, 2 * Q + 2 * W), generator=gen, device=DEV).to(torch.bfloat16)
    cos, sin = (f(torch.rand((64, D // 2), generator=gen, device=DEV) * 6.28) for f in (torch.cos, torch.sin))
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    slots = torch.arange(T, device=DEV)
    caches = [reqat.Kv4Cache(4, 16, H, D, k_scale=2.0 ** -6, v_scale=2.0 ** -6, device=DEV) for _ in range(2)]
    k, v, q = wide[:, Q:Q + W], wide[:, Q + W:Q + 2 * W], wide[:, :Q]
    want = reqat.kv4_append(caches[0], k, v, slots, q=q, rope=(cos, sin), positions=pos)
    before = wide.clone()
    reqat.kv4_append(caches[1], k, v, slots, q=q, rope=(cos, sin), positions=pos, q_out=wide[:, Q + 2 * W:])
    assert torch.equal(wide[:, Q + 2 * W:], want) and torch.equal(wide[:, :Q + 2 * W], before[:, :Q + 2 * W])
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        assert torch.equal(getattr(caches[0], name), getattr(caches[1], name))


def test_keys_and_values_read_back_side_by_side():
    s = Setup([100], 2, 128, 32, seed=7)
    slots = torch.from_numpy(s.table[0, :4].astype("int64") * 32).to(DEV).repeat_interleave(25) + torch.arange(100, device=DEV) % 25
    k, v = reqat.kv4_gather(s.cache, slots)
    both = torch.empty((100, 512), dtype=torch.bfloat16, device=DEV)
    reqat.kv4_gather(s.cache, slots, out=(both[:, 256:], both[:, :256]))
    bits = both.view(torch.int16)                       # slots without a token hold NaN
    assert torch.equal(bits[:, 256:], k.view(torch.int16)) and torch.equal(bits[:, :256], v.view(torch.int16))
