"""GPU: one workspace, sized for the largest call, in calls of every smaller size: the results of a workspace of their
own, and nothing written behind it."""
import pytest
import torch

from paper_2606_15682_amd import reqat
from tests.test_gpu_kv4_attention import Setup

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("D", [64, 128])
def test_one_workspace_for_all_calls(D):
    H, group, most_q, most_kv, most_b = 2, 5, 70, 3000, 5
    need = reqat.reqat_kv4_attention_workspace_bytes(most_b, most_b * most_q, most_q, most_kv, H * group, H, D)
    room = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
    for lens, nqs in (([3000], [1]), ([2999, 300, 0, 1, 2500], [1] * 5), ([2100, 3000], [6, 2]), ([700], [1]),
                      ([600, 3000, 5], [70, 9, 3]), ([3000], [70]), ([1025], [33])):
        print("workspace: lens=%s q=%s D=%d" % (lens, nqs, D), flush=True)
        s = Setup(lens, H, D, 16, seed=41)
        q = s.queries(nqs, group, 2.0)
        want = s.run(q, nqs)
        got = s.run(q, nqs, ws=room[:need])
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert bool((room[need:] == 0x5A).all())
        s.check(got, q, nqs)


def test_more_rows_than_the_sequences_have():
    """Rows before, between and behind the sequences (q_start names few of many): partial rows go by sequence."""
    s = Setup([2500, 900], 1, 128, 16, seed=42)
    q = s.queries([1] * 40, 4, 2.0).to(DEV)
    starts = torch.tensor([11, 13, 14], dtype=torch.int32, device=DEV)
    out = torch.full_like(q, 3.0)
    reqat.kv4_attention(q, s.cache, s.dtable, torch.tensor(s.lens, dtype=torch.int32, device=DEV), q_start=starts, max_q=2,
                        max_kv=2500, out=out)
    got = s.run(q[11:14].contiguous(), [2, 1], max_q=2)
    assert torch.equal(out[11:14], got[0])
    s.check(got, q[11:14], [2, 1])
    assert bool((out[:11] == 3.0).all()) and bool((out[14:] == 3.0).all())
