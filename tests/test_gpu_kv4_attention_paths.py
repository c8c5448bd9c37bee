"""Attention over the KV4 cache where its paths meet: NaN tokens, non-finite queries, lost pages and lengths in calls of one
piece (four and eight waves) and of several that are joined, few queries and prompts, both head sizes; prompts of more
sequences than are sorted by length."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv4_attention import Setup, go

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# lens, queries, KV heads, group: decode in pieces, by eight waves, in one piece; few queries in pieces; prompts in pieces
CALLS = [([2500, 70], [1, 1], 2, 5), ([400], [1], 2, 5), ([200, 70], [1, 1], 1, 7), ([2500, 70], [6, 3], 2, 5),
         ([1500, 180], [65, 40], 2, 3), ([180, 60], [65, 40], 1, 4)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,nqs,H,group", CALLS)
@pytest.mark.parametrize("which", ["k", "v"])
def test_nan_tokens(which, lens, nqs, H, group, D):
    """In the middle, in the last piece, and at the end, where only the last queries see them; every block of channels."""
    n = lens[0]
    for at in ([n // 2], [n - 1], [n - 3, n - 1, 5], [max(0, n - nqs[0] - 1)]):
        s = Setup(lens, H, D, 16, seed=51)
        q = s.queries(nqs, group)
        for i, j in enumerate(at):
            s.spoil(0, j, (i + 1) % H, (3 * i + j) % (D // 16), which)
        s.upload()
        print("NaN %s at %s: lens=%s q=%s D=%d" % (which, at, lens, nqs, D), flush=True)
        got = s.run(q, nqs)
        s.check(got, q, nqs)
        assert bool(torch.isnan(got[0]).any())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,nqs,H,group", CALLS)
def test_every_block_of_channels(lens, nqs, H, group, D):
    """A NaN value is in its 16 channels and nowhere else."""
    for block in range(D // 16):
        s = Setup(lens, H, D, 16, seed=52)
        q = s.queries(nqs, group)
        s.spoil(0, lens[0] - 1, H - 1, block, "v")
        s.upload()
        print("NaN block %d: lens=%s q=%s D=%d" % (block, lens, nqs, D), flush=True)
        got = s.run(q, nqs)
        s.check(got, q, nqs)
        bad = torch.isnan(got[0]).view(-1, H, group, D // 16, 16)
        want = torch.zeros_like(bad)
        want[nqs[0] - 1, H - 1, :, block] = True             # the last query of the first sequence alone sees the token
        assert torch.equal(bad, want)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,nqs,H,group", CALLS)
def test_nonfinite_queries(lens, nqs, H, group, D):
    s = Setup(lens, H, D, 16, seed=53)
    q = s.queries(nqs, group)
    x = q.view(len(q), -1, D)
    x[0, 0, 3], x[-1, 1, D - 1], x[len(x) // 2, 2, 7] = float("nan"), float("inf"), float("-inf")
    print("non-finite queries: lens=%s q=%s D=%d" % (lens, nqs, D), flush=True)
    out, lse = s.run(q, nqs)
    lost = ~torch.isfinite(q.float()).view(x.shape).all(-1).to(DEV)
    clean = torch.where(torch.isfinite(q), q, torch.zeros_like(q))
    want, want_lse = s.run(clean, nqs)
    assert bool(torch.isnan(out.view(x.shape)[lost]).all()) and bool(torch.isnan(lse[lost]).all())
    assert torch.equal(out.view(x.shape)[~lost], want.view(x.shape)[~lost]) and torch.equal(lse[~lost], want_lse[~lost])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,nqs,H,group", CALLS)
def test_lost_pages(lens, nqs, H, group, D):
    """A page entry outside the cache: NaN for the rows that see its tokens, the others bit for bit as before."""
    s = Setup(lens, H, D, 16, seed=54)
    q = s.queries(nqs, group)
    want = s.run(q, nqs)
    n, first = lens[0], torch.arange(sum(nqs), device=DEV) < nqs[0]
    for page in (0, (n // 2) // 16, (n - 1) // 16):
        for entry in (-1, s.pages, 2 ** 31 - 1):
            print("lost page %d: lens=%s q=%s D=%d" % (page, lens, nqs, D), flush=True)
            s.dtable[0, page] = entry
            out, lse = s.run(q, nqs)
            sees = first & (n - nqs[0] + torch.arange(sum(nqs), device=DEV) >= page * 16)
            assert bool(torch.isnan(out[sees]).all()) and bool(torch.isnan(lse[sees]).all())
            assert torch.equal(out[~sees], want[0][~sees]) and torch.equal(lse[~sees], want[1][~sees])
        s.dtable[0, page] = int(s.table[0, page])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,nqs,H,group", CALLS)
def test_lost_lengths(lens, nqs, H, group, D):
    """A length beyond max_kv, or beyond the table: NaN in all rows of the sequence, the others as they are."""
    s = Setup(lens, H, D, 16, seed=55)
    q = s.queries(nqs, group)
    first = torch.arange(sum(nqs), device=DEV) < nqs[0]
    print("lost lengths: lens=%s q=%s D=%d" % (lens, nqs, D), flush=True)

    def others(got):
        out, lse = got
        assert bool(torch.isnan(out[first]).all()) and bool(torch.isnan(lse[first]).all())
        if len(nqs) > 1:
            s.check((out[~first], lse[~first]), q[nqs[0]:], [0] + nqs[1:])

    others(s.run(q, nqs, max_kv=lens[0] - 1))
    s.dtable = s.dtable[:, :(lens[0] - 1) // 16].contiguous()
    others(s.run(q, nqs))


@pytest.mark.parametrize("count", [63, 64, 65, 100])
@pytest.mark.parametrize("causal", [True, False])
def test_prompts_of_many_sequences(count, causal):
    """The longest of up to 64 sequences go first, more go as they come; equal lengths and empty ones among them."""
    lens = [(37 * b) % 90 if b % 5 else 40 for b in range(count)]
    nqs = [1 + (13 * b) % 40 for b in range(count)]
    nqs[3] = 40
    go(lens, nqs, 1, 3, 64, 16, causal, seed=56)
    go(lens, nqs, 1, 3, 128, 32, causal, seed=57)
