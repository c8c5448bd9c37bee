"""The attention half of one W4A4KV4 decoder layer, as a serving loop runs it:

    python examples/kv4_serving.py [--model 14b] [--seqs 4] [--prompt 700] [--steps 32]

Each sequence's prompt goes through in pieces and then a step per token: the QKV product on 4-bit weights and
activations, one pass that rotates queries and keys, takes the shift off the keys and writes keys and values into the
pages of the 4-bit cache, and attention over the pages.  The decode step is captured in one HIP graph and replayed;
what differs from step to step (tokens, positions, slots, lengths) is written into its buffers on the device.

Random weights and inputs; the last step is checked against FP32 attention over the cache read back.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2606_15682_amd import reqat  # noqa: E402

HEAD, PAGE, PIECE = 128, 64, 256
# hidden width, query heads, key/value heads
MODELS = {"1.5b": (1536, 12, 2), "7b": (3584, 28, 4), "14b": (5120, 40, 8)}


class Layer:
    """QKV weights, rotary tables and the cache of one layer, for `seqs` sequences of up to `longest` tokens."""

    def __init__(self, model, seqs, longest, dev, seed=0):
        self.hidden, self.hq, self.hkv = MODELS[model]
        self.seqs, self.dev = seqs, dev
        gen = torch.Generator(device=dev).manual_seed(seed)
        rows = (self.hq + 2 * self.hkv) * HEAD
        w = (torch.randn((rows, self.hidden), generator=gen, device=dev) * 0.02).to(torch.bfloat16)
        self.w_codes, self.w_scales, self.w_g = reqat.quantize(w, reqat.NVFP4)
        self.packed, self.rows = reqat.pack_w4a4(self.w_codes, self.w_scales, reqat.NVFP4), rows
        angle = torch.arange(longest, device=dev, dtype=torch.float64)[:, None] * \
            1e6 ** (-torch.arange(0, HEAD, 2, device=dev, dtype=torch.float64) / HEAD)
        self.rope = (angle.cos().float(), angle.sin().float())
        pages = -(-longest // PAGE)
        self.table = torch.randperm(seqs * pages, generator=gen, device=dev).to(torch.int32).view(seqs, pages)
        shift = torch.randn(self.hkv * HEAD, generator=gen, device=dev) * 0.1        # as a calibration would give it
        self.cache = reqat.Kv4Cache(seqs * pages, PAGE, self.hkv, HEAD, k_scale=2.0 ** -6, v_scale=2.0 ** -6,
                                    k_shift=shift, device=dev)

    def slots(self, seq, pos):
        """Cache slots of tokens `pos` of sequences `seq` (index tensors of one shape)."""
        return self.table[seq, pos // PAGE].long() * PAGE + pos % PAGE

    def split(self, qkv):
        q, kv = self.hq * HEAD, self.hkv * HEAD
        return qkv[:, :q], qkv[:, q:q + kv], qkv[:, q + kv:]

    def prompt(self, xs):
        """The prompts xs (bfloat16 [tokens, hidden] of each sequence) in pieces; returns their attention outputs."""
        outs = [[] for _ in xs]
        for at in range(0, max(len(x) for x in xs), PIECE):
            new = [x[at:at + PIECE] for x in xs]
            counts = [len(x) for x in new]
            qkv, _ = reqat.linear(torch.cat(new), reqat.NVFP4, self.w_codes, self.w_scales, self.w_g)
            q, k, v = self.split(qkv)
            seq = torch.repeat_interleave(torch.arange(self.seqs), torch.tensor(counts)).to(self.dev)
            pos = torch.cat([torch.arange(at, at + n) for n in counts]).to(self.dev)
            q = reqat.kv4_append(self.cache, k, v, self.slots(seq, pos), q=q, rope=self.rope, positions=pos.int())
            start = torch.tensor([0] + counts).cumsum(0).int().to(self.dev)
            lens = torch.tensor([min(len(x), at + PIECE) for x in xs], dtype=torch.int32).to(self.dev)
            out = reqat.kv4_attention(q, self.cache, self.table, lens, q_start=start, max_q=max(counts), max_kv=at + PIECE)
            for s, o in enumerate(out.split(counts)):
                outs[s].append(o)
        return [torch.cat(o) for o in outs]

    def capture(self, longest):
        """The decode step as a graph over buffers: x, lens (tokens cached before the step) -> out, q."""
        dev, B = self.dev, self.seqs
        self.x = torch.zeros((B, self.hidden), dtype=torch.bfloat16, device=dev)
        self.lens = torch.zeros(B, dtype=torch.int32, device=dev)
        self.everyone = torch.arange(B, device=dev)
        qkv = torch.empty((B, self.rows), dtype=torch.bfloat16, device=dev)
        need = reqat.reqat_kv4_attention_workspace_bytes(B, B, 1, longest, self.hq, self.hkv, HEAD)
        ws = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)

        def step():
            reqat.linear_packed(self.x, reqat.NVFP4, self.packed, self.rows, self.w_g, out=qkv)
            q, k, v = self.split(qkv)
            reqat.kv4_append(self.cache, k, v, self.slots(self.everyone, self.lens.long()), q=q, q_out=q, rope=self.rope,
                             positions=self.lens)
            self.lens += 1
            self.q, self.out = q, reqat.kv4_attention(q, self.cache, self.table, self.lens, max_kv=longest, ws=ws)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):                       # once outside the graph; the prompts overwrite what it cached
            step()
        torch.cuda.current_stream().wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            step()

    def reference(self):
        """FP32 attention of the last step's queries over the cache read back."""
        outs = []
        for s, n in enumerate(self.lens.tolist()):
            pos = torch.arange(n, device=self.dev)
            k, v = (t.float().view(n, self.hkv, HEAD) for t in reqat.kv4_gather(self.cache, self.slots(s, pos)))
            q = self.q[s].float().view(self.hkv, -1, HEAD)
            score = torch.einsum("hgd,nhd->hgn", q, k) * HEAD ** -0.5
            outs.append(torch.einsum("hgn,nhd->hgd", score.softmax(-1), v).flatten())
        return torch.stack(outs)


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--model", choices=sorted(MODELS), default="14b")
    ap.add_argument("--seqs", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=700)
    ap.add_argument("--steps", type=int, default=32)
    a = ap.parse_args(argv)
    dev = torch.device("cuda:0")
    longest = a.prompt + a.steps + 1
    layer = Layer(a.model, a.seqs, longest, dev)
    layer.capture(longest)
    gen = torch.Generator(device=dev).manual_seed(1)
    lens = [max(1, a.prompt - 37 * s) for s in range(a.seqs)]
    layer.prompt([torch.randn((n, layer.hidden), generator=gen, device=dev).to(torch.bfloat16) for n in lens])
    layer.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(a.steps):
        layer.x.normal_(generator=gen)
        layer.graph.replay()
    end.record()
    torch.cuda.synchronize()
    want = layer.reference()
    err = float((layer.out.float() - want).norm() / want.norm())
    print("%d sequences, %s tokens after %d steps of %.1f us; the last step is %.1e off FP32 attention over the same cache"
          % (a.seqs, layer.lens.tolist(), a.steps, begin.elapsed_time(end) * 1e3 / max(a.steps, 1), err))
    return err


if __name__ == "__main__":
    sys.exit(0 if main() < 5e-3 else 1)
