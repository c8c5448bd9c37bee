"""Timing cases of the 4-bit KV cache: writing keys and values into it, reading
them back, and attention over it, through the calls of
``paper_2606_15682_amd.reqat``.

The head layouts are those of the Qwen-family reasoning models that the
library's benchmark names (heads of 128 channels) and of their tensor-parallel
shards.  Keys are a unit Gaussian around per-channel means, which the shift
removes; values are Gaussian; queries give scores with a standard deviation of
two.  The tensor scales are calibrated powers of two.

Each case has a ``kind``:
  ``append``     T new tokens, q, k and v as column slices of the fused QKV
                 output: q and k rotated to their positions, k shifted, k and v
                 quantized into the pages of the cache.  The slots just written
                 are read back, so that the pass returns what the cache holds.
  ``gather``     the cached keys and values of T tokens read back as bfloat16,
                 the shift of the keys added again.
  ``attn``       attention of the new queries of every sequence over its cached
                 tokens: one query each (decode), a few (drafts that are
                 checked), or a prompt or a piece of one, causal.

``run`` is the calls alone; the cache, its page table and the lengths are what a
serving loop holds.  Where ``own`` is false everything is elementary torch
operations in 32 bits, on a cache of plain codes and scale bytes.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
HEAD = 128

# query heads, key/value heads
MODELS = {"1.5b": (12, 2), "7b": (28, 4), "14b": (40, 8), "32b": (40, 8)}
G_K, G_V = 2.0 ** -6, 2.0 ** -6      # calibrated tensor scales: a block of 16 may reach 24.5
SM_SCALE = HEAD ** -0.5
ROPE_BASE = 1.0e6
ROPE_LEN = 32768


def listed():
    return [
        # one user, a short conversation, smallest model: launches and latency count
        {"name": "decode_1.5b_b1_c1021", "kind": "attn", "model": "1.5b", "tp": 1, "B": 1, "q": 1, "ctx": 1021,
         "page": 16, "lse": False},
        # an ordinary decode step of the main model, sequences of all lengths
        {"name": "decode_14b_b16_c8192", "kind": "attn", "model": "14b", "tp": 1, "B": 16, "q": 1, "ctx": 8192,
         "page": 64, "lse": False},
        # one of four tensor-parallel ranks: one KV head, seven query heads, long reasoning traces
        {"name": "decode_7b_tp4_b8_c32768", "kind": "attn", "model": "7b", "tp": 4, "B": 8, "q": 1, "ctx": 32768,
         "page": 32, "lse": True},
        # a full decode batch: the cache is most of what a step reads
        {"name": "decode_14b_b64_c16384", "kind": "attn", "model": "14b", "tp": 1, "B": 64, "q": 1, "ctx": 16384,
         "page": 128, "lse": False},
        # one very long sequence: the work has to be split over its length
        {"name": "decode_32b_b1_c131072", "kind": "attn", "model": "32b", "tp": 1, "B": 1, "q": 1, "ctx": 131072,
         "page": 64, "lse": False},
        # up to five draft tokens of each sequence checked in one step
        {"name": "verify_14b_b16_q5_c4001", "kind": "attn", "model": "14b", "tp": 1, "B": 16, "q": 5, "ctx": 4001,
         "page": 16, "lse": False},
        # pieces of several users' prompts in one batch
        {"name": "chunk_7b_b5_q777_c9001", "kind": "attn", "model": "7b", "tp": 1, "B": 5, "q": 777, "ctx": 9001,
         "page": 64, "lse": False},
        # a whole long prompt of the main model
        {"name": "prompt_14b_b1_q8192_c8192", "kind": "attn", "model": "14b", "tp": 1, "B": 1, "q": 8192, "ctx": 8192,
         "page": 64, "lse": False},
        # the new token of each sequence of a decode batch
        {"name": "append_14b_b64_t64", "kind": "append", "model": "14b", "tp": 1, "B": 64, "T": 64, "ctx": 8192,
         "page": 64},
        # the tokens of a few prompts, ragged
        {"name": "append_7b_b3_t5003", "kind": "append", "model": "7b", "tp": 1, "B": 3, "T": 5003, "ctx": 8192,
         "page": 32},
        # a short shared prefix read back
        {"name": "gather_1.5b_t601", "kind": "gather", "model": "1.5b", "tp": 1, "T": 601, "page": 16},
        # a whole long context read back
        {"name": "gather_14b_t32768", "kind": "gather", "model": "14b", "tp": 1, "T": 32768, "page": 64},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    """Seconds a pass needs at rates near this card's."""
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 5e14


def _most_cost():
    return max(_cost(c) for c in listed())


def draw(rng):
    most = _most_cost()
    while True:
        kind = rng.choice(["decode", "decode", "decode", "verify", "chunk", "prompt", "append", "gather"])
        model = rng.choice(sorted(MODELS))
        tp = rng.choice([1, 2, 4])
        if model == "1.5b":                    # two KV heads: at most two ranks
            tp = min(tp, 2)
        case = {"kind": "attn", "model": model, "tp": tp, "page": rng.choice([16, 32, 64, 128])}
        if kind == "decode":
            case.update(B=_log_uniform(rng, 1, 128), q=1, ctx=_log_uniform(rng, 16, 131072), lse=rng.random() < 0.25)
        elif kind == "verify":
            case.update(B=_log_uniform(rng, 1, 64), q=rng.randint(2, 16), ctx=_log_uniform(rng, 64, 16384),
                        lse=rng.random() < 0.25)
        elif kind == "chunk":
            case.update(B=_log_uniform(rng, 1, 8), q=_log_uniform(rng, 17, 2048), ctx=_log_uniform(rng, 2048, 16384),
                        lse=rng.random() < 0.25)
        elif kind == "prompt":
            n = _log_uniform(rng, 16, 8192)
            case.update(B=_log_uniform(rng, 1, 4), q=n, ctx=n, lse=rng.random() < 0.25)
        elif kind == "append":
            B = _log_uniform(rng, 1, 64)
            case.update(kind="append", B=B, T=rng.choice([B, max(B, _log_uniform(rng, 16, 16384))]), ctx=16384)
        else:
            case.update(kind="gather", T=_log_uniform(rng, 16, 65536))
        if _cost(case) <= most and _tokens(case) <= 2 * 64 * 16384:
            return case


# ------------------------------------------------------------------ shapes

def _heads(case):
    hq, hkv = MODELS[case["model"]]
    return hq // case["tp"], hkv // case["tp"]


def _rng(case):
    return random.Random("%s" % sorted((k, v) for k, v in case.items() if k != "name"))


def _lengths(case):
    """Per sequence, the number of new tokens and of tokens in all (new ones included).

    attn: the first sequence has the case's sizes, the others are shorter; from
    eight decoding sequences on, one batch slot holds no sequence (a query, no
    tokens), as in a captured graph of a fixed batch."""
    r = _rng(case)
    if case["kind"] == "gather":
        return [(case["T"], case["T"])]
    if case["kind"] == "append":
        B, T = case["B"], case["T"]
        cuts = sorted(r.sample(range(1, T), B - 1)) if T > B else list(range(1, B))
        new = [b - a for a, b in zip([0] + cuts, cuts + [T])]
        return [(n, max(n, r.randint(n, max(n, case["ctx"])) if T == B else n)) for n in new]
    out = []
    for b in range(case["B"]):
        if b == 0:
            out.append((case["q"], case["ctx"]))
            continue
        if case["q"] == 1 and case["B"] >= 8 and b == case["B"] // 2:
            out.append((1, 0))
            continue
        q = case["q"] if case["q"] == 1 else r.randint(max(1, case["q"] // 2), case["q"])
        ctx = q if case["ctx"] == case["q"] else max(q, int(case["ctx"] * r.uniform(0.25, 1.0)))
        out.append((q, ctx))
    return out


def _tokens(case):
    return sum(n for _, n in _lengths(case))


def work(case):
    """Bytes and operations of one pass: every input read once, every output written once."""
    hq, hkv = _heads(case)
    cached = 2 * hkv * (HEAD // 2 + HEAD // 16)          # keys and values of one token, with their scales
    if case["kind"] == "gather":
        return {"bytes": case["T"] * (cached + 2 * hkv * HEAD * 2 + 8), "flops": case["T"] * 2 * hkv * HEAD}
    if case["kind"] == "append":
        t = case["T"]
        moved = (hq + 2 * hkv) * HEAD * 2 + hq * HEAD * 2 + 2 * cached + 2 * hkv * HEAD * 2 + HEAD * 4
        return {"bytes": t * moved, "flops": t * (6 * (hq + hkv) * HEAD + 4 * hkv * HEAD)}
    lens = _lengths(case)
    pairs = sum(sum(max(0, n - q + i + 1) for i in range(q)) for q, n in lens)
    tokens, rows = sum(n for _, n in lens), sum(q for q, _ in lens)
    return {"bytes": tokens * cached + rows * hq * (4 * HEAD + (4 if case["lse"] else 0)),
            "flops": 4 * HEAD * hq * pairs}


# ------------------------------------------------------------------ inputs

def _generator(seed, stream):
    return torch.Generator(device=DEV).manual_seed(1000003 * (seed % (1 << 40)) + stream)


def _bf16(gen, rows, cols, std=1.0, mean=None):
    x = torch.randn((rows, cols), generator=gen, device=DEV)
    if std != 1.0:
        x *= std
    if mean is not None:
        x += mean
    return x.to(torch.bfloat16)


def _shift(case, seed):
    """The calibrated channel means of the keys."""
    return torch.randn(_heads(case)[1] * HEAD, generator=_generator(seed, 1), device=DEV) * 2.0


def _kv_of(case, seed, b, tokens, shift):
    """Keys and values of sequence b, as they are before they are cached."""
    gen = _generator(seed, 100 + b)
    width = _heads(case)[1] * HEAD
    return _bf16(gen, tokens, width, mean=shift), _bf16(gen, tokens, width)


def _block_table(case, seed):
    """Pages of the sequences, scattered over the cache: [B, pages of the longest], int32, and the number of pages."""
    page = case["page"]
    need = [-(-n // page) for _, n in _lengths(case)]
    total = sum(need)
    perm = torch.randperm(total, generator=_generator(seed, 2), device=DEV).to(torch.int32)
    table = torch.zeros((len(need), max(max(need), 1)), dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, total


def _slots(table, b, start, end, page):
    """Cache slots of the tokens start .. end of sequence b, int64."""
    pos = torch.arange(start, end, device=DEV)
    return table[b, pos // page].to(torch.int64) * page + pos % page


def _rope_tables():
    inv = ROPE_BASE ** (-torch.arange(0, HEAD, 2, dtype=torch.float64, device=DEV) / HEAD)
    ang = torch.arange(ROPE_LEN, dtype=torch.float64, device=DEV)[:, None] * inv[None, :]
    return torch.cos(ang).to(torch.float32), torch.sin(ang).to(torch.float32)


def _queries(case, seed):
    rows = sum(q for q, _ in _lengths(case))
    return _bf16(_generator(seed, 3), rows, _heads(case)[0] * HEAD, std=2.0)


def _new_tokens(case, seed):
    """The fused QKV output of an append case, the positions and the slots of its tokens.

    From sixteen decoding sequences on, the last batch slot is padding (slot -1)."""
    hq, hkv = _heads(case)
    shift = _shift(case, seed)
    gen = _generator(seed, 4)
    T = case["T"]
    # keys reach the cache rotated, so their means are given to them in pairs of channels here
    qkv = torch.cat([_bf16(gen, T, hq * HEAD, std=2.0), _bf16(gen, T, hkv * HEAD, mean=shift),
                     _bf16(gen, T, hkv * HEAD)], dim=1)
    table, pages = _block_table(case, seed)
    pos, slots = [], []
    for b, (new, n) in enumerate(_lengths(case)):
        pos.append(torch.arange(n - new, n, device=DEV, dtype=torch.int32))
        slots.append(_slots(table, b, n - new, n, case["page"]))
    slots = torch.cat(slots)
    if case["T"] == case["B"] and case["B"] >= 16:
        slots[-1] = -1
    return qkv, torch.cat(pos), slots, pages, shift


def _fill(case, seed, put):
    """Hands the keys and values of every sequence to put(k, v, slots), in pieces."""
    shift = _shift(case, seed)
    table, pages = _block_table(case, seed)
    for b, (_, n) in enumerate(_lengths(case)):
        if n:
            k, v = _kv_of(case, seed, b, n, shift)
            put(k, v, _slots(table, b, 0, n, case["page"]))


def prepare(case, seed):
    hq, hkv = _heads(case)
    state = {"case": case, "hq": hq, "hkv": hkv}
    if case["kind"] == "append":
        qkv, pos, slots, pages, shift = _new_tokens(case, seed)
        state.update(q=qkv[:, :hq * HEAD], k=qkv[:, hq * HEAD:(hq + hkv) * HEAD], v=qkv[:, (hq + hkv) * HEAD:],
                     pos=pos, slots=slots, rope=_rope_tables())
    else:
        table, pages = _block_table(case, seed)
        shift = _shift(case, seed)
        state.update(table=table)
    if own:
        from paper_2606_15682_amd import reqat
        cache = reqat.Kv4Cache(pages, case["page"], hkv, HEAD, k_scale=G_K, v_scale=G_V, k_shift=shift, device=DEV)
        state.update(reqat=reqat, cache=cache)
        if case["kind"] != "append":
            _fill(case, seed, lambda k, v, slots: reqat.kv4_append(cache, k, v, slots))
    else:
        size = pages * case["page"]
        cache = {"shift": shift}
        for name in ("k", "v"):
            cache[name] = (torch.zeros((size, hkv, HEAD // 2), dtype=torch.uint8, device=DEV),
                           torch.zeros((size, hkv, HEAD // 16), dtype=torch.uint8, device=DEV))
        state.update(cache=cache)
        if case["kind"] != "append":
            _fill(case, seed, lambda k, v, slots: _plain_put(cache, k.float(), v.float(), slots, hkv))
    if case["kind"] == "gather":
        state["slots"] = _slots(state["table"], 0, 0, case["T"], case["page"])
    if case["kind"] == "attn":
        lens = _lengths(case)
        state.update(q=_queries(case, seed), lens=lens, rows=sum(q for q, _ in lens),
                     kv_len=torch.tensor([n for _, n in lens], dtype=torch.int32, device=DEV),
                     max_q=max(q for q, _ in lens), max_kv=max(n for _, n in lens), q_start=None)
        if case["q"] > 1:
            starts = [0]
            for q, _ in lens:
                starts.append(starts[-1] + q)
            state["q_start"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
        if own:
            need = reqat.reqat_kv4_attention_workspace_bytes(len(lens), state["rows"], state["max_q"],
                                                             state["max_kv"], hq, hkv, HEAD)
            state["ws"] = torch.empty(max(need, 1), dtype=torch.uint8, device=DEV)
    return state


# ------------------------------------------------------------------ plain forms

def _e4m3_grid(device, dtype):
    """Values of the E4M3 bytes 0x00 .. 0x7E."""
    b = torch.arange(0x7F, device=device)
    e, m = b // 8, (b % 8).to(dtype)
    return torch.where(e == 0, m * 2.0 ** -9, (1.0 + m / 8.0) * torch.exp2((e - 7).to(dtype)))


def _plain_quantize(d, g):
    """E1M2 codes (two a byte) and E4M3 scale bytes of the blocks of 16 of d [..., D]; g a power of two, so that
    every bound and threshold below is exact in 32 bits."""
    grid = _e4m3_grid(d.device, torch.float32)
    blk = d.unflatten(-1, (-1, 16))
    amax = blk.abs().amax(-1)
    byte = torch.bucketize(amax, 3.5 * grid[1:] * g) + 1
    byte = torch.where(amax == 0, torch.zeros_like(byte), byte.clamp(max=0x7E))
    step = (grid[byte] * g)[..., None]
    a = blk.abs()
    code = torch.zeros_like(a)
    for i in range(7):                         # ties go to the even code
        bound = (0.5 * i + 0.25) * step
        code += ((a > bound) if i % 2 == 0 else (a >= bound)).to(torch.float32)
    code = torch.where(amax[..., None] == 0, torch.zeros_like(code), code)
    c = (code.to(torch.uint8) + 8 * torch.signbit(blk).to(torch.uint8)).flatten(-2)
    return c[..., 0::2] + 16 * c[..., 1::2], byte.to(torch.uint8)


def _plain_values(codes, scales, g):
    """The 32-bit values that codes and scale bytes stand for."""
    grid = _e4m3_grid(codes.device, torch.float32)
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)
    mag = 0.5 * (c & 7).to(torch.float32)
    val = torch.where((c & 8) != 0, -mag, mag).unflatten(-1, (-1, 16))
    return (val * (grid[scales.long()] * g)[..., None]).flatten(-2)


def _plain_rotate(x, cos, sin):
    half = HEAD // 2
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _plain_put(cache, k, v, slots, hkv):
    """Quantizes keys (rotated, 32 bits) less the shift, and values, into the slots >= 0."""
    keep = slots >= 0
    at = slots[keep]
    for name, x, g in (("k", k - cache["shift"], G_K), ("v", v, G_V)):
        codes, scales = _plain_quantize(x.unflatten(-1, (hkv, HEAD))[keep], g)
        cache[name][0][at] = codes
        cache[name][1][at] = scales


def _plain_gather(cache, slots, shift):
    out = []
    for name, g in (("k", G_K), ("v", G_V)):
        at = slots.clamp(min=0)
        x = _plain_values(cache[name][0][at], cache[name][1][at], g).flatten(1)
        if name == "k" and shift is not None:
            x = x + shift
        out.append(torch.where((slots >= 0)[:, None], x, torch.zeros_like(x)).to(torch.bfloat16))
    return tuple(out)


def _plain_attention(state):
    case, cache, hq, hkv = state["case"], state["cache"], state["hq"], state["hkv"]
    group, at = hq // hkv, 0
    out = torch.zeros((state["rows"], hq * HEAD), dtype=torch.bfloat16, device=DEV)
    lse = torch.full((state["rows"], hq), -math.inf, device=DEV)
    for b, (nq, n) in enumerate(state["lens"]):
        if n:
            slots = _slots(state["table"], b, 0, n, case["page"])
            k = _plain_values(cache["k"][0][slots], cache["k"][1][slots], G_K).permute(1, 2, 0).contiguous()
            v = _plain_values(cache["v"][0][slots], cache["v"][1][slots], G_V).permute(1, 0, 2).contiguous()
            piece = max(1, int(2e8) // (hq * n))
            for i0 in range(0, nq, piece):
                i1 = min(nq, i0 + piece)
                q = state["q"][at + i0:at + i1].float().view(i1 - i0, hkv, group, HEAD)
                q = q.permute(1, 2, 0, 3).reshape(hkv, group * (i1 - i0), HEAD)
                s = torch.matmul(q, k) * SM_SCALE
                s = s.view(hkv, group, i1 - i0, n)
                last = torch.arange(n - nq + i0, n - nq + i1, device=DEV)
                s = s.masked_fill(torch.arange(n, device=DEV)[None, :] > last[:, None], -math.inf)
                top = s.amax(-1, keepdim=True)
                p = torch.exp(s - top)
                total = p.sum(-1, keepdim=True)
                o = torch.matmul(p.view(hkv, -1, n), v).view(hkv, group, i1 - i0, HEAD) / total
                out[at + i0:at + i1] = o.permute(2, 0, 1, 3).reshape(i1 - i0, hq * HEAD).to(torch.bfloat16)
                lse[at + i0:at + i1] = (top + torch.log(total)).squeeze(-1).permute(2, 0, 1).reshape(i1 - i0, hq)
        at += nq
    return (out, lse) if case["lse"] else out


# ------------------------------------------------------------------ one pass

def run(state):
    kind, cache = state["case"]["kind"], state["cache"]
    if not own:
        if kind == "attn":
            return _plain_attention(state)
        if kind == "gather":
            return _plain_gather(cache, state["slots"], cache["shift"])
        hq, hkv = state["hq"], state["hkv"]
        cos, sin = (t[state["pos"].long()][:, None] for t in state["rope"])
        q = _plain_rotate(state["q"].float().unflatten(-1, (hq, HEAD)), cos, sin).flatten(1)
        k = _plain_rotate(state["k"].float().unflatten(-1, (hkv, HEAD)), cos, sin).flatten(1)
        _plain_put(cache, k, state["v"].float(), state["slots"], hkv)
        return (q.to(torch.bfloat16),) + _plain_gather(cache, state["slots"], None)
    reqat = state["reqat"]
    if kind == "attn":
        return reqat.kv4_attention(state["q"], cache, state["table"], state["kv_len"], q_start=state["q_start"],
                                   max_q=state["max_q"], max_kv=state["max_kv"], causal=True, sm_scale=SM_SCALE,
                                   return_lse=state["case"]["lse"], ws=state["ws"])
    if kind == "gather":
        return reqat.kv4_gather(cache, state["slots"], add_shift=True)
    q = reqat.kv4_append(cache, state["k"], state["v"], state["slots"], q=state["q"], rope=state["rope"],
                         positions=state["pos"])
    return (q,) + reqat.kv4_gather(cache, state["slots"])


# ------------------------------------------------------------------ the definition in 64 bits

def _exact_kv4(d, g):
    """What the 4-bit format holds of d [..., D] (float64), by division and rounding."""
    scales = sorted({(m / 8.0 + (1.0 if e else 0.0)) * 2.0 ** (max(e, 1) - 7)
                     for e in range(16) for m in range(8) if (e, m) != (15, 7)} - {0.0})
    table = torch.tensor(scales, dtype=torch.float64, device=d.device)
    shape = d.shape
    d = d.reshape(-1, 16)
    top = d.abs().max(dim=1).values
    which = torch.searchsorted(table, top / (3.5 * g)).clamp(max=len(scales) - 1)
    unit = (0.5 * g * table[which])[:, None]
    return (torch.round(d / unit).clamp(-7, 7) * unit).reshape(shape)


def exact(case, seed):
    hq, hkv = _heads(case)
    f64, f32 = torch.float64, torch.float32
    shift = _shift(case, seed)
    if case["kind"] == "append":
        qkv, pos, slots, _, _ = _new_tokens(case, seed)
        q, k, v = qkv.double().split([hq * HEAD, hkv * HEAD, hkv * HEAD], dim=1)
        cos, sin = (t.double()[pos.long()][:, None, :] for t in _rope_tables())

        def turned(x, heads):
            x = x.view(-1, heads, 2, HEAD // 2)
            lo, hi = x[:, :, 0], x[:, :, 1]
            # the definition takes each product and the sum to 32 bits; the products are exact in 64
            r = [((lo * cos).to(f32).double() - (hi * sin).to(f32).double()).to(f32).double(),
                 ((hi * cos).to(f32).double() + (lo * sin).to(f32).double()).to(f32).double()]
            return torch.stack(r, dim=2).reshape(-1, heads * HEAD)

        keys = (turned(k, hkv) - shift.double()).to(f32).double()
        held = [_exact_kv4(keys, G_K), _exact_kv4(v, G_V)]
        for x in held:
            x[slots < 0] = 0.0
        return (turned(q, hq), *held)

    def cached(b, n):
        k, v = _kv_of(case, seed, b, n, shift)
        return _exact_kv4((k.to(f32) - shift).double(), G_K), _exact_kv4(v.double(), G_V)

    if case["kind"] == "gather":
        k, v = cached(0, case["T"])
        return k + shift.double(), v
    queries = _queries(case, seed).double()
    outs, lses, at = [], [], 0
    for b, (nq, n) in enumerate(_lengths(case)):
        if n:
            k, v = cached(b, n)
        for h in range(hq if n else 0):
            hk = h // (hq // hkv)
            kh = k[:, hk * HEAD:(hk + 1) * HEAD]
            vh = v[:, hk * HEAD:(hk + 1) * HEAD]
            z = queries[at:at + nq, h * HEAD:(h + 1) * HEAD] @ kh.t().contiguous() * SM_SCALE
            hidden = torch.ones((nq, n), dtype=torch.bool, device=DEV).triu(diagonal=n - nq + 1)
            z[hidden] = -math.inf
            log_total = torch.logsumexp(z, dim=1)
            outs.append(torch.exp(z - log_total[:, None]) @ vh)
            lses.append(log_total)
        if not n:
            outs += [torch.zeros((nq, HEAD), dtype=f64, device=DEV)] * hq
            lses += [torch.full((nq,), -math.inf, dtype=f64, device=DEV)] * hq
        at += nq
    per = [torch.stack(x, dim=1) for x in (outs[i:i + hq] for i in range(0, len(outs), hq))]
    out = torch.cat(per).reshape(-1, hq * HEAD)
    if not case["lse"]:
        return out
    return out, torch.cat([torch.stack(lses[i:i + hq], dim=1) for i in range(0, len(lses), hq)])
