"""Refusals of the paged KV4 cache's entry points (CPU: every call here ends
before a launch), and the binding's checks of its tensors."""
import ctypes
import os

import pytest
import torch

from paper_2606_15682_amd import reqat

P = 1 << 20
OK, E_NULL, E_SHAPE, E_ALIGN, E_UNSUP = 0, 1, 2, 3, 5

pytestmark = pytest.mark.skipif(not os.path.exists(reqat.LIB_PATH), reason="libreqat.so not built")


def cache(**kw):
    c = reqat.Kv4CacheStruct(P, P, P, P, P, P, None, 4, 16, 2, 128)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def append(c=None, T=4, slots=P, k=P, ldk=256, v=P, ldv=256, q=P, ldq=1024, q_heads=8, q_out=2 * P, ldqo=1024, cos=P, sin=P,
           pos=P, rope_len=9):
    return reqat.reqat_kv4_append(cache() if c is None else c, T, slots, k, ldk, v, ldv, q, ldq, q_heads, q_out, ldqo, cos,
                                  sin, pos, rope_len, None)


def gather(c=None, T=4, slots=P, k=P, ldk=256, v=P, ldv=256, add=0):
    return reqat.reqat_kv4_gather(cache() if c is None else c, T, slots, k, ldk, v, ldv, add, None)


def attend(c=None, B=2, T=2, q=P, ldq=1024, q_heads=8, q_start=None, kv_len=P, table=P, ldt=4, cols=4, max_q=1, max_kv=64,
           causal=1, scale=0.1, out=2 * P, ldo=1024, lse=None, ws=P):
    return reqat.reqat_kv4_attention(cache() if c is None else c, B, T, q, ldq, q_heads, q_start, kv_len, table, ldt, cols,
                                     max_q, max_kv, causal, scale, out, ldo, lse, ws, None)


@pytest.mark.parametrize("call", [append, gather, attend])
def test_cache_arguments(call):
    if call is gather:
        assert reqat.reqat_kv4_gather(None, 4, P, P, 256, P, 256, 0, None) == E_NULL
    for name in ("k_codes", "k_scales", "v_codes", "v_scales", "k_tensor_scale", "v_tensor_scale"):
        assert call(cache(**{name: None})) == E_NULL
    for name in ("k_codes", "k_scales", "v_codes", "v_scales", "k_shift"):
        assert call(cache(**{name: P + 8})) == E_ALIGN
    assert call(cache(k_tensor_scale=P + 2)) == E_ALIGN
    assert call(cache(num_pages=-1)) == E_SHAPE
    assert call(cache(num_pages=2 ** 62)) == E_SHAPE
    for size in (0, 8, 24, 48, -16, 1 << 21):
        assert call(cache(page_size=size)) == E_SHAPE
    for heads in (0, -1, 1 << 20):
        assert call(cache(kv_heads=heads)) == E_SHAPE
    for d in (0, 32, 80, 96, 256):
        assert call(cache(head_dim=d)) == E_UNSUP


def test_append_arguments():
    assert append(T=-1) == E_SHAPE and append(T=1 << 31) == E_SHAPE
    assert append(q_heads=-1) == E_SHAPE and append(rope_len=-1) == E_SHAPE
    for name in ("slots", "k", "v", "q", "q_out", "cos", "sin", "pos"):
        assert append(**{name: None}) == E_NULL, name
    assert append(cos=None, sin=None, pos=None) == E_NULL             # queries need the tables
    for name in ("ldk", "ldv"):
        assert append(**{name: 248}) == E_SHAPE and append(**{name: 260}) == E_ALIGN
    for name in ("ldq", "ldqo"):
        assert append(**{name: 1016}) == E_SHAPE and append(**{name: 1028}) == E_ALIGN
    for name in ("k", "v", "q", "q_out", "cos", "sin"):
        assert append(**{name: P + 8}) == E_ALIGN, name
    assert append(slots=P + 4) == E_ALIGN and append(pos=P + 2) == E_ALIGN
    assert append(q_out=P + 64) == E_UNSUP                            # overlaps q
    assert append(q_out=P, ldqo=1032) == E_UNSUP                      # in place needs one stride
    assert append(T=0, slots=None, k=None, v=None, q=None, q_out=None, pos=None) == OK


def test_gather_arguments():
    assert gather(T=-1) == E_SHAPE and gather(slots=None) == E_NULL
    assert gather(ldk=248) == E_SHAPE and gather(ldv=260) == E_ALIGN and gather(k=P + 8) == E_ALIGN
    assert gather(slots=P + 4) == E_ALIGN
    assert gather(T=0) == OK and gather(k=None, v=None) == OK


def test_attention_arguments():
    for name in ("B", "T", "max_q", "max_kv", "cols"):
        assert attend(**{name: -1}) == E_SHAPE, name
    assert attend(B=3) == E_SHAPE                                     # one query each needs T == B
    assert attend(B=1 << 16, T=1 << 16) == E_SHAPE
    assert attend(q_heads=7) == E_SHAPE and attend(q_heads=0) == E_SHAPE
    assert attend(ldt=3) == E_SHAPE
    for name in ("q", "out", "kv_len", "table"):
        assert attend(**{name: None}) == E_NULL, name
    assert attend(ldq=1016) == E_SHAPE and attend(ldo=1028) == E_ALIGN and attend(q=P + 8) == E_ALIGN
    assert attend(kv_len=P + 2) == E_ALIGN and attend(lse=P + 1) == E_ALIGN and attend(ws=P + 4) == E_ALIGN
    for s in (0.0, -1.0, float("nan"), float("inf")):
        assert attend(scale=s) == E_UNSUP
    assert attend(out=P + 512) == E_UNSUP                             # overlaps q
    need = reqat.reqat_kv4_attention_workspace_bytes(1, 1, 1, 1 << 20, 8, 2, 128)
    if need > 0:
        assert attend(B=1, T=1, max_kv=1 << 20, ws=None) == E_NULL
    assert attend(B=0, T=0) == OK and attend(max_q=0) == OK


def test_workspace_query():
    f = reqat.reqat_kv4_attention_workspace_bytes
    for bad in ((-1, 1, 1, 1, 8, 2, 128), (1, -1, 1, 1, 8, 2, 128), (1, 1, -1, 1, 8, 2, 128), (1, 1, 1, -1, 8, 2, 128),
                (1, 1, 1, 1, 7, 2, 128), (1, 1, 1, 1, 8, 0, 128), (1, 1, 1, 1, 8, 2, 96), (1 << 17, 1, 1, 1, 8, 2, 128)):
        assert f(*bad) == 0
    for B in (1, 3, 64, 65535):
        for kv in (0, 1, 1000, 131072, 2 ** 31 - 1):
            for q in (1, 5, 64, 8192):
                assert 0 <= f(B, B * q, q, kv, 40, 8, 128) < 2 ** 40


def test_binding_checks_before_any_call():
    with pytest.raises(ValueError):
        reqat.Kv4Cache(4, 24, 2, 128, device="cpu")
    with pytest.raises(ValueError):
        reqat.Kv4Cache(4, 16, 2, 80, device="cpu")
    with pytest.raises(ValueError):
        reqat.Kv4Cache(4, 16, 2, 128, k_scale=0.0, device="cpu")
    with pytest.raises(ValueError):
        reqat.Kv4Cache(4, 16, 2, 128, k_shift=torch.zeros(128), device="cpu")
    c = reqat.Kv4Cache(4, 16, 2, 128, device="cpu")
    assert c.k_codes.numel() == 4 * 16 * 2 * 64 and c.v_scales.numel() == 4 * 16 * 2 * 8 and c.width == 256
    assert ctypes.sizeof(c.struct) == 88
    bf = lambda r, n: torch.zeros((r, n), dtype=torch.bfloat16)
    slots = torch.zeros(3, dtype=torch.int64)
    cos = torch.zeros((5, 64))
    pos = torch.zeros(3, dtype=torch.int32)
    for bad, err in ((dict(k=bf(3, 128)), ValueError), (dict(v=bf(2, 256)), ValueError), (dict(slots=slots.int()), TypeError),
                     (dict(slots=slots[:2]), ValueError), (dict(k=torch.zeros((3, 256))), TypeError),
                     (dict(q=bf(3, 256)), ValueError), (dict(q=bf(3, 100), rope=(cos, cos), positions=pos), ValueError),
                     (dict(rope=(cos, cos[:4]), positions=pos), ValueError), (dict(rope=(cos, cos)), TypeError),
                     (dict(positions=pos), ValueError), (dict(q_out=bf(3, 256)), ValueError)):
        args = dict(k=bf(3, 256), v=bf(3, 256), slots=slots)
        args.update(bad)
        with pytest.raises(err):
            reqat.kv4_append(c, **args)
    with pytest.raises(TypeError):                  # all else holds: the tensors are not on a GPU
        reqat.kv4_append(c, bf(3, 256), bf(3, 256), slots)
    with pytest.raises(TypeError):
        reqat.kv4_gather(c, slots)
    with pytest.raises(TypeError):
        reqat.kv4_gather(c, slots.int())
    table, n = torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for bad, err in ((dict(q=bf(3, 300)), ValueError), (dict(q=bf(2, 512)), ValueError), (dict(block_table=table.long()), TypeError),
                     (dict(kv_len=n[:2]), ValueError), (dict(q_start=n), ValueError),
                     (dict(ws=torch.zeros(4)), TypeError), (dict(out=bf(3, 256)), ValueError)):
        args = dict(q=bf(3, 512), block_table=table, kv_len=n)
        args.update(bad)
        with pytest.raises(err):
            reqat.kv4_attention(cache=c, **args)
    with pytest.raises(TypeError):
        reqat.kv4_attention(c, bf(3, 512), table, n)
