"""Refusals of the calls around the quantized layers (policy loss, norm, embedding, AdamW): on the host, before the device."""
import ctypes
import math
import os

import pytest
import torch

from paper_2606_15682_amd import reqat

P = 1 << 20                                             # an aligned address that nothing reads
F32, BF16 = reqat.DT_F32, reqat.DT_BF16
OK, NULL, SHAPE, ALIGN, ENUM, UNSUPPORTED = range(6)


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(reqat.LIB_PATH):
        pytest.skip("libreqat.so not built")
    return reqat.load()


def refused(call, base, want, **change):
    """The call with some of its arguments changed; every call here is refused."""
    unknown = set(change) - set(base)
    assert not unknown, unknown
    assert call(*{**base, **change}.values()) == want, change


def test_policy_loss():
    base = dict(logits=P, dtype=BF16, T=4, V=100, ld=104, targets=P, old=P, adv=P, ref=P, weights=None, low=0.2, high=0.2,
                kl=0.1, temp=1.0, stats=P, loss=P, grad=None, ldg=0, ws=P, stream=None)
    no = lambda want, **c: refused(reqat.reqat_policy_loss, base, want, **c)
    no(ENUM, dtype=2)
    no(ENUM, dtype=-1)
    for c in (dict(T=-1), dict(T=(1 << 22) + 1), dict(V=0), dict(V=-3), dict(V=(1 << 30) + 1, ld=1 << 31), dict(ld=99),
              dict(ld=1 << 62), dict(grad=2 * P, ldg=99), dict(grad=2 * P, ldg=1 << 62)):
        no(SHAPE, **c)
    for name in ("logits", "targets", "old", "adv", "ref", "stats", "loss"):
        no(NULL, **{name: None})
    for name, off in (("logits", 1), ("targets", 2), ("old", 1), ("adv", 2), ("ref", 2), ("weights", 2), ("stats", 8),
                      ("loss", 2)):
        no(ALIGN, **{name: P + off})
    no(ALIGN, dtype=F32, logits=P + 2)
    no(ALIGN, ws=P + 4)
    no(NULL, V=100000, ld=100000, ws=None)
    assert reqat.reqat_policy_loss_workspace_bytes(BF16, 4, 100) == 0
    assert reqat.reqat_policy_loss_workspace_bytes(BF16, 4, 100000) >= 4 * 16
    assert reqat.reqat_policy_loss_workspace_bytes(BF16, 100000, 100000) == 0
    assert reqat.reqat_policy_loss_workspace_bytes(5, 4, 100000) == reqat.reqat_policy_loss_workspace_bytes(F32, -1, 9) == 0
    no(ALIGN, grad=2 * P + 1, ldg=104)
    for c in (dict(low=-0.1), dict(low=1.5), dict(high=-0.1), dict(low=math.nan), dict(high=math.nan), dict(temp=0.0),
              dict(temp=-1.0), dict(temp=math.inf), dict(temp=math.nan), dict(grad=P + 2, ldg=104), dict(grad=P, ldg=100)):
        no(UNSUPPORTED, **c)


def test_policy_loss_backward():
    base = dict(logits=P, dtype=F32, T=4, V=100, ld=100, targets=P, stats=P, temp=1.0, grad_loss=None, grad=2 * P, ldg=100,
                stream=None)
    no = lambda want, **c: refused(reqat.reqat_policy_loss_backward, base, want, **c)
    no(ENUM, dtype=7)
    for c in (dict(T=-1), dict(V=0), dict(ld=99), dict(ldg=99)):
        no(SHAPE, **c)
    for name in ("logits", "targets", "stats", "grad"):
        no(NULL, **{name: None})
    no(ALIGN, grad=2 * P + 2)
    no(ALIGN, grad_loss=P + 1)
    no(UNSUPPORTED, grad=P + 4)
    no(UNSUPPORTED, temp=0.0)
    refused(reqat.reqat_policy_loss_backward, base, OK, T=0)


def test_layer_norm():
    base = dict(x=P, dtype=BF16, rows=3, cols=64, ldx=64, w=P, b=None, w_dtype=F32, eps=1e-6, center=1, y=2 * P, ldy=64,
                stats=P, stream=None)
    no = lambda want, **c: refused(reqat.reqat_layer_norm, base, want, **c)
    no(ENUM, dtype=3)
    no(ENUM, w_dtype=3)
    for c in (dict(rows=-1), dict(cols=0), dict(ldx=63), dict(ldy=63), dict(ldx=1 << 61)):
        no(SHAPE, **c)
    for name in ("x", "w", "y", "stats"):
        no(NULL, **{name: None})
    for name, off in (("x", 1), ("w", 2), ("b", 2), ("y", 1), ("stats", 2)):
        no(ALIGN, **{name: 2 * P + off})
    for c in (dict(cols=32769, ldx=32769, ldy=32769), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(y=P + 2),
              dict(y=P, ldy=72)):
        no(UNSUPPORTED, **c)
    refused(reqat.reqat_layer_norm, base, OK, rows=0)


def test_layer_norm_backward():
    base = dict(dy=3 * P, lddy=64, x=P, ldx=64, dtype=BF16, rows=3, cols=64, w=P, w_dtype=F32, stats=P, center=1, dx=2 * P,
                lddx=64, dw=P, db=None, ws=P, stream=None)
    no = lambda want, **c: refused(reqat.reqat_layer_norm_backward, base, want, **c)
    no(ENUM, dtype=3)
    for c in (dict(rows=-1), dict(cols=0), dict(ldx=63), dict(lddy=63), dict(lddx=63)):
        no(SHAPE, **c)
    for name in ("dy", "x", "w", "stats", "dx", "dw", "ws"):
        no(NULL, **{name: None})
    for name, off in (("dy", 1), ("dx", 1), ("dw", 2), ("db", 2), ("ws", 2)):
        no(ALIGN, **{name: 4 * P + off})
    for c in (dict(dx=P + 2), dict(dx=3 * P, lddx=72), dict(cols=40000, ldx=40000, lddy=40000, lddx=40000)):
        no(UNSUPPORTED, **c)


def test_layer_norm_workspace_never_falls():
    for dt in (F32, BF16):
        for cols in (1, 63, 1537, 5120, 32768):
            last = 0
            for rows in list(range(0, 2100, 7)) + [10 ** 6]:
                n = reqat.reqat_layer_norm_workspace_bytes(dt, rows, cols, 1)
                assert n >= last and n == 2 * reqat.reqat_layer_norm_workspace_bytes(dt, rows, cols, 0)
                last = n
    assert reqat.reqat_layer_norm_workspace_bytes(BF16, 5, 32769, 1) == 0
    assert reqat.reqat_layer_norm_workspace_bytes(9, 5, 5, 1) == 0


def test_embedding():
    base = dict(ids=P, T=5, table=P, dtype=F32, V=10, D=8, ld=8, scale=1.0, out=2 * P, ldo=8, stream=None)
    no = lambda want, **c: refused(reqat.reqat_embedding, base, want, **c)
    no(ENUM, dtype=4)
    for c in (dict(T=-1), dict(T=(1 << 22) + 1), dict(V=-1), dict(V=(1 << 23) + 1), dict(D=0), dict(D=(1 << 20) + 1), dict(ld=7),
              dict(ldo=7), dict(ld=1 << 61)):
        no(SHAPE, **c)
    for name in ("ids", "table", "out"):
        no(NULL, **{name: None})
    for name in ("ids", "table", "out"):
        no(ALIGN, **{name: 4 * P + 2})
    no(UNSUPPORTED, out=P + 32)
    refused(reqat.reqat_embedding, base, OK, T=0)


def test_embedding_backward():
    base = dict(dy=P, dtype=BF16, lddy=8, ids=P, T=5, V=10, D=8, scale=1.0, dtable=2 * P, tdtype=F32, ldt=8, accumulate=0, ws=P,
                stream=None)
    no = lambda want, **c: refused(reqat.reqat_embedding_backward, base, want, **c)
    no(ENUM, dtype=4)
    no(ENUM, tdtype=4)
    for c in (dict(T=-1), dict(V=-1), dict(D=0), dict(lddy=7), dict(ldt=7)):
        no(SHAPE, **c)
    for name in ("dy", "ids", "dtable"):
        no(NULL, **{name: None})
    no(NULL, T=1000, ws=None, dtable=4 * P)
    for name, off in (("dy", 1), ("ids", 2), ("dtable", 2), ("ws", 8)):
        no(ALIGN, **{name: 4 * P + off})
    no(UNSUPPORTED, dtable=P + 16)
    refused(reqat.reqat_embedding_backward, base, OK, T=0, accumulate=1)
    refused(reqat.reqat_embedding_backward, base, OK, V=0)


def test_embedding_workspace_never_falls():
    size = reqat.reqat_embedding_workspace_bytes
    for T in (0, 1, 63, 64, 65, 1000, 1 << 22):
        for V in (0, 1, 9, 152064):
            for D in (1, 7, 5120):
                n = size(T, V, D)
                assert n >= 16 * T if T > 512 else n == 0
                assert size(min(T + 1, 1 << 22), V, D) >= n and size(T, V + 1, D) >= n and size(T, V, D + 1) >= n
    assert size(-1, 5, 5) == 0 and size(5, -1, 5) == 0 and size(5, 5, 0) == 0


def test_adamw_step():
    def tensors(**change):
        t = (reqat.AdamwTensor * 2)()
        for x in t:
            x.p, x.g, x.m, x.v, x.m_scale, x.v_scale, x.copy, x.n = P, P, P, P, P, P, None, 10
        for k, v in change.items():
            setattr(t[1], k, v)
        return t

    def hyper(**change):
        h = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0, step=1)
        h.update(change)
        return reqat.AdamwHyper(*h.values())

    def call(t=None, count=2, p=F32, g=F32, bits=8, h=None, scale=None, coef=None):
        return reqat.reqat_adamw_step(tensors() if t is None else t, count, p, g, bits, hyper() if h is None else h, scale, coef,
                                      None)

    assert call(p=2) == ENUM and call(g=-1) == ENUM
    assert call(count=-1) == SHAPE
    assert call(bits=16) == UNSUPPORTED
    assert reqat.reqat_adamw_step(None, 2, F32, F32, 8, hyper(), None, None, None) == NULL
    assert reqat.reqat_adamw_step(tensors(), 2, F32, F32, 8, None, None, None, None) == NULL
    for c in (dict(step=0), dict(step=-5), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan),
              dict(eps=-1e-9), dict(eps=math.inf), dict(lr=math.nan), dict(weight_decay=math.inf)):
        assert call(h=hyper(**c)) == UNSUPPORTED, c
    assert call(scale=P + 2) == ALIGN and call(coef=P + 1) == ALIGN
    for name in ("p", "g", "m", "v", "m_scale", "v_scale"):
        assert call(tensors(**{name: None})) == NULL, name
    for name in ("p", "g", "m_scale", "v_scale"):
        assert call(tensors(**{name: P + 2})) == ALIGN, name
    for name in ("m", "v"):
        assert call(tensors(**{name: P + 2}), bits=32) == ALIGN, name
    assert call(tensors(copy=P + 1)) == ALIGN
    assert call(tensors(n=-1)) == SHAPE and call(tensors(n=(1 << 35) + 1)) == SHAPE
    assert call(count=0) == OK
    both = tensors(n=0, p=None, g=None)
    both[0].n = 0
    assert call(both) == OK                              # nothing but empty tensors


def test_adamw_other_calls():
    h = reqat.AdamwHyper(1e-3, 0.9, 0.99, 1e-8, 0.0, 1)
    f = reqat.reqat_adamw_coefficients
    assert f(None, P, P, P, None) == NULL and f(h, P, None, P, None) == NULL and f(h, P, P, None, None) == NULL
    assert f(h, P + 1, P, P, None) == ALIGN and f(h, P, P + 2, P, None) == ALIGN and f(h, P, P, P + 2, None) == ALIGN
    f = reqat.reqat_adamw_moments
    args = [P, P, P, P, 10, P, P, None]
    for i in (0, 1, 2, 3, 5, 6):
        assert f(*args[:i], None, *args[i + 1:]) == NULL
    for i in (1, 3, 5, 6):
        assert f(*args[:i], P + 2, *args[i + 1:]) == ALIGN
    assert f(*args[:4], -1, *args[5:]) == SHAPE and f(*args[:4], 0, *args[5:]) == OK
    assert ctypes.sizeof(reqat.AdamwTensor) == 64


# ------------------------------------------------------------------ the binding, on CPU tensors: refused before the C call

def no(exc, fn, *args, **kw):
    with pytest.raises(exc):
        fn(*args, **kw)


def test_binding_policy_loss():
    z, y, f = torch.zeros(3, 8), torch.zeros(3, dtype=torch.int32), torch.zeros(3)
    for call in (reqat.policy_loss, reqat.policy_loss_grad):
        no(TypeError, call, z, y, f, f)                   # a CPU tensor
        no(TypeError, call, z.half(), y, f, f)
        no(TypeError, call, z[0], y, f, f)
        no(ValueError, call, z.t(), torch.zeros(8, dtype=torch.int32), torch.zeros(8), torch.zeros(8))
        no(ValueError, call, z[:1].expand(3, 8), y, f, f)
        no(TypeError, call, z, y.long(), f, f)
        no(ValueError, call, z, y[:2], f, f)
        no(TypeError, call, z, y, f.double(), f)
        no(ValueError, call, z, y, f, f[:2])
        no(ValueError, call, z, y, f, f, kl_coef=0.1)
        no(ValueError, call, z, y, f, f, ref_logp=f[:1])
        no(ValueError, call, z, y, f, f, weights=torch.zeros(6)[::2])
    no(TypeError, reqat.policy_loss_grad, z, y, f, f, out=z.bfloat16())
    no(ValueError, reqat.policy_loss_grad, z, y, f, f, out=z[:2])
    no(ValueError, reqat.policy_loss_backward, z, y, f)
    no(TypeError, reqat.policy_loss_backward, z, y, torch.zeros(3, 4, dtype=torch.float64))
    no(TypeError, reqat.policy_loss_backward, z, y, torch.zeros(3, 4), grad_loss=2.0)
    no(TypeError, reqat.policy_loss_backward, z, y, torch.zeros(3, 4))


def test_binding_layer_norm():
    x, w = torch.zeros(3, 8), torch.zeros(8)
    no(TypeError, reqat.layer_norm, x, w)
    no(TypeError, reqat.layer_norm, x.double(), w)
    no(TypeError, reqat.layer_norm, x, w.half())
    no(ValueError, reqat.layer_norm, x, w[:7])
    no(TypeError, reqat.layer_norm, x, w, w.bfloat16())
    no(ValueError, reqat.layer_norm, x, w, out=x[:2])
    s = torch.zeros(3, 2)
    no(ValueError, reqat.layer_norm_backward, x[:2], x, w, s)
    no(ValueError, reqat.layer_norm_backward, x.bfloat16(), x, w, s)
    no(ValueError, reqat.layer_norm_backward, x, x, w, s.t().contiguous())
    no(ValueError, reqat.layer_norm_backward, x, x, w, s, ws=torch.zeros(3, dtype=torch.uint8))
    no(ValueError, reqat.layer_norm_backward, torch.zeros(8).expand(3, 8), x, w, s)
    no(TypeError, reqat.layer_norm_backward, x, x, w, s)


def test_binding_embedding():
    ids, table = torch.zeros(4, dtype=torch.int32), torch.zeros(5, 8)
    no(TypeError, reqat.embedding, ids, table)
    no(TypeError, reqat.embedding, ids.long(), table)
    no(TypeError, reqat.embedding, ids.view(2, 2), table)
    no(ValueError, reqat.embedding, torch.zeros(8, dtype=torch.int32)[::2], table)
    no(TypeError, reqat.embedding, ids, table.half())
    no(TypeError, reqat.embedding, ids, table, out=torch.zeros(4, 8).bfloat16())
    dy = torch.zeros(4, 8)
    no(ValueError, reqat.embedding_backward, dy, ids[:3], 5)
    no(ValueError, reqat.embedding_backward, dy, ids, 5, accumulate=True)
    no(ValueError, reqat.embedding_backward, dy, ids, 5, out=torch.zeros(4, 8))
    no(TypeError, reqat.embedding_backward, dy, ids, 5, out_dtype=torch.float16)
    no(ValueError, reqat.embedding_backward, torch.zeros(600, 8), torch.zeros(600, dtype=torch.int32), 5,
       ws=torch.zeros(9, dtype=torch.uint8))
    no(TypeError, reqat.embedding_backward, dy, ids, 5)


def test_binding_adamw():
    p = [torch.zeros(10), torch.zeros(3, 4)]
    no(ValueError, reqat.AdamW, [], 1e-3)
    no(ValueError, reqat.AdamW, p, 1e-3, state_bits=16)
    no(TypeError, reqat.AdamW, [torch.zeros(3).half()], 1e-3)
    no(TypeError, reqat.AdamW, [p[0], p[1].bfloat16()], 1e-3)
    no(ValueError, reqat.AdamW, [torch.zeros(4, 3).t()], 1e-3)
    no(ValueError, reqat.AdamW, [p[0], p[0]], 1e-3)       # the same twice
    no(ValueError, reqat.AdamW, [p[0][:6], p[0][5:]], 1e-3)
    no(ValueError, reqat.AdamW, p, 1e-3, copies=[None])
    no(TypeError, reqat.AdamW, p, 1e-3, copies=[torch.zeros(10), None])
    no(ValueError, reqat.AdamW, p, 1e-3, copies=[torch.zeros(9).bfloat16(), None])
    opt = reqat.AdamW(p, 1e-3, state_bits=8, copies=[torch.zeros(10).bfloat16(), None])
    assert opt.offsets == [0, 128] and opt.m.numel() == 256 and opt.m.dtype == torch.uint8 and opt.m_scale.numel() == 2
    assert reqat.AdamW([torch.zeros(0), torch.zeros(129)], 1e-3).m.numel() == 256
    g = [torch.zeros(10), torch.zeros(3, 4)]
    no(ValueError, opt.step, g[:1])
    no(ValueError, opt.step, [g[0], g[1].view(-1)])
    no(TypeError, opt.step, [g[0], g[1].bfloat16()])
    no(TypeError, opt.step, [g[0].half(), None])
    no(TypeError, opt.step, [g[0], 3.0])
    no(TypeError, opt.step, g, grad_scale=0.5)
    no(TypeError, opt.step, g)                            # CPU tensors
    assert opt.steps == 0
