"""AdamW's host side on CPU tensors, with the C calls recorded instead of made: what a step hands over."""
import contextlib
import copy

import pytest
import torch

from paper_2606_15682_amd import reqat

WORDS = ("p", "g", "m", "v", "m_scale", "v_scale", "copy", "n")


@pytest.fixture
def calls(monkeypatch):
    """The calls made: (name of the C function, its arguments, the descriptors as dicts where it takes some)."""
    made = []

    def record(fn, device, *args):
        words = None
        if fn is reqat.reqat_adamw_step:
            words = [dict(zip(WORDS, args[0][8 * i:8 * i + 8])) for i in range(args[1])]
        made.append((fn.__name__, args, words))

    monkeypatch.setattr(reqat, "_call", record)
    monkeypatch.setattr(reqat, "_require_cuda", lambda *a: None)
    return made


def _params():
    return [torch.ones(10), torch.ones(3, 4), torch.ones(7)]


def _grads():
    return [torch.ones(10), torch.ones(3, 4), torch.ones(7)]


def _steps(calls):
    return [(args, words) for name, args, words in calls if name == "reqat_adamw_step"]


@pytest.mark.parametrize("bits", [8, 32])
def test_copies_taken_away_and_given(calls, bits):
    """Without copies no address of an earlier step's stays in the descriptors; given ones are the ones handed over."""
    p, g = _params(), _grads()
    copies = [torch.empty(10, dtype=torch.bfloat16), None, torch.empty(7, dtype=torch.bfloat16)]
    opt = reqat.AdamW(p, 1e-3, state_bits=bits, copies=copies)
    opt.step(g)
    assert [w["copy"] for w in _steps(calls)[-1][1]] == [copies[0].data_ptr(), 0, copies[2].data_ptr()]
    opt.copies = None
    opt.step(g)
    assert [w["copy"] for w in _steps(calls)[-1][1]] == [0, 0, 0]
    opt.copies = [None, torch.empty(3, 4, dtype=torch.bfloat16), None]
    opt.step(g)
    assert [w["copy"] for w in _steps(calls)[-1][1]] == [0, opt.copies[1].data_ptr(), 0]
    opt.copies = [None, None, None]
    opt.step(g)
    assert [w["copy"] for w in _steps(calls)[-1][1]] == [0, 0, 0]
    for wrong in ([None, None], [None] * 4):
        opt.copies = wrong
        with pytest.raises(ValueError):
            opt.step(g)
    opt.copies = None
    opt.step(g)
    assert opt.steps == 5 and len(_steps(calls)) == 5
    for x, w in zip(p, _steps(calls)[-1][1]):
        assert w["p"] == x.data_ptr() and w["n"] == x.numel()


def _counts(calls, params):
    """Parameter -> its step, of the calls made for one step; no parameter is in two of them."""
    out = {}
    for args, words in _steps(calls):
        for i, w in enumerate(words):
            if w["n"]:
                assert i not in out and w["n"] == params[i].numel() and w["g"]
                out[i] = args[5].step
    calls.clear()
    return out


def test_left_out_parameters_keep_their_count(calls):
    """The bias correction of a parameter goes by the steps that its moments have taken."""
    p, g = _params(), _grads()
    opt = reqat.AdamW(p, 1e-3)
    opt.step(g)
    assert _counts(calls, p) == {0: 1, 1: 1, 2: 1}
    for k in range(2, 6):
        opt.step([g[0], None, g[2]])
        assert _counts(calls, p) == {0: k, 2: k}
    opt.step(g)
    assert _counts(calls, p) == {0: 6, 1: 2, 2: 6}
    opt.step([None, None, None])
    assert _counts(calls, p) == {}
    opt.step([None, g[1], g[2]])
    assert _counts(calls, p) == {1: 3, 2: 7}
    opt.step(g)
    assert _counts(calls, p) == {0: 7, 1: 4, 2: 8} and opt.steps == 9 and opt.missed == [2, 5, 1]
    other = copy.deepcopy(opt)
    other.step(g)
    assert _counts(calls, other.params) == {0: 8, 1: 5, 2: 9} and opt.steps == 9
    opt.steps, opt.missed = 100, [0, 0, 40]
    opt.step(g)
    assert _counts(calls, p) == {0: 101, 1: 101, 2: 61}


def test_captured_steps_have_one_count(calls, monkeypatch):
    """On the device one count serves all parameters, so all steps have gradients for the same; what a capture records has
    not run and is not counted."""
    capturing = [False]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    p, g = _params(), _grads()
    opt = reqat.AdamW(p, 1e-3, captured=True)
    opt.step([None] * 3)                                  # moves nothing and counts nothing
    assert not calls and opt.steps == 0
    opt.step([g[0], None, g[2]])
    assert [c[0] for c in calls] == ["reqat_adamw_coefficients", "reqat_adamw_step"]
    assert [w["n"] for w in calls[1][2]] == [10, 0, 7]
    for wrong in (g, [g[0], g[1], None], [None] * 3):
        with pytest.raises(ValueError):
            opt.step(wrong)
    capturing[0] = True
    opt.step([g[0], None, g[2]])
    assert len(calls) == 4 and opt.steps == 1


@pytest.mark.parametrize("bits", [8, 32])
def test_other_tensors_in_the_same_memory_are_checked(calls, bits):
    """A replaced tensor is checked also where it begins at the address of the one before it."""
    p, g = _params(), _grads()
    opt = reqat.AdamW(p, 1e-3, state_bits=bits, copies=[torch.empty(10, dtype=torch.bfloat16), None, None])
    opt.step(g)
    for name, wrong in (("params", p[0][:5]), ("params", p[0].view(2, 5)), ("params", p[0].view(torch.int32)),
                        ("copies", opt.copies[0][:9]), ("copies", opt.copies[0].view(torch.float16))):
        held = getattr(opt, name)
        kept, held[0] = held[0], wrong
        with pytest.raises((TypeError, ValueError)):
            opt.step(g)
        held[0] = kept
    for name in ("m", "v", "m_scale", "v_scale")[:2 if bits == 32 else 4]:
        kept = getattr(opt, name)
        for wrong in (kept[:1], kept.view(torch.int32 if bits == 32 or "scale" in name else torch.int8), None):
            setattr(opt, name, wrong)
            with pytest.raises((TypeError, ValueError)):
                opt.step(g)
        setattr(opt, name, kept)
    kept, opt.v = opt.v, opt.m                            # one buffer for both
    with pytest.raises(ValueError):
        opt.step(g)
    opt.v, opt.copies = kept, None
    opt.step(g)
    for i, w in enumerate(_steps(calls)[-1][1]):          # nothing of what was refused stays
        at = opt.offsets[i]
        assert w["m"] == opt.m[at:].data_ptr() and w["v"] == opt.v[at:].data_ptr()
        if bits == 8:
            assert w["m_scale"] == opt.m_scale[at // 128:].data_ptr() and w["v_scale"] == opt.v_scale[at // 128:].data_ptr()
    opt.params[0] = p[0][:5]
    with pytest.raises(ValueError):
        opt.step(g)
    assert opt.steps == 2 and len(_steps(calls)) == 2
