"""Operators on rows of class logits, what needs no GPU: the refusals of their entry points (all made before any call of the
runtime), and the plain implementation that the GPU tests compare with, itself against differences and hand-made values."""
import ctypes as C
import itertools
import math

import numpy as np
import pytest

import logit_rows_plain as plain
import paper_2108_09413_amd as isr

BASE = 0x7F0000000000   # addresses that no check reads from


def _logits(data=BASE, kind=isr.BF16, classes=100, rows=4, stride=104, scale=1.0):
    return isr.Logits(data, kind, classes, rows, stride, scale)


def _teacher(cls=BASE + (1 << 30), logit=BASE + (1 << 31), kind=isr.F32, top=8, scale=1.0, rest=0):
    return isr.Teacher(cls, logit, kind, top, scale, rest)


P = [BASE + (1 << 32) + i * (1 << 24) for i in range(8)]


def _logprobs(l, given=P[0], n=2, top=3, lp=P[1], h=P[2], tc=P[3], tl=P[4], st=P[5], ws=P[6], bytes_=0):
    return isr.lib().isr_logprobs(C.byref(l) if l else None, given, n, top, lp, h, tc, tl, st, ws, bytes_, None)


def _grad(l, given=P[0], n=2, up=P[1], h=P[2], up_h=P[3], st=P[4], out=P[5], stride=104):
    return isr.lib().isr_logprobs_grad(C.byref(l) if l else None, given, n, up, h, up_h, st, out, stride, None)


def _distill(l, t, w=P[0], loss=P[1], st=P[2], out=P[3], stride=104, ws=P[4], bytes_=0):
    return isr.lib().isr_distill(C.byref(l) if l else None, C.byref(t) if t else None, w, loss, st, out, stride, ws, bytes_, None)


def _distill_grad(l, t, w=P[0], st=P[1], out=P[2], stride=104):
    return isr.lib().isr_distill_grad(C.byref(l) if l else None, C.byref(t) if t else None, w, st, out, stride, None)


BAD_LOGITS = [dict(data=None), dict(data=BASE + 1), dict(kind=4), dict(kind=-1), dict(classes=0), dict(classes=(1 << 24) + 1, stride=1 << 25),
              dict(rows=1 << 31), dict(stride=99), dict(stride=1 << 62), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf),
              dict(scale=math.nan), dict(scale=1e-31), dict(scale=2e30), dict(kind=isr.F32, data=BASE + 2)]


@pytest.mark.parametrize("bad", BAD_LOGITS, ids=str)
def test_bad_logits_are_refused_by_every_entry_point(bad):
    l = _logits(**bad)
    for rc in (_logprobs(l), _grad(l, stride=1 << 25), _distill(l, _teacher(), stride=1 << 25, bytes_=1 << 40), _distill_grad(l, _teacher(), stride=1 << 25)):
        assert rc == isr.ISR_ERR_ARG


def test_null_descriptors_are_refused():
    assert _logprobs(None) == _grad(None) == _distill(None, _teacher()) == _distill(_logits(), None) == isr.ISR_ERR_ARG
    assert _distill_grad(None, _teacher()) == _distill_grad(_logits(), None) == isr.ISR_ERR_ARG
    L = isr.lib()
    assert L.isr_logprobs_workspace_bytes(None, 5) == 0 and L.isr_distill_workspace_bytes(None, None) == 0


@pytest.mark.parametrize("bad", [dict(n=129), dict(top=129), dict(given=None), dict(lp=None), dict(tc=None), dict(tl=None), dict(given=P[0] + 2),
                                 dict(lp=P[0] + 1), dict(h=P[0] + 3), dict(tc=P[0] + 2), dict(tl=P[0] + 2), dict(st=P[0] + 2),
                                 dict(n=0, top=0, h=None, st=None)], ids=str)
def test_bad_arguments_of_logprobs_are_refused(bad):
    assert _logprobs(_logits(), **bad, bytes_=1 << 40) == isr.ISR_ERR_ARG


def test_more_top_alternatives_than_classes_are_refused():
    assert _logprobs(_logits(classes=3), top=4, bytes_=1 << 40) == isr.ISR_ERR_ARG


@pytest.mark.parametrize("bad", [dict(n=129), dict(given=None), dict(up=None), dict(st=None), dict(out=None), dict(h=None), dict(up_h=None),
                                 dict(n=0, h=None, up_h=None), dict(stride=99), dict(out=P[5] + 1), dict(st=P[4] + 2), dict(up=P[1] + 1),
                                 dict(out=BASE), dict(out=BASE + 16), dict(out=BASE - 16), dict(out=BASE + 3 * 104 * 2)], ids=str)
def test_bad_arguments_of_the_gradient_are_refused(bad):
    """The last four: over the logits' memory with another stride, and across either end of it."""
    args = dict(bad)
    if bad.get("out") == BASE:
        args["stride"] = 112
    assert _grad(_logits(), **args) == isr.ISR_ERR_ARG


def test_int32_logits_are_not_overwritten():
    assert _grad(_logits(kind=isr.I32), out=BASE) == isr.ISR_ERR_ARG


@pytest.mark.parametrize("bad", [dict(cls=None), dict(logit=None), dict(cls=P[7] + 2), dict(logit=P[7] + 2), dict(kind=isr.I32), dict(kind=-1),
                                 dict(top=0), dict(top=129), dict(scale=0.0), dict(scale=math.nan), dict(rest=2), dict(rest=-1)], ids=str)
def test_bad_teachers_are_refused(bad):
    t = _teacher(**bad)
    assert _distill(_logits(), t, bytes_=1 << 40) == _distill_grad(_logits(), t) == isr.ISR_ERR_ARG


@pytest.mark.parametrize("bad", [dict(loss=None), dict(loss=P[1] + 1), dict(w=P[0] + 2), dict(st=P[2] + 2), dict(stride=99), dict(out=P[3] + 1)], ids=str)
def test_bad_arguments_of_the_distillation_are_refused(bad):
    assert _distill(_logits(), _teacher(), **bad, bytes_=1 << 40) == isr.ISR_ERR_ARG


def test_workspaces_too_small_are_refused():
    t = _teacher()
    for rows, classes in itertools.product((1, 64, 4096), (100, 5003, 262144, 1 << 24)):
        l = _logits(classes=classes, rows=rows, stride=classes)
        need = isr.lib().isr_distill_workspace_bytes(C.byref(l), C.byref(t))
        assert need > 0 or classes < 262144
        if need:
            assert _distill(l, t, out=None, bytes_=need - 1) == _distill(l, t, out=None, ws=None, bytes_=need) == isr.ISR_ERR_WORKSPACE
    for rows, classes, top in itertools.product((1, 64), (100, 262144, 1 << 24), (0, 1, 128)):
        l = _logits(classes=classes, rows=rows, stride=classes)
        need = isr.lib().isr_logprobs_workspace_bytes(C.byref(l), min(top, classes))
        if need:
            assert _logprobs(l, top=min(top, classes), bytes_=need - 1) == isr.ISR_ERR_WORKSPACE
            assert _logprobs(l, top=min(top, classes), ws=None, bytes_=need) == isr.ISR_ERR_WORKSPACE


def test_no_rows_are_no_work():
    l, t = _logits(data=None, rows=0), _teacher(cls=None, logit=None)
    assert _logprobs(l, given=None, lp=None) == _grad(l, given=None, up=None, st=None, out=None) == isr.ISR_OK
    assert _distill(l, t, loss=None, out=None) == _distill_grad(l, t, st=None, out=None) == isr.ISR_OK


def test_tensors_outside_the_device_are_refused():
    import torch
    x = torch.zeros(2, 5)
    for call in (lambda: isr.isr_logprobs(x, top=1), lambda: isr.isr_logprobs(x.double(), top=1),
                 lambda: isr.isr_distill(x, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1))):
        with pytest.raises(isr.IsrError) as e:
            call()
        assert e.value.status == isr.ISR_ERR_ARG


# ---- the plain implementation ------------------------------------------------------

def test_plain_logprobs_by_hand():
    x = np.log(np.array([[1.0, 2.0, 5.0, 2.0]]))
    lp, h, tc, tl = plain.logprobs(x, 1.0, np.array([[2, -1, 4, 2]]), 4)
    assert np.allclose(lp[0][[0, 1, 3]], [math.log(0.5), 0.0, math.log(0.5)], atol=1e-15) and np.isnan(lp[0][2])
    assert h[0] == pytest.approx(0.5 * math.log(2) + 0.1 * math.log(10) + 0.4 * math.log(5), abs=1e-15)
    assert tc[0].tolist() == [2, 1, 3, 0] and tl[0][3] == pytest.approx(math.log(0.1))
    lp, h, tc, tl = plain.logprobs(np.array([[-np.inf, -np.inf], [np.nan, 0], [0, -np.inf]]), 2.0, np.array([[1], [1], [0]]), 2)
    assert lp[0][0] == -np.inf and h[0] == 0 and tc[0].tolist() == [-1, -1] and np.isnan(lp[1][0]) and tc[1].tolist() == [-1, -1]
    assert lp[2][0] == 0 and h[2] == 0 and tc[2].tolist() == [0, -1] and tl[2].tolist() == [0, -np.inf]


def test_plain_distillation_by_hand():
    """Student and teacher agree: no loss, no gradient.  The rest class alone: log of its share."""
    x = np.log(np.array([[1.0, 2.0, 5.0, 2.0]]))
    entry, value = np.array([[2, 0]]), np.log(np.array([[0.5, 0.1]]))
    loss, _, g, _ = plain.distill(x, 1.0, entry, value, 1.0, True)
    assert abs(loss[0]) < 1e-15 and np.abs(g).max() < 1e-15
    loss, _, g, _ = plain.distill(x, 1.0, np.array([[2, -1]]), np.array([[3.0, 9.0]]), 1.0, False)
    assert loss[0] == pytest.approx(math.log(2)) and np.allclose(g[0], [0.1, 0.2, -0.5, 0.2])
    loss, _, g, _ = plain.distill(x, 1.0, np.array([[2, 2]]), np.log(np.array([[0.25, 0.25]])), 1.0, True)
    assert loss[0] == pytest.approx(0.5 * math.log(0.5)) and np.abs(g).max() < 1e-15   # the class named twice gets both
    loss, _, g, _ = plain.distill(x, 1.0, np.array([[-1, -1]]), value, 1.0, True)
    assert loss[0] == 0 and not g.any()


@pytest.mark.parametrize("seed", range(3))
def test_plain_gradients_against_differences(seed):
    rng = np.random.default_rng(seed)
    x, step = rng.normal(size=(3, 9)) * 2, 1e-5
    given, up, up_h = rng.integers(-1, 9, (3, 2)), rng.normal(size=(3, 2)), rng.normal(size=3)
    entry, value, w = rng.integers(-1, 9, (3, 4)), rng.normal(size=(3, 4)) - 2.5, rng.normal(size=3)

    def f_logprobs(z):
        lp, h, _, _ = plain.logprobs(z, 0.7, given, 0)
        return (lp * up).sum(1) + h * up_h

    for f, g in [(f_logprobs, plain.logprobs_grad(x, 0.7, given, up, up_h)[0])] + [
            (lambda z, rest=rest: w * plain.distill(z, 0.7, entry, value, 1.3, rest)[0], plain.distill(x, 0.7, entry, value, 1.3, rest, w)[2]) for rest in (False, True)]:
        for j in range(9):
            e = np.zeros(9)
            e[j] = step
            assert np.allclose((f(x + e) - f(x - e)) / (2 * step), g[:, j], atol=1e-8)
