"""Operators on rows of class logits on the GPU against the plain implementation in 64 bits (logit_rows_plain.py, which also
says how far 32 bits may be off)."""
import ctypes as C
import math

import numpy as np
import pytest

import logit_rows_plain as plain

pytestmark = pytest.mark.gpu
TYPES = ("f32", "bf16", "f16", "i32")


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


@pytest.fixture(scope="module")
def isr(torch):
    import paper_2108_09413_amd as lib
    return lib


def dtype_of(torch, kind):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i32": torch.int32}[kind]


def make(torch, kind, rows, classes, seed, pad=0, shift=0, peaks=4):
    """(device [rows, classes] view with `pad` foreign columns a row, `shift` elements into its memory; its values in 64 bits)"""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(rows, classes)) * 2.5
    for r in range(rows):
        x[r, rng.integers(0, classes, peaks)] = 4 + 8 * rng.random(peaks)
    x = np.round(x * 1000) if kind == "i32" else x
    return put(torch, kind, x, pad, shift)


def put(torch, kind, x, pad=0, shift=0):
    rows, classes = x.shape
    dtype = dtype_of(torch, kind)
    flat = torch.full((shift + rows * (classes + pad) + 64,), 1000, dtype=dtype)   # foreign columns would be the largest
    view = flat[shift:shift + rows * (classes + pad)].view(rows, classes + pad)[:, :classes]
    view.copy_(torch.from_numpy(np.ascontiguousarray(x)).to(dtype))
    wide = view.to(torch.float64).numpy() if kind != "i32" else view.numpy().astype(np.float64)
    dev = flat.cuda()
    return dev[shift:shift + rows * (classes + pad)].view(rows, classes + pad)[:, :classes], wide


def scale_of(kind, s=1.0):
    return s * (2.0 ** -10 if kind == "i32" else 1.0)


def close(got, want, tol, what):
    got, want = got.double().cpu().numpy(), np.asarray(want)
    assert got.shape == want.shape, what
    # results are fp32: what is beyond its largest number by more than half a step rounds to infinity (the difference of fp32's
    # two ends is 2 * 3.4e38)
    want = np.where(np.abs(want) >= 2.0 ** 128 * (1 - 2.0 ** -25), np.copysign(np.inf, want), want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    fin = np.isfinite(want)
    assert np.array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)]), what
    with np.errstate(invalid="ignore"):
        over = np.abs(got - want) > np.broadcast_to(tol, want.shape)
    bad = np.argwhere(over & fin)
    assert not len(bad), (what, len(bad), bad[0], got[tuple(bad[0])], want[tuple(bad[0])], np.broadcast_to(tol, want.shape)[tuple(bad[0])])


def grad_tol(kind, want, tol):
    """The rounding to the logits' type: half a step of the value, or of the smallest number."""
    half = {"f32": 2.0 ** -24, "i32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[kind]
    least = {"f32": 2.0 ** -126, "i32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}[kind]
    return tol + half * (np.abs(np.nan_to_num(want)) + tol) + least


def check_logprobs(isr, torch, kind, dev, wide, scale, given=None, top=0):
    g = None if given is None else torch.from_numpy(np.ascontiguousarray(given, dtype=np.int32)).cuda()
    r = isr.isr_logprobs(dev, g, top=top, entropy=True, scale=scale, stats=True)
    lp, h, tc, tl = plain.logprobs(wide, scale, given, top)
    if given is not None:
        close(r.given, lp, plain.logp_tol(lp), "log-probabilities")
    # the entropy is log s - t / s: two sums of terms up to log V times a probability
    close(r.entropy, h, plain.U * plain.SUM * (2 + 2 * math.log(dev.shape[1]) + 1), "entropy")
    if top:
        assert np.array_equal(r.top_class.cpu().numpy(), tc), "top classes"
        close(r.top, tl, plain.logp_tol(tl), "top log-probabilities")
    return r


def check_grad(isr, torch, kind, dev, wide, scale, given, up, up_h, r, out=None):
    g = None if given is None else torch.from_numpy(np.ascontiguousarray(given, dtype=np.int32)).cuda()
    up32 = None if up is None else torch.from_numpy(np.ascontiguousarray(up, dtype=np.float32)).cuda()
    h32 = None if up_h is None else torch.from_numpy(up_h.astype(np.float32)).cuda()
    got = isr.isr_logprobs_grad(dev, g, up32, r.stats, entropy=r.entropy if up_h is not None else None, grad_entropy=h32, scale=scale, out=out)
    want, tol = plain.logprobs_grad(wide, scale, given if given is not None else None, None if up is None else up.astype(np.float32).astype(np.float64),
                                    None if up_h is None else up_h.astype(np.float32).astype(np.float64))
    close(got, want, grad_tol(kind, want, tol), "gradient")
    return got


CLASSES = [1, 2, 3, 7, 10, 15, 16, 17, 64, 65, 101, 128, 129, 255, 256, 257, 511, 513, 1000, 1024, 1025, 2047, 2049, 2055, 4099, 8193, 16385, 32771, 50021, 131080]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("classes", CLASSES)
def test_logprobs_and_gradient(isr, torch, kind, classes):
    """Sizes next to every boundary of the kernels, rows that start at any element, foreign columns behind them."""
    rng = np.random.default_rng(classes)
    for case, (rows, pad, shift, n, top, s) in enumerate(((3, 0, 0, 1, 5, 1.0), (5, 3, 1, 3, 20, 0.5), (2, 8, 5, 1, 64, 1.25), (1, 1, 3, 8, 128, 2.0))):
        if classes > 20000 and case in (1, 3):
            continue
        print(kind, classes, case, flush=True)
        dev, wide = make(torch, kind, rows, classes, 7 * classes + case, pad, shift)
        scale, top = scale_of(kind, s), min(top, classes)
        given = rng.integers(-1, classes, (rows, n))
        r = check_logprobs(isr, torch, kind, dev, wide, scale, given, top)
        check_grad(isr, torch, kind, dev, wide, scale, given, rng.normal(size=(rows, n)), rng.normal(size=rows) if case % 2 == 0 else None, r)


@pytest.mark.parametrize("kind", ["bf16", "i32"])
@pytest.mark.parametrize("rows,classes,top", [(1, 10, 10), (63, 10, 2), (4099, 10, 1), (1000, 101, 5), (203, 200, 128), (70, 257, 64), (300, 1000, 20), (301, 1000, 128), (17, 4096, 128)])
def test_many_rows(isr, torch, kind, rows, classes, top):
    rng = np.random.default_rng(rows)
    dev, wide = make(torch, kind, rows, classes, rows, pad=rows % 3)
    given = rng.integers(-1, classes, (rows, 2))
    r = check_logprobs(isr, torch, kind, dev, wide, scale_of(kind), given, top)
    check_grad(isr, torch, kind, dev, wide, scale_of(kind), given, rng.normal(size=(rows, 2)), rng.normal(size=rows), r)


@pytest.mark.parametrize("kind", ["f32", "f16"])
@pytest.mark.parametrize("classes", [5, 100, 256, 257, 3001, 20011])
@pytest.mark.parametrize("n", [64, 65, 128])
def test_many_given_classes_with_repetitions(isr, torch, kind, classes, n):
    """The given of up to 128, of few different classes, so that many name one; in place as well."""
    rng = np.random.default_rng(n)
    dev, wide = make(torch, kind, 3, classes, n, pad=1)
    some = rng.integers(0, classes, 20)
    given = np.where(rng.random((3, n)) < 0.1, -1, rng.choice(some, (3, n)))
    r = check_logprobs(isr, torch, kind, dev, wide, 1.0, given, 1)
    up = rng.normal(size=(3, n))
    check_grad(isr, torch, kind, dev, wide, 1.0, given, up, None, r)
    check_grad(isr, torch, kind, dev, wide, 1.0, given, up, up[:, 0], r, out=dev)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("classes", [10, 200, 5003, 50021])
def test_each_result_alone(isr, torch, kind, classes):
    dev, wide = make(torch, kind, 3, classes, classes, shift=1)
    scale, given = scale_of(kind), np.array([[1, -1], [0, 0], [classes - 1, 2]])
    g = torch.from_numpy(given.astype(np.int32)).cuda()
    lp, h, tc, tl = plain.logprobs(wide, scale, given, 9)
    a = isr.isr_logprobs(dev, g, scale=scale)
    assert a.entropy is a.top is a.top_class is a.stats is None
    close(a.given, lp, plain.logp_tol(lp), "given")
    b = isr.isr_logprobs(dev, entropy=True, scale=scale)
    assert b.given is None
    close(b.entropy, h, plain.U * plain.SUM * (3 + 2 * math.log(classes)), "entropy")
    c = isr.isr_logprobs(dev, top=9, scale=scale)
    close(c.top, tl, plain.logp_tol(tl), "top")
    assert np.array_equal(c.top_class.cpu().numpy(), tc)
    d = isr.isr_logprobs(dev, stats=True, scale=scale)
    up = np.ones((3, 2))
    check_grad(isr, torch, kind, dev, wide, scale, given, up, None, d)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("classes,top", [(16400, 128), (20011, 20), (40007, 64), (40007, 1)])
def test_top_alternatives_of_many_long_rows(isr, torch, kind, classes, top):
    """Rows that a workgroup goes through by chunks: ordinary ones, ascending ones (each chunk beats the last), descending, of few
    values, of one, with few possible classes, empty, with NaN; every row's classes against a stable sort."""
    rows = 1100
    gen = torch.Generator(device="cuda")
    gen.manual_seed(classes + top)
    x = torch.randn((rows, classes), generator=gen, device="cuda") * 3
    x[7] = x[7].sort().values
    x[8] = x[8].sort(descending=True).values
    x[9] = x[9].round()
    x[10] = 1.5
    x[11:40] += torch.linspace(0, 40, classes, device="cuda")
    x[40, classes // 2:] = 30
    if kind == "i32":
        x = (x * 1000).round().to(torch.int32)
        x[12] = torch.iinfo(torch.int32).min
    else:
        x[13] = -math.inf
        x[14, top // 2 + 1:] = -math.inf
        x[15, 5:classes - 3] = -math.inf
        x[16, classes - 1] = math.nan
        x = x.to(dtype_of(torch, kind))
    r = isr.isr_logprobs(x, top=top, entropy=True, scale=scale_of(kind))
    wide = x.double()
    value, index = torch.sort(wide, dim=1, descending=True, stable=True)
    index[value == -math.inf] = -1
    index = index[:, :top].to(torch.int32)
    if kind != "i32":
        index[16] = -1
    assert torch.equal(r.top_class, index)
    some = [0, 7, 8, 9, 10, 12, 13, 14, 15, 16, 17, 39, 40, rows - 1]
    _, h, _, tl = plain.logprobs(wide[some].cpu().numpy(), scale_of(kind), None, top)
    close(r.top[some], tl, plain.logp_tol(tl), "top log-probabilities")
    close(r.entropy[some], h, plain.U * plain.SUM * (3 + 2 * math.log(classes)), "entropy")


@pytest.mark.parametrize("kind,rows,classes,top", [("bf16", 515, 20011, 5), ("bf16", 300, 50021, 64), ("f16", 520, 32003, 128), ("f32", 600, 9001, 100),
                                                   ("i32", 270, 20011, 20), ("bf16", 1025, 17001, 0), ("f32", 1024, 8207, 0), ("bf16", 3, 70003, 0)])
def test_rows_by_chunks(isr, torch, kind, rows, classes, top):
    """More rows, or longer ones, than go by a workgroup each; the special rows among them."""
    rng = np.random.default_rng(classes)
    dev, wide = make(torch, kind, rows, classes, classes)
    special, special_wide = put(torch, kind, np.stack(list(special_rows(kind, classes, rng).values())[:rows]))
    dev[:len(special)] = special
    wide[:len(special)] = special_wide
    print(kind, rows, classes, top, flush=True)
    given = rng.integers(0, classes, (rows, 2))
    check_logprobs(isr, torch, kind, dev, wide, scale_of(kind), given, top)
    for rest in (False, True):
        check_distill(isr, torch, kind, dev, wide, scale_of(kind), make_teacher(torch, rng, rows, classes, 9, rest), 1.0, rest)


def test_more_rows_than_a_launch_takes(isr, torch):
    """Behind 2^22 workgroups the next launch goes on: rows on both sides against the same rows by themselves."""
    for classes, rows in ((260, (1 << 22) + 5), (1, (1 << 26) + 5)):
        print(classes, rows, flush=True)
        x = torch.randn((rows, classes), device="cuda", dtype=torch.bfloat16)
        e = torch.zeros((rows, 1), device="cuda", dtype=torch.int32)
        v = torch.full((rows, 1), -0.5, device="cuda")
        at = torch.tensor([0, 1, (1 << 22) - 1, 1 << 22, rows - 2, rows - 1])
        few = x[at].contiguous()
        r, s = (isr.isr_logprobs(z, e[:len(z)], top=1, entropy=True, stats=True) for z in (x, few))
        d, f = (isr.isr_distill(z, e[:len(z)], v[:len(z)], rest=True, grad=True) for z in (x, few))
        g, h = (isr.isr_logprobs_grad(z, e[:len(z)], v[:len(z)], q.stats) for z, q in ((x, r), (few, s)))
        for big, small in zip([*r, d.loss, d.grad, g], [*s, f.loss, f.grad, h]):
            assert torch.equal(big[at], small)
        assert bool((r.top_class >= 0).all()) and bool(torch.isfinite(r.given).all()) and bool(torch.isfinite(d.loss).all() or classes == 1)


def special_rows(kind, classes, rng):
    """Rows that a mask or a broken model leaves, name by name."""
    big = {"f32": np.finfo(np.float32).max, "bf16": 2.0 ** 127 * (2 - 2.0 ** -7), "f16": 65504.0, "i32": 2.0 ** 31 - 1}[kind]
    low = -big - (1 if kind == "i32" else 0)
    x = np.round(rng.normal(size=classes) * 3 * (1000 if kind == "i32" else 1), 2 if kind != "i32" else 0)
    rows = {"equal": np.zeros(classes), "two values": np.where(rng.random(classes) < 0.5, 1.0, 2.0), "lowest": np.full(classes, low),
            "lowest but one": np.where(np.arange(classes) == classes // 2, 1.0, low), "both ends": np.where(np.arange(classes) % 2 == 0, big, low),
            "ascending": np.sort(x), "descending": -np.sort(-x), "far off": np.round(x) + (2.0 ** 20 if kind in ("f32", "i32") else 100),
            "first": np.where(np.arange(classes) == 0, 50.0, 0.0), "last": np.where(np.arange(classes) == classes - 1, 50.0, 0.0)}
    if kind != "i32":
        inf = np.inf
        rows |= {"empty": np.full(classes, -inf), "one possible": np.where(np.arange(classes) == classes * 2 // 3, x, -inf),
                 "half possible": np.where(rng.random(classes) < 0.5, x, -inf), "a run possible": np.where((np.arange(classes) >= classes // 3) & (np.arange(classes) < classes // 3 + 70), x, -inf),
                 "nan": np.where(np.arange(classes) == classes // 2, np.nan, x), "all nan": np.full(classes, np.nan),
                 "nan beside impossible": np.where(np.arange(classes) == classes - 1, np.nan, -inf),
                 "infinite": np.where(np.arange(classes) == classes - 1, inf, x), "zeros of both signs": np.where(rng.random(classes) < 0.5, -0.0, 0.0)}
    return rows


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("classes", [2, 10, 101, 256, 300, 1000, 2500, 20011, 70001])
def test_masked_tied_and_extreme_rows(isr, torch, kind, classes):
    rng = np.random.default_rng(classes)
    named = special_rows(kind, classes, rng)
    x = np.stack(list(named.values()))
    dev, wide = put(torch, kind, x, pad=1)
    rows = len(x)
    for top in sorted({1, min(20, classes), min(128, classes)}):
        print(kind, classes, top, list(named), flush=True)
        scale = scale_of(kind)
        given = np.stack([np.full(rows, classes // 2), np.full(rows, classes * 2 // 3), np.full(rows, -1), np.full(rows, classes), np.full(rows, classes // 2)], 1)
        check_logprobs(isr, torch, kind, dev, wide, scale, given, top)
    given = given[:, [0, 1, 2, 4]]   # without the class outside, which makes the whole row NaN
    r = check_logprobs(isr, torch, kind, dev, wide, scale, given, 1)
    up, up_h = rng.normal(size=(rows, 4)), rng.normal(size=rows)
    check_grad(isr, torch, kind, dev, wide, scale, given, up, up_h, r)
    check_grad(isr, torch, kind, dev, wide, scale, given, up, None, r)
    given[:] = -1   # rows that do not count: zeros whatever they hold
    check_grad(isr, torch, kind, dev, wide, scale, given, up, None, r)
    check_grad(isr, torch, kind, dev, wide, scale, given, up, np.where(np.arange(rows) % 2 == 0, 0.0, up_h), r)
    given[:, 0] = classes
    check_grad(isr, torch, kind, dev, wide, scale, given, up, None, r)


def test_a_class_outside_makes_the_gradient_nan_and_no_more(isr, torch):
    dev, wide = make(torch, "f32", 4, 50, 1)
    given = np.array([[3], [50], [2 ** 31 - 1], [-5]])
    r = check_logprobs(isr, torch, "f32", dev, wide, 1.0, given, 2)
    got = check_grad(isr, torch, "f32", dev, wide, 1.0, given, np.ones((4, 1)), None, r)
    assert torch.isnan(got[1:3]).all() and not torch.isnan(got[0]).any() and (got[3] == 0).all()


def make_teacher(torch, rng, rows, classes, top, rest, ragged=True, dup=False, kind="f32"):
    entry = np.stack([rng.permutation(classes)[:top] if classes < 5000 else rng.choice(classes, top, replace=False) for _ in range(rows)])
    value = rng.normal(size=(rows, top)) * 2
    value = value - np.log(np.exp(value).sum(1, keepdims=True)) + np.log(1 - 0.3 * rng.random((rows, 1))) if rest else value * 3 + 20
    if ragged:
        entry[rng.random(entry.shape) < 0.2] = -1
        entry[rng.random(rows) < 0.1] = -1
    if dup and top > 2:
        entry[:, top // 2] = entry[:, 0]
    v = torch.from_numpy(value).to(dtype_of(torch, kind))
    return entry, v.double().numpy(), torch.from_numpy(entry.astype(np.int32)).cuda(), v.cuda()


def check_distill(isr, torch, kind, dev, wide, scale, teacher, vs, rest, weight=None, in_place=False):
    entry, value, e, v = teacher
    w = None if weight is None else torch.from_numpy(weight.astype(np.float32)).cuda()
    loss, ltol, g, gtol = plain.distill(wide, scale, entry, value, vs, rest, None if weight is None else weight.astype(np.float32).astype(np.float64))
    gtol = grad_tol(kind, g, gtol)
    a = isr.isr_distill(dev, e, v, rest=rest, scale=scale, teacher_scale=vs, stats=True)
    close(a.loss, loss, ltol, "loss alone")
    assert a.grad is None
    b = isr.isr_distill_grad(dev, e, v, a.stats, weight=w, rest=rest, scale=scale, teacher_scale=vs)
    close(b, g, gtol, "gradient alone")
    c = isr.isr_distill(dev, e, v, weight=w, rest=rest, scale=scale, teacher_scale=vs, grad=True)
    close(c.loss, loss, ltol, "loss with gradient")
    close(c.grad, g, gtol, "gradient with loss")
    if in_place and kind != "i32":
        copy = dev.clone()   # dense: its rows start elsewhere, where the sums' terms are grouped in another way, within the same bounds
        d = isr.isr_distill(copy, e, v, weight=w, rest=rest, scale=scale, teacher_scale=vs, grad=copy)
        assert d.grad.data_ptr() == copy.data_ptr()
        close(d.loss, loss, ltol, "loss with gradient in place")
        close(copy, g, gtol, "gradient in place")
        same = torch.empty_strided(dev.shape, dev.stride(), dtype=dev.dtype, device="cuda") if dev.data_ptr() % 16 == 0 else None
        if same is not None:   # rows that lie alike: bit by bit
            same.copy_(dev)
            d = isr.isr_distill(same, e, v, weight=w, rest=rest, scale=scale, teacher_scale=vs, grad=same)
            assert torch.equal(same.nan_to_num(7.0), c.grad.nan_to_num(7.0)) and torch.equal(d.loss.nan_to_num(7.0), c.loss.nan_to_num(7.0))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("classes", CLASSES[1:])
def test_distillation(isr, torch, kind, rest, classes):
    rng = np.random.default_rng(classes + rest)
    for case, (rows, pad, shift, top, s, vs) in enumerate(((3, 0, 0, 4, 1.0, 1.0), (6, 5, 3, 20, 0.5, 1.0), (2, 2, 1, 128, 2.0, 0.75))):
        if classes > 20000 and case == 1:
            continue
        top = min(top, classes)
        print(kind, rest, classes, case, flush=True)
        dev, wide = make(torch, kind, rows, classes, classes + case, pad, shift)
        teacher = make_teacher(torch, rng, rows, classes, top, rest, dup=case == 1, kind=("f32", "bf16", "f16")[case])
        check_distill(isr, torch, kind, dev, wide, scale_of(kind, s), teacher, vs if not rest else 1.0, rest, rng.normal(size=rows) if case else None, in_place=case < 2)


@pytest.mark.parametrize("kind", ["f32", "f16"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,classes,top", [(4099, 10, 3), (1000, 101, 10), (300, 1000, 20), (65, 5003, 64)])
def test_distillation_of_many_rows(isr, torch, kind, rest, rows, classes, top):
    rng = np.random.default_rng(rows)
    dev, wide = make(torch, kind, rows, classes, rows, pad=rows % 3)
    check_distill(isr, torch, kind, dev, wide, 1.0, make_teacher(torch, rng, rows, classes, top, rest), 1.0, rest, rng.random(rows), in_place=True)


@pytest.mark.parametrize("kind", ["f32", "bf16", "i32"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("classes", [10, 101, 300, 1030, 5000, 20011, 70001])
def test_distillation_of_special_rows(isr, torch, kind, rest, classes):
    rng = np.random.default_rng(classes)
    named = special_rows(kind, classes, rng)
    x = np.stack(list(named.values()))
    dev, wide = put(torch, kind, x)
    rows, top = len(x), min(classes, 9)
    print(kind, rest, classes, list(named), flush=True)
    for absent in (False, True):
        entry, value, e, v = make_teacher(torch, rng, rows, classes, top, rest, ragged=False)
        if absent:
            entry[:] = -1
            e.fill_(-1)
        weight = rng.normal(size=rows)
        weight[::3] = 0
        check_distill(isr, torch, kind, dev, wide, scale_of(kind), (entry, value, e, v), 1.0, rest, weight, in_place=True)


@pytest.mark.parametrize("rest", [False, True])
def test_special_teachers(isr, torch, rest):
    """Values of minus infinity (no share), all of them so, NaN, infinity, more than all of the probability, a class outside,
    entries that cover every class, one class named by all entries."""
    inf, classes, top = np.inf, 6, 6
    rng = np.random.default_rng(5)
    entry = np.tile(np.arange(6), (8, 1))
    value = np.log(np.tile([0.1, 0.2, 0.1, 0.1, 0.2, 0.2], (8, 1)))
    value[0, 2:4] = -inf
    value[1] = -inf
    value[2, 1] = np.nan
    value[3, 1] = inf
    value[4] += 0.3
    entry[5, 3] = 6
    entry[7] = 2
    entry[0, 5] = -1
    for kind in ("f32", "bf16"):
        dev, wide = make(torch, kind, 8, classes, 3)
        teacher = (entry, torch.from_numpy(value).float().double().numpy(), torch.from_numpy(entry.astype(np.int32)).cuda(), torch.from_numpy(value).float().cuda())
        check_distill(isr, torch, kind, dev, wide, 1.0, teacher, 1.0, rest, rng.normal(size=8), in_place=True)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("classes", [6, 40, 300, 5000])
def test_bad_teachers_of_empty_rows(isr, torch, rest, classes):
    """A class outside or a NaN value makes all of a row's results NaN, of an empty row too; a weight of 0 its gradient 0."""
    entry = np.tile(np.arange(3), (5, 1))
    entry[0, 1] = classes
    value = np.log(np.tile([0.1, 0.2, 0.3], (5, 1)))
    value[1, 2] = np.nan
    value[3, 0] = np.nan
    dev, wide = put(torch, "f32", np.full((5, classes), -np.inf))
    teacher = (entry, torch.from_numpy(value).float().double().numpy(), torch.from_numpy(entry.astype(np.int32)).cuda(), torch.from_numpy(value).float().cuda())
    check_distill(isr, torch, "f32", dev, wide, 1.0, teacher, 1.0, rest, np.array([1.0, -2.0, 1.0, 0.0, 3.0]), in_place=True)


def test_more_rows_of_one_wave_or_workgroup_than_a_launch_takes(isr, torch):
    """As above, for log-probabilities by a wave and by a workgroup a row."""
    for classes, rows, top in ((257, (1 << 24) + 5, 1), (1025, (1 << 22) + 5, 2)):
        print(classes, rows, flush=True)
        x = torch.empty((rows, classes), device="cuda", dtype=torch.bfloat16).uniform_(-4, 0)
        x[:, 0] = 1
        x[:, 1] = 2
        g = torch.ones((rows, 1), device="cuda", dtype=torch.int32)
        at = torch.tensor([0, 1, (1 << 22) - 1, 1 << 22, (1 << 22) + 1, rows - 6, rows - 5, rows - 2, rows - 1])
        few = x[at].contiguous()
        r, s = (isr.isr_logprobs(z, g[:len(z)], top=top, entropy=True, stats=True) for z in (x, few))
        _, h, tc, tl = plain.logprobs(few.double().cpu().numpy(), 1.0, None, top)
        for q, of in ((r, at), (s, slice(None))):
            assert np.array_equal(q.top_class[of].cpu().numpy(), tc)
            close(q.top[of], tl, plain.logp_tol(tl), "top log-probabilities")
            close(q.entropy[of], h, plain.U * plain.SUM * (3 + 2 * math.log(classes)), "entropy")


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_gradient_over_the_logits_and_foreign_memory(isr, torch, kind):
    """In place, with foreign columns; and into rows of another stride: what lies between and behind the rows stays."""
    for classes, rows in ((10, 9), (101, 4), (2500, 3), (20011, 2)):
        dev, wide = make(torch, kind, rows, classes, classes, pad=5, shift=3)
        rng = np.random.default_rng(classes)
        given = rng.integers(0, classes, (rows, 2))
        up = rng.normal(size=(rows, 2))
        r = check_logprobs(isr, torch, kind, dev, wide, 1.0, given, 2)
        wide_out = torch.full((rows + 2, classes + 7), 42.0, dtype=dev.dtype, device="cuda")
        out = wide_out[1:-1, 2:2 + classes]
        got = check_grad(isr, torch, kind, dev, wide, 1.0, given, up, up[:, 0], r, out=out)
        assert got.data_ptr() == out.data_ptr()
        keep = torch.ones_like(wide_out, dtype=torch.bool)
        keep[1:-1, 2:2 + classes] = False
        assert (wide_out[keep] == 42).all()
        want = got.clone()
        base = dev._base if dev._base is not None else dev
        before = base.clone()
        check_grad(isr, torch, kind, dev, wide, 1.0, given, up, up[:, 0], r, out=dev)
        assert torch.equal(dev, want)
        flat, old = base.flatten(), before.flatten()
        touched = torch.zeros_like(flat, dtype=torch.bool)
        touched[3:3 + rows * (classes + 5)].view(rows, classes + 5)[:, :classes] = True
        assert torch.equal(flat[~touched], old[~touched])


def test_rows_beyond_32_bits_of_elements(isr, torch):
    stride, classes = (1 << 31) + 8, 1000
    flat = torch.empty(2 * stride + classes, dtype=torch.bfloat16, device="cuda")
    dev = flat.as_strided((3, classes), (stride, 1))
    src, wide = make(torch, "bf16", 3, classes, 9)
    dev.copy_(src)
    rng = np.random.default_rng(1)
    given = rng.integers(0, classes, (3, 1))
    r = check_logprobs(isr, torch, "bf16", dev, wide, 1.0, given, 20)
    check_grad(isr, torch, "bf16", dev, wide, 1.0, given, rng.normal(size=(3, 1)), None, r, out=dev)
    dev.copy_(src)
    e, v = make_teacher(torch, rng, 3, classes, 8, True, ragged=False)[2:]
    a, b = isr.isr_distill(dev, e, v, rest=True, grad=dev), isr.isr_distill(src, e, v, rest=True, grad=True)
    assert torch.equal(a.loss, b.loss) and torch.equal(dev, b.grad)


def test_no_rows(isr, torch):
    x = torch.empty((0, 10), device="cuda")
    r = isr.isr_logprobs(x, torch.empty((0, 1), dtype=torch.int32, device="cuda"), top=3, entropy=True, stats=True)
    assert r.given.shape == (0, 1) and r.top.shape == (0, 3)
    d = isr.isr_distill(x, torch.empty((0, 2), dtype=torch.int32, device="cuda"), torch.empty((0, 2), device="cuda"), grad=True, stats=True)
    assert d.loss.shape == (0,) and d.grad.shape == (0, 10)


def test_operands_that_do_not_fit_are_refused(isr, torch):
    x = torch.zeros((4, 10), device="cuda")
    i32, f32 = torch.int32, torch.float32
    given = torch.zeros((4, 1), dtype=i32, device="cuda")
    up, stats, h = torch.zeros((4, 1), device="cuda"), torch.zeros((4, 2), device="cuda"), torch.zeros(4, device="cuda")
    e, v = torch.zeros((4, 2), dtype=i32, device="cuda"), torch.zeros((4, 2), device="cuda")
    calls = [lambda: isr.isr_logprobs(x, given.long()), lambda: isr.isr_logprobs(x, given[:3]), lambda: isr.isr_logprobs(x, given.cpu()),
             lambda: isr.isr_logprobs(x, given[:, 0]), lambda: isr.isr_logprobs(x.t(), top=1), lambda: isr.isr_logprobs(x[0], top=1), lambda: isr.isr_logprobs(x),
             lambda: isr.isr_logprobs(x, top=11), lambda: isr.isr_logprobs(x, top=-1), lambda: isr.isr_logprobs(x.double(), top=1), lambda: isr.isr_logprobs(x, top=1, scale=0.0),
             lambda: isr.isr_logprobs(x[:1].expand(4, 10), top=1), lambda: isr.isr_logprobs(x[:, :0], entropy=True),
             lambda: isr.isr_logprobs_grad(x, given, up.half(), stats), lambda: isr.isr_logprobs_grad(x, given, up, stats[:3]),
             lambda: isr.isr_logprobs_grad(x, given, up, stats, grad_entropy=h), lambda: isr.isr_logprobs_grad(x, given, up, stats, out=x.half()),
             lambda: isr.isr_logprobs_grad(x, given, up, stats, out=x[:3]), lambda: isr.isr_logprobs_grad(x, given, up, torch.zeros((4, 4), device="cuda")[:, ::2]),
             lambda: isr.isr_distill(x, e, v[:3]), lambda: isr.isr_distill(x, e.long(), v), lambda: isr.isr_distill(x, e, v.double()),
             lambda: isr.isr_distill(x, e[:, :0].contiguous(), v[:, :0].contiguous()), lambda: isr.isr_distill(x, e, v, weight=h[:2]),
             lambda: isr.isr_distill(x, e, v, grad=x.t()), lambda: isr.isr_distill_grad(x, e, v, stats)]
    for i, call in enumerate(calls):
        with pytest.raises(isr.IsrError) as err:
            call()
        assert err.value.status == isr.ISR_ERR_ARG, i
    assert (x == 0).all()


@pytest.mark.parametrize("classes,rows", [(10, 33), (101, 5), (5003, 3), (70001, 2)])
def test_other_streams_and_captured_calls(isr, torch, classes, rows):
    """Two streams at once, then one graph that holds all operators: each replay, on new inputs and with eager work between,
    gives what eager calls give, bit by bit."""
    rng = np.random.default_rng(classes)
    xs = [make(torch, "bf16", rows, classes, s)[0].contiguous() for s in range(4)]
    given = torch.from_numpy(rng.integers(-1, classes, (rows, 2)).astype(np.int32)).cuda()
    up, up_h = torch.randn((rows, 2), device="cuda"), torch.randn(rows, device="cuda")
    e, v = make_teacher(torch, rng, rows, classes, min(20, classes), True)[2:]

    def step(x):
        r = isr.isr_logprobs(x, given, top=min(7, classes), entropy=True, stats=True)
        g = isr.isr_logprobs_grad(x, given, up, r.stats, entropy=r.entropy, grad_entropy=up_h)
        d = isr.isr_distill(x, e, v, rest=True, stats=True)
        f = isr.isr_distill(x, e, v, weight=up_h, rest=True, grad=True)
        return [*r, g, d.loss, d.stats, isr.isr_distill_grad(x, e, v, d.stats, weight=up_h, rest=True), f.loss, f.grad]

    want = [step(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = []
    for x, st in zip(xs, streams):
        with torch.cuda.stream(st):
            got.append(step(x))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(i, j) for i, j in zip(a, b))
    x = xs[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(x)
    for k in (1, 2, 3, 0, 2):
        x.copy_(xs[k])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(i, j) for i, j in zip(held, want[k])), k
        assert all(torch.equal(i, j) for i, j in zip(step(xs[k]), want[k])), k


def test_c_calls_with_memory_of_the_caller(isr, torch):
    """The C entry points themselves: a workspace of exactly the size asked for, nothing written beside it or behind the results."""
    rows, classes, top = 5, 40009, 20
    dev, wide = make(torch, "f16", rows, classes, 4)
    L, x = isr.lib(), isr.Logits(dev.data_ptr(), isr.F16, classes, rows, dev.stride(0), 1.0)
    need = L.isr_logprobs_workspace_bytes(C.byref(x), top)
    ws = torch.full((need + 512,), 77, dtype=torch.uint8, device="cuda")
    at = (-ws.data_ptr()) % 256
    tc, tl = torch.full((rows + 1, top), 7, dtype=torch.int32, device="cuda"), torch.full((rows + 1, top), 7.0, device="cuda")
    assert L.isr_logprobs(C.byref(x), None, 0, top, None, None, tc.data_ptr(), tl.data_ptr(), None, ws.data_ptr() + at, need, None) == isr.ISR_OK
    torch.cuda.synchronize()
    _, _, want, want_l = plain.logprobs(wide, 1.0, None, top)
    assert np.array_equal(tc[:-1].cpu().numpy(), want) and (tc[-1] == 7).all() and (tl[-1] == 7).all()
    close(tl[:-1], want_l, plain.logp_tol(want_l), "top")
    assert (ws[:at] == 77).all() and (ws[at + need:] == 77).all()


def test_teacher_to_student_on_the_networks(isr, torch):
    """As they are used together: the fp32 network's logits of noisy copies become the teacher's stored top logits, the int8
    network's logits of the same network are the student's; a descent on float copies of the student's logits along the
    gradient lowers the loss by what the gradient says."""
    import synth
    m = isr.isr_load_model(synth.build_model(1))
    isr.isr_set_workspace(m, 512, float_fp=True)
    x = synth.make_image(1, 3)
    n = 64
    teacher = torch.from_numpy(isr.isr_float_debug_forward(m, x, 16.0, 5, 0, 0, 0, n, isr.FLOATRS_FP)[0]).cuda()
    student = torch.from_numpy(isr.isr_debug_forward(m, x, 16, 5, 0, 0, 0, n)[0]).cuda()
    assert student.dtype == torch.int32 and teacher.dtype == torch.float32
    scale = 4.0 / float(teacher.std())
    stored = isr.isr_logprobs(teacher, top=4, entropy=True, scale=scale)
    loss, ltol, g, gtol = plain.distill(student.cpu().numpy().astype(np.float64), np.float32(scale), stored.top_class.cpu().numpy(),
                                        stored.top.double().cpu().numpy(), 1.0, True)
    d = isr.isr_distill(student, stored.top_class, stored.top, rest=True, scale=scale, grad=True)
    close(d.loss, loss, ltol, "loss")
    close(d.grad, g, grad_tol("i32", g, gtol), "gradient")
    # by differences, in the operator's own arithmetic: the loss along the gradient
    s = student.float()
    step = 1e-2 / scale / float(d.grad.double().norm(dim=1).max() / scale)
    moved = [isr.isr_distill(s + k * step * d.grad / scale, stored.top_class, stored.top, rest=True, scale=scale).loss.double() for k in (1, -1)]
    slope = (moved[0] - moved[1]) / (2 * step / scale)
    want = (d.grad.double() ** 2).sum(1)
    assert torch.allclose(slope, want, rtol=2e-2, atol=1e-2 * float(want.max()) + 1e-12)
    # what the two say of the label they were certified for
    lab = stored.top_class[:, :1].contiguous()
    a, b = isr.isr_logprobs(teacher, lab, scale=scale).given, isr.isr_logprobs(student, lab, scale=scale).given
    assert torch.equal(a[:, 0], stored.top[:, 0]) and torch.isfinite(b).all()
    m.close()
