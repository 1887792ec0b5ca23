"""Operators on rows of class logits at the ends of their ranges: teachers that leave nothing to a rest class, sums over many chunks,
log-probabilities next to the largest number, shares of the teacher next to zero, and workspaces of a larger call."""
import ctypes as C
import math

import numpy as np
import pytest

import logit_rows_plain as plain
from test_gpu_logit_rows import TYPES, check_logprobs, close, dtype_of, grad_tol, isr, make, put, scale_of, torch  # noqa: F401

pytestmark = pytest.mark.gpu
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}   # half a step, relative
LOWEST = {"f32": -float(np.finfo(np.float32).max), "bf16": -2.0 ** 127 * (2 - 2.0 ** -7), "f16": -65504.0, "i32": -2.0 ** 31}


def rest_rounding(v, top, kind, value_scale=1.0):
    """How far 1 - sum exp v may lie from 0 by the rounding of v alone, as isr.h has it."""
    e = -(np.exp(v) * v).sum()
    return HALF[kind] * (e + value_scale * 2.0 ** -14) + 2.0 ** -24 * (top + 16 + 4 * e)


def possible_rows(torch, kind, rows, classes, possible, mask, seed):
    """Rows of which `possible` classes are ordinary and the others hold `mask`."""
    dev, wide = make(torch, kind, rows, classes, seed)
    rng = np.random.default_rng(seed)
    for r in range(rows):
        out = rng.permutation(classes)[possible:]
        wide[r, out] = mask
    return put(torch, kind, wide, pad=seed % 3)


NOTHING_LEFT = [(kind, classes, classes, None) for kind in TYPES for classes in (1, 2, 10, 101, 128)] + [
    (kind, classes, possible, mask) for kind, mask in (("f32", "-inf"), ("f32", "lowest"), ("f32", "-1e9"), ("bf16", "-inf"), ("bf16", "lowest"), ("f16", "-inf"), ("f16", "lowest"), ("i32", "lowest"))
    for classes, possible in ((10, 4), (200, 20), (300, 20), (1000, 20), (5003, 100), (20011, 20), (70001, 20))]


@pytest.mark.parametrize("stored_as", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind,classes,possible,mask", NOTHING_LEFT)
def test_teachers_that_leave_nothing_to_the_rest(isr, torch, kind, classes, possible, mask, stored_as):
    """A row's own stored log-probabilities of all its possible classes: they add up to 1 but for their rounding, so the rest class
    has no share, and loss and gradient are those of the entries alone, whichever call makes them."""
    rows, scale = 24, scale_of(kind)
    low = LOWEST[kind] if mask == "lowest" else float(mask) if mask else 0.0
    dev, wide = possible_rows(torch, kind, rows, classes, possible, low, classes)
    top = min(classes, 128, possible + (3 if mask == "-inf" else 0))
    print(kind, classes, possible, mask, stored_as, flush=True)
    stored = isr.isr_logprobs(dev, top=top, scale=scale)
    value = stored.top.to(dtype_of(torch, stored_as))
    entry, v = stored.top_class.cpu().numpy(), value.double().cpu().numpy()
    for r in range(rows):
        there = entry[r] >= 0
        assert there.sum() == possible and abs(1 - np.exp(v[r][there]).sum()) <= rest_rounding(v[r][there], top, stored_as)
    check_rest(isr, torch, kind, dev, wide, scale, stored.top_class, value, True)
    # a share that is more than rounding stays: a student without a class for it is infinitely far off
    check_rest(isr, torch, kind, dev, wide, scale, stored.top_class, (value.float() - 0.1).to(value.dtype), False)


def check_rest(isr, torch, kind, dev, wide, scale, cls, value, nothing):
    """Loss and gradient, together and one after the other, of rows whose possible classes are all entries.  The others are all
    alike, so each has its part of the rest class."""
    entry, v = cls.cpu().numpy(), value.double().cpu().numpy()
    rows, classes = wide.shape
    loss, ltol, g, gtol = np.zeros(rows), np.zeros(rows), np.zeros((rows, classes)), np.zeros((rows, classes))
    for r in range(rows):
        there = entry[r] >= 0
        c, w = entry[r][there], v[r][there]
        logp, q = plain.row_logp(wide[r], scale)[0], np.exp(w)
        left = 0.0 if nothing else 1 - q.sum()
        other = np.ones(classes, dtype=bool)
        other[c] = False
        loss[r] = (q * (w - logp[c])).sum()
        ltol[r] = (q * (2 * plain.logp_tol(logp[c]) + plain.U * (8 * np.abs(w) + 8))).sum()
        if left > 0:
            lr = logp[other].max() + math.log(other.sum()) if other.any() else -np.inf
            loss[r] += left * (math.log(left) - lr)
            ltol[r] += left * (2 * plain.logp_tol(lr) + plain.U * (8 * abs(math.log(left)) + 8))
        ltol[r] += 4 * plain.U * abs(loss[r])
        p, total = np.exp(logp[c]), q.sum() + left
        g[r, c] = total * p - q
        gtol[r, c] = plain.U * (total * p * (plain.SUM + 4 * np.abs(logp[c])) + q * (16 + 4 * np.abs(w)) + 4 * np.abs(g[r, c]))
        if left > 0 and np.isfinite(wide[r, other]).all():
            g[r, other] = -left / max(1, other.sum())
            gtol[r, other] = plain.U * (plain.SUM + 8) * np.abs(g[r, other])
    g, gtol = scale * g, grad_tol(kind, scale * g, scale * gtol)
    a = isr.isr_distill(dev, cls, value, rest=True, scale=scale, stats=True)
    b = isr.isr_distill(dev, cls, value, rest=True, scale=scale, grad=True)
    close(a.loss, loss, ltol, "loss alone")
    close(b.loss, loss, ltol, "loss with gradient")
    close(b.grad, g, gtol, "gradient with loss")
    close(isr.isr_distill_grad(dev, cls, value, a.stats, rest=True, scale=scale), g, gtol, "gradient alone")


@pytest.mark.parametrize("classes,named", [(4, 4), (40, 4), (300, 4), (5000, 4)])
def test_the_least_share_of_a_rest_class(isr, torch, classes, named):
    """On both sides of the rounding that counts as nothing; a teacher's scale of 0.25 takes the values themselves four times as far."""
    bound = rest_rounding(np.full(named, -math.log(named)), named, "f32", 0.25)
    x = np.full((4, classes), -np.inf)
    x[:, :named] = 0
    dev, wide = put(torch, "f32", x)
    e = torch.arange(named, dtype=torch.int32, device="cuda").repeat(4, 1)
    left = np.array([-0.5, 0.25, 0.75, 1.5]) * bound
    v = (4 * (-math.log(named) + np.log1p(-left)))[:, None].repeat(named, 1)
    v32 = torch.from_numpy(v).float().cuda()
    d = isr.isr_distill(dev, e, v32, rest=True, teacher_scale=0.25, grad=True)
    assert torch.isfinite(d.loss[:3]).all() and (d.loss[:3].abs() <= 2 * bound).all()
    assert d.loss[3] == math.inf and torch.isfinite(d.grad).all()


@pytest.mark.parametrize("kind,classes", [("bf16", 262144), ("i32", 300007), ("f16", 1 << 22)])
def test_one_class_above_a_long_flat_tail(isr, torch, kind, classes):
    """Terms far smaller than the largest, many of them: a row of one class 15 to 17 above all others, in its first chunk, in the
    middle, in its last.  More rows than go by chunks, so a workgroup goes through its row and adds up all of it."""
    rows, unit = 1030, 1000 if kind == "i32" else 1
    scale = 1.0 / unit
    x = torch.zeros((rows, classes), dtype=dtype_of(torch, kind), device="cuda")
    at = [0, 1, 255, 256 * 8, classes // 2, classes - 3000, classes - 1, classes - 8]
    some = list(range(len(at))) + [rows - 1]
    for r, j in enumerate(at + [77]):
        x[some[r], j] = (15 + r % 3) * unit
    print(kind, classes, flush=True)
    given = torch.tensor((at + [77]), dtype=torch.int32, device="cuda")
    all_given = torch.zeros((rows, 2), dtype=torch.int32, device="cuda")
    all_given[some, 0] = given
    all_given[some, 1] = (given + 5) % classes
    r = isr.isr_logprobs(x, all_given, top=2, entropy=True, scale=scale, stats=True)
    # by hand: one class of l, classes - 1 of 0
    l = np.array([15 + k % 3 for k in range(len(some))], dtype=np.float64)
    logz = np.log1p((classes - 1) * np.exp(-l))
    want = np.stack([-logz, -l - logz], 1)
    close(r.given[some], want, plain.logp_tol(want), "given")
    close(r.top[some], want, plain.logp_tol(want), "top")
    p = np.exp(want)
    h = -p[:, 0] * want[:, 0] - (classes - 1) * p[:, 1] * want[:, 1]
    close(r.entropy[some], h, plain.U * plain.SUM * (3 + 2 * math.log(classes)), "entropy")
    close(r.stats[some, 1], logz, plain.logp_tol(logz), "statistics")


def test_a_row_that_rises_chunk_by_chunk(isr, torch):
    """Each chunk's largest a little above the last one's: the sum is referred to another maximum every time, and most of it is old."""
    rows, classes = 1024, 1 << 20
    x = torch.empty((rows, classes), device="cuda")
    x[:] = torch.linspace(0, 0.5, classes, device="cuda")
    r = isr.isr_logprobs(x, top=1, entropy=True)
    lp, h, tc, tl = plain.logprobs(x[:1].double().cpu().numpy(), 1.0, None, 1)
    assert (r.top_class == int(tc[0, 0])).all()
    for k in (0, rows - 1):
        close(r.top[k:k + 1], tl, plain.logp_tol(tl), "top")
        close(r.entropy[k:k + 1], h, plain.U * plain.SUM * (3 + 2 * math.log(classes)), "entropy")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes", [(3, 10), (3, 200), (5, 300), (3, 3001), (3, 20011), (3, 140001), (1100, 20011)])
def test_log_probabilities_further_down_than_logits_differ(isr, torch, kind, rows, classes):
    """Logits of both ends of the type: their difference has no number, the log-probability at a scale below one half has."""
    x = np.zeros((rows, classes))
    x[:, classes // 2] = 3e38
    x[:, 1] = -3e38
    x[:, classes - 1] = -2e38
    x[1] = np.where(np.arange(classes) % 2, 3e38, -3e38)
    x[2, :] = -np.inf
    x[2, [0, 3]] = 3e38, -3e38
    dev, wide = put(torch, kind, x, pad=1)
    given = np.tile(np.array([1, classes - 1, classes // 2, 3]), (rows, 1))
    print(kind, rows, classes, flush=True)
    for scale in (0.5, 0.25, 2.0 ** -20, 1e-30):
        check_logprobs(isr, torch, kind, dev, wide, float(np.float32(scale)), given, min(classes, 6))


@pytest.mark.parametrize("kind,classes,top", [("bf16", 32000, 20), ("bf16", 131072, 20), ("f32", 20011, 3), ("bf16", 50021, 64)])
def test_a_workspace_serves_all_smaller_batches(isr, torch, kind, classes, top):
    """Of the size asked for 2048 rows once, for calls of fewer, with other memory behind it."""
    L = isr.lib()
    most = 2048
    x = torch.randn((most, classes), device="cuda").to(dtype_of(torch, kind))
    at = {"f32": isr.F32, "bf16": isr.BF16}[kind]
    size = L.isr_logprobs_workspace_bytes(C.byref(isr.Logits(x.data_ptr(), at, classes, most, classes, 1.0)), top)
    ws = torch.full((size + 256,), 77, dtype=torch.uint8, device="cuda")
    want = isr.isr_logprobs(x, top=top)
    for rows in (most, 1024, 1023, 700, 600, 513, 512, 257, 256, 129, 65, 64, 33, 32, 1):
        tc, tl = torch.empty((rows, top), dtype=torch.int32, device="cuda"), torch.empty((rows, top), device="cuda")
        l = isr.Logits(x.data_ptr(), at, classes, rows, classes, 1.0)
        assert L.isr_logprobs(C.byref(l), None, 0, top, None, None, tc.data_ptr(), tl.data_ptr(), None, ws.data_ptr(), size, None) == isr.ISR_OK, rows
        torch.cuda.synchronize()
        assert torch.equal(tc, want.top_class[:rows]), rows
    assert (ws[size:] == 77).all()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("kind", ["f32", "i32"])
@pytest.mark.parametrize("classes", [10, 101, 200, 300, 3001, 20011, 70001])
def test_small_shares_of_the_teacher(isr, torch, kind, classes, rest):
    """A class that the student all but excludes has the teacher's share as its gradient: the same bits from the call that makes the
    loss as from the statistics, and with the rest class (where a share is the exponential of what is stored) to the last places."""
    rows, scale = 3, scale_of(kind)
    x = np.zeros((rows, classes))
    x[:, 2:5] = -200 / scale
    dev, _ = put(torch, kind, x, pad=1)
    e = torch.tensor([[1, 2, 3, 4]], dtype=torch.int32, device="cuda").repeat(rows, 1)
    v = torch.tensor([[-0.02, -80.1, -33.7, -7.123], [-0.1, -50.3, -61.7, -20.9], [-0.05, -77.77, -3.3, -11.1]], device="cuda")
    weight = torch.tensor([1.0, 2.0, 0.5], device="cuda")
    a = isr.isr_distill(dev, e, v, weight=weight, rest=rest, scale=scale, teacher_scale=0.99, stats=True)
    b = isr.isr_distill(dev, e, v, weight=weight, rest=rest, scale=scale, teacher_scale=0.99, grad=True)
    c = isr.isr_distill_grad(dev, e, v, a.stats, weight=weight, rest=rest, scale=scale, teacher_scale=0.99)
    assert torch.equal(b.grad[:, 2:5], c[:, 2:5])
    lq = float(np.float32(0.99)) * v.double().cpu().numpy()
    if not rest:
        lq = lq - np.log(np.exp(lq).sum(1, keepdims=True))
    want = -np.exp(lq[:, 1:]) * scale * weight.double().cpu().numpy()[:, None]
    # rest: the share's rounding and two products'.  Otherwise its exponent in fp32 too, and the sum of shares
    tol = np.abs(want) * plain.U * (4 if rest else 16 + 2 * np.abs(lq[:, 1:]))
    close(b.grad[:, 2:5], want, tol, "gradient")


def test_logits_that_a_model_made(isr, torch):
    """Results are detached, and the gradient by the logits takes a model behind them to its own."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    w = torch.randn((50, 8), generator=gen, device="cuda", requires_grad=True)
    x = torch.randn((16, 8), generator=gen, device="cuda")
    e = torch.arange(4, dtype=torch.int32, device="cuda").repeat(16, 1)
    v = torch.log_softmax(torch.randn((16, 4), generator=gen, device="cuda"), 1) - 0.1
    logits = x @ w.t()
    r = isr.isr_logprobs(logits, e, top=2, entropy=True, stats=True)
    d = isr.isr_distill(logits, e, v, rest=True, grad=True)
    assert not any(t.requires_grad for t in (*r, d.loss, d.grad))
    logits.backward(d.grad)
    want = d.grad.double().t() @ x.double()
    # a product of 16 terms in fp32
    assert bool(((w.grad.double() - want).abs() <= 17 * plain.U * (d.grad.double().abs().t() @ x.double().abs())).all())
