"""The loss over the vocabulary where logits are large, through every kernel that forms it: a workgroup for a few short rows, a wavefront and a
workgroup to a row, rows that are longer than a workgroup holds, rows that are cut into parts, and the gradient from a saved lse.

Tolerances count roundings: u = 2^-24 is half a step of fp32.  A row's probabilities depend on the differences between its logits alone, which are
exact where the row's values are equal or neighbours; so their bounds have no term for the size of the logits."""
import numpy as np
import pytest
import torch

import paper_2511_09741_amd.binding as taw
from oracle import model_ops as M
from tests.test_gpu_model import DT, IDS, f64, on_gpu, scratch

pytestmark = pytest.mark.gpu
u = 2.0 ** -24
TYPES = [("bf16", "bf16", "i64"), ("f32", "bf16", "i32"), ("f32", "f32", "i64")]
# few rows in one launch; a wavefront a row; workgroups of 256 and 512; longer than a workgroup holds; cut into parts
SHAPES = [(16, 40), (80, 40), (80, 3001), (80, 9001), (80, 30001), (160, 70001), (48, 70001), (80, 140003)]


def call_loss(l, y, dtype, grad, ldt, gradient=True, **kw):
    """(loss, rows, lse, dlogits) of logits and labels given in fp64, and the logits as stored"""
    T, V = l.shape
    t = on_gpu(l, DT[dtype][1])
    d = taw.make_loss_desc(DT[dtype][0], T, V, grad_dtype=DT[grad][0], **kw)
    loss, rows, lse = torch.full((4,), 5.0, device="cuda"), torch.full((T,), 5.0, device="cuda"), torch.full((T,), 5.0, device="cuda")
    out = torch.full((T, V), 9.0, dtype=DT[grad][1], device="cuda")
    labels, ws = on_gpu(y, IDS[ldt]), scratch(taw.taw_loss_workspace_bytes(d))
    if gradient:
        taw.taw_loss_fwd_bwd(d, t, labels, loss, rows, lse, out, ws)
    else:
        taw.taw_loss_fwd(d, t, labels, loss, rows, lse, ws)
    return f64(loss), f64(rows), f64(lse), f64(out), f64(t)


def saved(l, y, lse, w, dtype, grad, ldt, **kw):
    T, V = l.shape
    d = taw.make_loss_desc(DT[dtype][0], T, V, grad_dtype=DT[grad][0], **kw)
    out = torch.full((T, V), 9.0, dtype=DT[grad][1], device="cuda")
    taw.taw_loss_bwd(d, on_gpu(l, DT[dtype][1]), on_gpu(y, IDS[ldt]), on_gpu(lse, torch.float32), on_gpu(w, torch.float32), out)
    return f64(out)


def far_rows(T, V, seed):
    """Rows around maxima of every size: uniform ones, ones with a single logit above the rest or below it, ones with most classes masked."""
    maxima = [0.0]
    for m in (1e4, 1e6, 1e8, 1e9, 2.0 ** 30, 2.0 ** 30 + 128, 1.25e9, 3e9, 1e10, 1e12, 1e20, 9e29, 1e30, 2e30, 1e38, 3.3e38):
        maxima += [m, -m]
    rng = np.random.default_rng(seed)
    l, y = np.empty((T, V)), rng.integers(0, V, T)
    start = rng.integers(0, len(maxima))
    for t in range(T):
        m, kind, c = maxima[(start + t) % len(maxima)], (t // len(maxima) + t) % 4, rng.integers(0, V)
        l[t] = m
        if kind == 1:                       # one above the rest; every other of them is the label
            l[t] = m - 0.5 * abs(m) if m > -3e38 else m
            l[t, c] = m
            if rng.random() < 0.5:
                y[t] = c
        if kind == 2 and m < 3e38:          # one below the rest
            l[t, c] = m - 0.01 * abs(m) - 1000.0
        if kind == 3:
            l[t, rng.random(V) < 0.9] = -np.inf
            l[t, y[t]] = m
    return l, y


def near(got, want, tol, what):
    assert np.array_equal(np.isfinite(got), np.isfinite(want)), what
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine]), what
    tol = np.broadcast_to(tol, want.shape)[fine]
    worst = np.max(np.abs(got[fine] - want[fine]) / np.maximum(tol, 1e-300), initial=0.0)
    assert worst <= 1.0, (what, worst)


def gradient_bound(l, y, p, up, half, ref):
    """Every logit here is its row's maximum or has no probability (its exponential is below e^-64).  The exponentials of the maximum are one value; their
    sum adds a rounding for every 64 of them and a tree of 24; what is scaled, divided and subtracted has four of its size.  An exponential is held to
    2^-62: it is formed beside a factor of up to 2^64 that it shares with the sum."""
    T, V = l.shape
    tol = np.abs(up)[:, None] * (p * (V / 64 + 40) * u + 2.0 ** -61)
    tol[np.arange(T), y] += np.abs(up) * 4 * u
    return tol + half * np.abs(ref) + 2.0 ** -133


@pytest.mark.parametrize("T,V", SHAPES)
@pytest.mark.parametrize("dtype,grad,ldt", TYPES)
def test_loss_of_rows_far_from_zero(taw, T, V, dtype, grad, ldt):
    """A maximum of any size is a finite logit like any other: loss and lse are finite, probabilities are those of the differences."""
    l, y = far_rows(T, V, T + V)
    l = f64(on_gpu(l, DT[dtype][1]))
    want_rows, want_lse, counted = M.loss_fwd(l, y)
    assert counted.all() and np.isfinite(want_lse).all()
    up = np.full(T, 1.0 / T)
    ref = M.loss_bwd(l, y, want_lse, up)
    top = np.max(l, 1, keepdims=True)
    p = np.where(l == top, 1.0, 0.0) / np.sum(l == top, 1, keepdims=True)
    ref_p = p * up[:, None]                 # fp64 does not hold lse - l of the largest rows either
    ref_p[np.arange(T), y] -= up
    small = np.abs(top[:, 0]) < 1e6
    assert np.abs(ref - ref_p)[small].max() <= 1e-8 * up[0]
    size = np.max(np.abs(l), 1, where=np.isfinite(l), initial=0.0)
    tol = u * (V / 64 + 128 + 8 * size)     # what is formed of logits of that size, each rounding a half step of it
    for gradient in (False, True):
        loss, rows, lse, out, _ = call_loss(l, y, dtype, grad, ldt, gradient)
        near(lse, want_lse, tol, "lse")
        near(rows, want_rows, 2 * tol, "rows")
        assert loss[1] == T and list(loss[2:]) == [5.0, 5.0]
    near(out, ref_p, gradient_bound(l, y, p, up, DT[grad][2], ref_p), "dlogits")


@pytest.mark.parametrize("T,V", [(80, 40), (80, 3001), (80, 30001)])
@pytest.mark.parametrize("dtype,grad,ldt", TYPES)
def test_gradient_from_a_saved_lse_far_from_zero(taw, T, V, dtype, grad, ldt):
    l, y = far_rows(T, V, T + V + 1)
    l = f64(on_gpu(l, DT[dtype][1]))
    lse = M.loss_fwd(l, y)[1].astype(np.float32).astype(np.float64)
    w = np.random.default_rng(V).normal(size=T).astype(np.float32).astype(np.float64)
    ref = M.loss_bwd(l, y, lse, w)
    p = np.exp(np.minimum(l - lse[:, None], 0.0))
    # the lse as saved is the formula's; a probability has the exponent's rounding (of what remains of 2^+-64 and of the difference) and three of its own
    tol = np.abs(w)[:, None] * (p * u * (2 * 64 + 8 * np.minimum(np.abs(l - lse[:, None]), 1e3) + 16) + 2.0 ** -61)
    tol[np.arange(T), y] += np.abs(w) * 4 * u
    near(saved(l, y, lse, w, dtype, grad, ldt), ref, tol + DT[grad][2] * np.abs(ref) + 2.0 ** -133, "dlogits")


@pytest.mark.parametrize("T,V", [(3, 900), (40, 5001), (3, 20000), (160, 50001), (48, 50001), (100, 150001)])
@pytest.mark.parametrize("grad", ["bf16", "f32"])
@pytest.mark.parametrize("base", [1e4, -1e4, 1e6, 1e8])
def test_parts_of_a_row_weighed_against_each_other(taw, T, V, grad, base):
    """One logit above all the others, which are equal and have most of the sum between them: the parts of a cut row, and the wavefronts of another,
    have different maxima, at sizes where the rounding of a maximum times log2 e is worth up to the 2^4 of the largest base."""
    rng = np.random.default_rng(V + T)
    step = float(np.spacing(np.float32(abs(base))))
    l, y = np.empty((T, V)), rng.integers(0, V, T)
    log2e = np.longdouble(np.float32(1.44269504088896340736))
    for t in range(T):
        at = base + step * rng.integers(-400, 400, 200)
        product = at.astype(np.longdouble) * log2e
        l[t] = at[np.argmax(np.abs(product - product.astype(np.float32)))]      # the roundest of some
        l[t, rng.integers(0, V)] += max(step, round(rng.uniform(0.5, 6.0) / step) * step)
    assert np.array_equal(l, l.astype(np.float32))
    w = np.full(T, 1.0)
    want_rows, want_lse, _ = M.loss_fwd(l, y)
    loss, rows, lse, out, _ = call_loss(l, y, "f32", grad, "i64", flags=0)
    ref = M.loss_bwd(l, y, want_lse, w) if abs(base) < 1e6 else None
    d = l - np.max(l, 1, keepdims=True)
    p = np.exp(d) / np.sum(np.exp(d), 1, keepdims=True)
    want = p.copy()
    want[np.arange(T), y] -= 1.0
    if ref is not None:
        assert np.abs(ref - want).max() <= 1e-10
    # the difference's product with log2 e has two roundings and the exponential two more of its result, in the numerator and in the sum; then the sum's
    tol = p * u * (V / 64 + 40 + 4 * np.abs(d))
    tol[np.arange(T), y] += 4 * u
    near(out, want, tol + DT[grad][2] * np.abs(want) + 2.0 ** -61, "dlogits")


def lse_and_rows_bound(l, V, lse, rows):
    """A row's loss and lse are formed from its maximum m and from log sum exp(l - m), which is at most log V: that has the roundings of the sum, of the
    exponents, and of a logarithm of up to 64 + 24 and what is taken from it; lse one more of its own size, the loss one of m - l_y and one of itself."""
    m = np.max(l, 1)
    low = np.min(l, 1, where=np.isfinite(l), initial=np.inf)
    e = u * (V / 64 + 24 + 4 * np.minimum(m - low, 104.0) + 4 * 88)
    return e + u * np.abs(lse), e + 4 * u * np.abs(rows)


@pytest.mark.parametrize("T,V", SHAPES)
@pytest.mark.parametrize("dtype,grad,ldt", TYPES)
def test_loss_does_not_depend_on_where_a_row_lies(taw, T, V, dtype, grad, ldt):
    """lse is the nearest value but for the roundings of a sum of numbers below 1, never below the maximum, and the loss keeps what lse has no room for."""
    l, y = far_rows(T, V, T + V + 2)
    l = f64(on_gpu(l, DT[dtype][1]))
    rng = np.random.default_rng(V)
    near_rows = rng.normal(0, 2, (T, V)) + rng.choice([0.0, 20.0, -300.0, 5000.0], T)[:, None]
    for l in (l, f64(on_gpu(near_rows, DT[dtype][1]))):
        m = np.max(l, 1)
        log_sum = np.log(np.sum(np.exp(l - m[:, None]), 1))
        want_lse, want_rows = m + log_sum, (m - l[np.arange(T), y]) + log_sum
        t_lse, t_rows = lse_and_rows_bound(l, V, want_lse, want_rows)
        for gradient in (False, True):
            loss, rows, lse, _, _ = call_loss(l, y, dtype, grad, ldt, gradient, flags=0)
            near(lse, want_lse, t_lse, "lse")
            near(rows, want_rows, t_rows, "rows")
            assert np.all(lse >= m - u * (V / 64 + 400))
            with np.errstate(over="ignore"):
                total = np.sum(want_rows, keepdims=True).astype(np.float32).astype(np.float64)      # more than fp32 holds: infinite
            near(loss[:1], total, np.sum(t_rows) + 2 * u * np.abs(total), "loss")


@pytest.mark.parametrize("T,V", [(80, 40), (80, 3001), (80, 30001)])
@pytest.mark.parametrize("dtype,grad,ldt", TYPES)
def test_forward_and_backward_far_from_zero(taw, T, V, dtype, grad, ldt):
    """The gradient from the lse that the forward left: no probability is more than 1."""
    l, y = far_rows(T, V, T + V + 3)
    _, _, lse, _, l = call_loss(l, y, dtype, grad, ldt, False)
    assert np.all(lse >= np.max(l, 1) - u * (V / 64 + 400))
    w = np.full(T, 1.0)
    out = saved(l, y, lse, w, dtype, grad, ldt)
    p = out.copy()
    p[np.arange(T), y] += 1.0
    assert np.isfinite(out).all() and np.all(p <= 1.0 + 2.0 ** -7) and np.all(p >= -2.0 ** -8)


@pytest.mark.parametrize("T,V", [(3, 2), (40, 2), (3, 5001), (3, 70001), (160, 70001)])
@pytest.mark.parametrize("dtype,grad,ldt", TYPES)
def test_smoothed_loss_near_the_largest_number(taw, T, V, dtype, grad, ldt):
    """The difference of two logits may be more than fp32 holds where the loss, which has a share of it, is not."""
    eps = 0.5
    l = np.full((T, V), 2e38)
    l[:, 1] = -2.5e38 if V == 2 else -3e38
    l = f64(on_gpu(l, DT[dtype][1]))
    y = np.ones(T, dtype=np.int64)
    want = M.loss_fwd(l, y, eps)[0]
    assert np.all((want > 2e38) & (want < 3.4e38)) and np.all(l[:, 0] - l[:, 1] > 3.41e38)
    for gradient in (False, True):
        _, rows, _, _, _ = call_loss(l, y, dtype, grad, ldt, gradient, flags=0, label_smoothing=eps)
        # four roundings of the loss's size, and those of the weighted sum of logits of 3e38
        near(rows, want, u * (4 * want + eps * (V / 64 + 40) * 3e38), "rows")
