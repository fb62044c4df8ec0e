"""What stands around the layers, on the GPU through the C ABI, against the fp64 oracle: embedding, loss, gradient norm and clipping, and a
whole training step of a small model.

Tolerances count roundings: u = 2^-24 is half a step of fp32, and a value stored as bf16 is off by 2^-8 of itself at most (u8)."""
import math

import numpy as np
import pytest
import torch

import paper_2511_09741_amd.binding as taw
from oracle import decoder_layer as O
from oracle import model_ops as M
from paper_2511_09741_amd import inputs as I
from tests import util as U

pytestmark = pytest.mark.gpu
u, u8 = 2.0 ** -24, 2.0 ** -8
DT = {"f32": (taw.TAW_F32, torch.float32, u), "bf16": (taw.TAW_BF16, torch.bfloat16, u8)}
IDS = {"i32": torch.int32, "i64": torch.int64}


def f64(t):
    return t.detach().double().cpu().numpy()


def on_gpu(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def scratch(nbytes):
    """bytes that are anything but zero: nothing may rest on what a workspace holds"""
    return torch.full((max(16, nbytes),), 0xA5, dtype=torch.uint8, device="cuda")


# ----------------------------------------------------------------------------- embedding
def zipf_ids(rng, T, V):
    return np.minimum((np.exp(rng.random(T) * math.log(V + 1.0)) - 1.0).astype(np.int64), V - 1)


EMBED = [  # T, H, V
    (1, 1, 1), (1, 64, 509), (5, 7, 3), (63, 64, 5), (64, 8, 1000), (65, 100, 7), (128, 64, 509), (257, 520, 33), (333, 256, 32003),
    (1000, 1, 2), (1024, 264, 70), (2048, 24, 90), (2048, 256, 500), (1025, 72, 64), (1100, 6, 300001), (1500, 1032, 300), (2049, 513, 20000), (4503, 1024, 32001), (9001, 20, 5), (20000, 8, 1)]


@pytest.mark.parametrize("T,H,V", EMBED)
@pytest.mark.parametrize("dtype,idt,scale", [("f32", "i64", 1.0), ("bf16", "i32", 1.0), ("bf16", "i64", 11.3137), ("f32", "i32", 0.37)])
def test_embed_fwd(taw, T, H, V, dtype, idt, scale):
    code, tdt, half = DT[dtype]
    rng = np.random.default_rng(T * 7 + H)
    ids = rng.integers(0, V, T)
    ids[T // 2:T // 2 + 2] = [-1, V][:len(ids[T // 2:T // 2 + 2])]
    table = on_gpu(rng.normal(size=(V, H)), tdt)
    x = torch.full((T, H), float("nan"), dtype=tdt, device="cuda")
    taw.taw_embed_fwd(taw.make_embed_desc(code, T, H, V, scale=scale), on_gpu(ids, IDS[idt]), table, x)
    s32 = float(np.float32(scale))
    ref = M.embed_fwd(ids, f64(table), s32)
    # one fp32 product and one rounding to the type; exact where the scale is 1
    assert np.all(np.abs(f64(x) - ref) <= (0 if scale == 1.0 else (u + half if dtype == "bf16" else u) * np.abs(ref)))


@pytest.mark.parametrize("T,H,V", EMBED)
@pytest.mark.parametrize("dtype,idt,scale,accumulate", [("f32", "i32", 1.0, False), ("bf16", "i64", 1.0, True), ("bf16", "i32", 11.3137, False), ("f32", "i64", 0.37, True)])
@pytest.mark.parametrize("kind", ["zipf", "one", "outside"])
def test_embed_bwd(taw, T, H, V, dtype, idt, scale, accumulate, kind):
    code, tdt, _ = DT[dtype]
    rng = np.random.default_rng(T * 5 + H)
    ids = zipf_ids(rng, T, V)
    if kind == "one":                     # every token the same row
        ids[:] = V // 2
    if kind == "outside":                 # a padded batch, and a row that the table does not have
        ids[rng.random(T) < 0.4] = -1
        ids[-1] = V
    dx = on_gpu(rng.normal(size=(T, H)), tdt)
    G = on_gpu(rng.normal(size=(V, H)), torch.float32)
    G0, s32 = f64(G), float(np.float32(scale))
    d = taw.make_embed_desc(code, T, H, V, scale=scale, flags=taw.TAW_ACCUMULATE if accumulate else 0)
    ws = scratch(taw.taw_embed_bwd_workspace_bytes(d))
    taw.taw_embed_bwd(d, on_gpu(ids, IDS[idt]), dx, G, ws)
    ref = M.embed_bwd(ids, f64(dx), V, s32, G0 if accumulate else None)
    # n - 1 additions in fp32, the scale, and the addition to the shard, each half a step of what it adds up to
    size = M.embed_bwd(ids, np.abs(f64(dx)), V, abs(s32), np.abs(G0) if accumulate else None)
    n = max(1, int(np.bincount(ids[(ids >= 0) & (ids < V)], minlength=1).max()) if ((ids >= 0) & (ids < V)).any() else 1)
    assert np.all(np.abs(f64(G) - ref) <= (n + 2) * u * size)
    if accumulate:
        left = np.setdiff1d(np.arange(V), ids)
        assert np.array_equal(f64(G)[left], G0[left])


@pytest.mark.parametrize("T,V,H", [(5, 9, 24), (700, 50, 40), (3000, 4000, 264)])
def test_embed_strides_and_what_lies_between(taw, T, V, H):
    """Rows inside wider buffers, at strides that leave them aligned and at odd ones; nothing beside them is written."""
    rng = np.random.default_rng(T)
    for pad_t, pad_x in ((8, 16), (3, 5)):
        ids = rng.integers(-1, V + 1, T)
        table, x = on_gpu(rng.normal(size=(V, H + pad_t)), torch.bfloat16), torch.full((T, H + pad_x), 7.0, dtype=torch.bfloat16, device="cuda")
        d = taw.make_embed_desc(taw.TAW_BF16, T, H, V, ld_table=H + pad_t, ld_x=H + pad_x)
        taw.taw_embed_fwd(d, on_gpu(ids, torch.int64), table, x)
        assert np.array_equal(f64(x[:, :H]), M.embed_fwd(ids, f64(table[:, :H]))) and bool((x[:, H:] == 7.0).all())
        G = torch.full((V, H + pad_t), 3.0, dtype=torch.float32, device="cuda")
        taw.taw_embed_bwd(d, on_gpu(ids, torch.int64), x, G, scratch(taw.taw_embed_bwd_workspace_bytes(d)))
        ref = M.embed_bwd(ids, f64(x[:, :H]), V)
        size = M.embed_bwd(ids, np.abs(f64(x[:, :H])), V)
        assert np.all(np.abs(f64(G[:, :H]) - ref) <= T * u * size) and bool((G[:, H:] == 3.0).all())


def test_embed_bwd_past_the_caches(taw):
    """Gradients that no cache holds, which the kernels stream."""
    T, H, V = 9000, 4096, 600
    rng = np.random.default_rng(6)
    ids, dx = zipf_ids(rng, T, V), torch.randn((T, H), device="cuda", dtype=torch.bfloat16)
    for accumulate in (False, True):
        G = torch.randn((V, H), device="cuda")
        d = taw.make_embed_desc(taw.TAW_BF16, T, H, V, flags=taw.TAW_ACCUMULATE if accumulate else 0)
        ref, size = (G.double(), G.double().abs()) if accumulate else (torch.zeros(V, H, dtype=torch.float64, device="cuda") for _ in range(2))
        for v in range(V):
            rows = dx[torch.from_numpy(np.flatnonzero(ids == v)).cuda()].double()
            ref[v] += rows.sum(0)
            size[v] += rows.abs().sum(0)
        taw.taw_embed_bwd(d, on_gpu(ids, torch.int32), dx, G, scratch(taw.taw_embed_bwd_workspace_bytes(d)))
        assert bool(((G.double() - ref).abs() <= (int(np.bincount(ids).max()) + 2) * u * size).all())


def test_embed_bwd_repeats_its_bits_and_no_tokens_zero_the_shard(taw):
    T, H, V = 9000, 640, 777
    rng = np.random.default_rng(8)
    ids, dx = on_gpu(zipf_ids(rng, T, V), torch.int32), on_gpu(rng.normal(size=(T, H)), torch.bfloat16)
    d = taw.make_embed_desc(taw.TAW_BF16, T, H, V)
    got = []
    for _ in range(4):
        G = torch.full((V, H), float("nan"), device="cuda")
        taw.taw_embed_bwd(d, ids, dx, G, scratch(taw.taw_embed_bwd_workspace_bytes(d)))
        got.append(G)
    assert all(torch.equal(g, got[0]) for g in got)
    none = taw.make_embed_desc(taw.TAW_BF16, 0, H, V)
    taw.taw_embed_bwd(none, None, None, got[0], scratch(taw.taw_embed_bwd_workspace_bytes(none)))
    assert not got[0].any()
    ids[:] = -1                           # and with tokens that all name no row
    taw.taw_embed_bwd(d, ids, dx, got[1], scratch(taw.taw_embed_bwd_workspace_bytes(d)))
    assert not got[1].any()


# ----------------------------------------------------------------------------- loss
def loss_bounds(l, lse, up, eps, z, V, half):
    """(rows, lse, dlogits): what the roundings of the fp32 formulas come to.  An exponent (l - m) log2 e has three roundings of its size and the
    exponential another step of its result; the sum adds a rounding for every 64 terms (a thread's part is shorter) and a tree of 16; then the logarithm."""
    live = np.isfinite(l)
    top, low = np.max(l, 1, where=live, initial=-1e39), np.min(l, 1, where=live, initial=1e39)
    reach = np.where(live.any(1), top - low, 0.0)
    size = np.max(np.abs(l), 1, where=live, initial=0.0)
    e_lse = u * (3 * np.minimum(reach, 104.0) + V / 64 + 24 + 4 * size + 4 * np.abs(lse))
    e_rows = e_lse * (1 + 2 * z * np.abs(lse)) + u * (6 * size + 6 * np.abs(lse) + 4 * z * lse ** 2) + eps * u * (V / 64 + 24) * size
    with np.errstate(all="ignore"):
        p = np.exp(l - lse[:, None])
    off = e_lse[:, None] + u * (3 * np.abs(np.nan_to_num(l - lse[:, None], neginf=0.0, posinf=0.0)) + 12)
    grow = 1 + 2 * z * np.abs(lse)[:, None]
    e_d = np.abs(up)[:, None] * (p * grow * off + p * 2 * z * e_lse[:, None] + 4 * u * (p * grow + 1 + eps))
    return e_rows, e_lse, e_d


def check_loss(taw, T, V, dtype, grad, ldt, eps=0.0, z=0.0, mean=True, pad=0, odd=0, scale=1.0, logits=None, labels=None, in_place=False, seed=0):
    code, tdt, _ = DT[dtype]
    gcode, gdt, half = DT[grad]
    rng = np.random.default_rng(seed + 31 * T + V)
    if logits is None:
        logits = rng.normal(0.0, 2.0, (T, V))
    if labels is None:
        labels = rng.integers(0, V, T)
        labels[rng.random(T) < 0.2] = -100
        if T > 3:
            labels[3] = V                 # a class that is not there
    ld, V_pad = V + odd, V + pad
    buf = torch.full((T, ld), float("nan"), dtype=tdt, device="cuda")
    buf[:, :V] = on_gpu(logits, tdt)
    l = f64(buf[:, :V])
    y = on_gpu(labels, IDS[ldt])
    ldg = ld if in_place else V_pad + odd
    out = buf if in_place else torch.full((T, ldg), 9.0, dtype=gdt, device="cuda")
    loss, rows, lse = torch.full((4,), 5.0, device="cuda"), torch.full((T,), 5.0, device="cuda"), torch.full((T,), 5.0, device="cuda")
    d = taw.make_loss_desc(code, T, V, grad_dtype=gcode, ld=ld, ld_grad=ldg, V_pad=V_pad, label_smoothing=eps, z_loss=z, grad_scale=scale,
                           flags=taw.TAW_LOSS_MEAN if mean else 0)
    e32, z32 = float(np.float32(eps)), float(np.float32(z))
    r_rows, r_lse, counted = M.loss_fwd(l, labels, e32, z32)
    total, n = M.loss_total(r_rows, counted, mean)
    up = np.where(counted, scale / (max(n, 1) if mean else 1), 0.0)
    ref = M.loss_bwd(l, labels, r_lse, up, e32, z32, V_pad)
    t_rows, t_lse, t_d = loss_bounds(l, np.where(np.isfinite(r_lse), r_lse, 0.0), up, e32, z32, V, half)
    t_d = np.pad(t_d, ((0, 0), (0, pad))) + half * np.abs(ref) + 2.0 ** -133      # fp32 and bf16 hold nothing smaller

    def near(got, want, tol, what):
        fine = np.isfinite(want)
        assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]) and np.array_equal(np.isnan(got), np.isnan(want)), what
        worst = np.max(np.abs(got[fine] - want[fine]) / np.maximum(np.broadcast_to(tol, want.shape)[fine], 1e-300), initial=0.0)
        assert worst <= 1.0, (what, worst)

    # the loss alone
    taw.taw_loss_fwd(d, buf, y, loss, rows, lse, scratch(taw.taw_loss_workspace_bytes(d)))
    alone = [t.clone() for t in (loss, rows, lse)]
    near(f64(rows), r_rows, t_rows, "rows")
    near(f64(lse), r_lse, t_lse, "lse")
    got = f64(loss)
    assert got[1] == n and list(got[2:]) == [5.0, 5.0]
    near(got[:1], np.array([total]), np.sum(np.where(np.isfinite(t_rows), t_rows, 0)) / (max(n, 1) if mean else 1) + u * abs(total), "loss")
    # the gradient from a saved lse, with a gradient for every row
    w = rng.normal(size=T).astype(np.float32)
    if not in_place:
        taw.taw_loss_bwd(d, buf, y, lse, on_gpu(w, torch.float32), out)
        want = M.loss_bwd(l, labels, f64(lse), w.astype(np.float64) * counted, e32, z32, V_pad)
        _, _, tb = loss_bounds(l, np.where(np.isfinite(r_lse), r_lse, 0.0), w.astype(np.float64), e32, z32, V, half)
        near(f64(out[:, :V_pad]), want, np.pad(tb, ((0, 0), (0, pad))) + half * np.abs(want) + 2.0 ** -133, "dlogits of taw_loss_bwd")
        assert bool((out[:, V_pad:] == 9.0).all())
        out.fill_(9.0)
    # both in one call
    rest = buf[:, V:].clone()
    loss.fill_(5.0), rows.fill_(5.0), lse.fill_(5.0)
    taw.taw_loss_fwd_bwd(d, buf, y, loss, rows, lse, out, scratch(taw.taw_loss_workspace_bytes(d)))
    near(f64(out[:, :V_pad]), ref, t_d, "dlogits")
    near(f64(rows), r_rows, t_rows, "rows with the gradient")
    near(f64(lse), r_lse, t_lse, "lse with the gradient")
    assert f64(loss)[1] == n
    if in_place:
        assert torch.equal(buf[:, V_pad:].view(torch.uint8), rest[:, pad:].contiguous().view(torch.uint8))
    else:
        assert bool((out[:, V_pad:] == 9.0).all())
    return alone, out


TYPES = [("bf16", "bf16", "i64"), ("f32", "bf16", "i32"), ("f32", "f32", "i64")]
LOSS = [(1, 1), (1, 2), (3, 5), (5, 63), (7, 64), (4, 1000), (300, 257), (2, 2047), (3, 4097), (2, 8200), (2, 16391), (2, 32003), (2, 50001), (2, 65537), (2, 131073), (1, 262144), (129, 66000), (3, 600011)]


@pytest.mark.parametrize("T,V", LOSS)
@pytest.mark.parametrize("dtype,grad,ldt", TYPES)
def test_loss(taw, T, V, dtype, grad, ldt):
    check_loss(taw, T, V, dtype, grad, ldt)
    check_loss(taw, T, V, dtype, grad, ldt, eps=0.1, z=1e-3, mean=False, scale=0.5, pad=(-V) % 64, odd=3)


@pytest.mark.parametrize("T,V", [(9, 7), (16, 63), (17, 63), (16, 1025), (16, 2047), (16, 2056), (8, 4103), (8, 4104), (7, 2053)])
@pytest.mark.parametrize("dtype,grad,ldt", TYPES)
def test_loss_few_short_rows(taw, T, V, dtype, grad, ldt):
    """On both sides of the sizes up to which one launch does it all."""
    check_loss(taw, T, V, dtype, grad, ldt, eps=0.1, z=1e-3, pad=(-V) % 64, odd=5)
    check_loss(taw, T, V, dtype, grad, ldt, mean=False, labels=np.full(T, V - 1))


@pytest.mark.parametrize("T,V", [(5, 64), (6, 1003), (3, 32000), (3, 50001), (2, 131073)])
@pytest.mark.parametrize("dtype,ldt", [("bf16", "i64"), ("f32", "i32")])
def test_loss_in_place(taw, T, V, dtype, ldt):
    """dlogits is the logits: the same bits as in a buffer of its own, nothing beside the rows."""
    check_loss(taw, T, V, dtype, dtype, ldt, z=1e-4, pad=5, odd=8, in_place=True)
    rng = np.random.default_rng(V)
    l, y = on_gpu(rng.normal(0, 2, (T, V)), DT[dtype][1]), on_gpu(rng.integers(0, V, T), IDS[ldt])
    d = taw.make_loss_desc(DT[dtype][0], T, V)
    loss, ws, apart = torch.zeros(2, device="cuda"), scratch(taw.taw_loss_workspace_bytes(d)), torch.empty_like(l)
    taw.taw_loss_fwd_bwd(d, l, y, loss, None, None, apart, ws)
    taw.taw_loss_fwd_bwd(d, l, y, loss, None, None, l, ws)
    assert torch.equal(l, apart)


@pytest.mark.parametrize("T,V", [(8, 40), (8, 1001), (8, 32000), (8, 70001), (131, 70001), (131, 140003)])
@pytest.mark.parametrize("dtype,grad,ldt", TYPES)
def test_loss_masked_classes(taw, T, V, dtype, grad, ldt):
    """-inf in most places, in all but one, in all, at the label, in whole stretches; the type's lowest value; a peaked row; uniform rows of large values."""
    rng = np.random.default_rng(V)
    l = rng.normal(0, 2, (T, V))
    y = rng.integers(0, V, T)
    low = float(torch.finfo(DT[dtype][1]).min)
    l[0, rng.random(V) < 0.9] = -np.inf
    l[0, y[0]] = 1.0
    l[1, :] = -np.inf
    l[1, y[1]] = -3.0
    l[2, :] = -np.inf                      # nothing is left
    l[3, y[3]] = -np.inf                   # the label is masked
    l[4, V // 3:] = -np.inf
    y[4] = 0
    l[5, :] = low
    l[5, y[5]] = 0.5
    l[6, :] = 1e4
    l[7, (y[7] + 1) % V] = 300.0
    check_loss(taw, T, V, dtype, grad, ldt, logits=l, labels=y)
    check_loss(taw, T, V, dtype, grad, ldt, logits=l, labels=y, mean=False, odd=1)


@pytest.mark.parametrize("T,V", [(8, 40), (20, 1001), (8, 32000), (8, 70001), (131, 70001)])
@pytest.mark.parametrize("dtype,grad,ldt", TYPES)
def test_loss_smoothing_over_masked_classes(taw, T, V, dtype, grad, ldt):
    """Classes masked by the type's lowest value have a share of a smoothed label: the loss is large and finite, however many they are."""
    rng = np.random.default_rng(V + 1)
    l = rng.normal(0, 2, (T, V))
    l[:, 5:] = np.where(rng.random((T, V - 5)) < 0.8, float(torch.finfo(DT[dtype][1]).min), l[:, 5:])
    l[1] = float(torch.finfo(DT[dtype][1]).min)
    y = rng.integers(0, 5, T)
    _, out = check_loss(taw, T, V, dtype, grad, ldt, eps=0.1, logits=l, labels=y)
    # the bounds of rows of such size say little about lse and the gradient, which are those of classes masked by -inf
    l = f64(on_gpu(l, DT[dtype][1]))
    l[l < -1e38] = -np.inf
    rest = np.arange(T) != 1
    l, y, e32, up = l[rest], y[rest], float(np.float32(0.1)), np.full(T - 1, 1.0 / T)
    lse = M.loss_fwd(l, y)[1]
    ref = M.loss_bwd(l, y, lse, up, e32)
    bound = loss_bounds(l, lse, up, e32, 0.0, V, DT[grad][2])[2] + DT[grad][2] * np.abs(ref) + 2.0 ** -133
    assert np.max(np.abs(f64(out)[rest] - ref) / bound) <= 1.0


@pytest.mark.parametrize("T,V", [(6, 777), (6, 70001), (133, 70001)])
@pytest.mark.parametrize("dtype,grad,ldt", TYPES)
def test_loss_rows_of_infinities_and_nan(taw, dtype, grad, ldt, T, V):
    """+inf or NaN make all of a counted row's results NaN, and say nothing of a row that is not counted or of another row."""
    rng = np.random.default_rng(1)
    l = rng.normal(0, 2, (T, V))
    l[0, 5], l[1, V - 77], l[2, 9], l[3, :] = np.inf, np.nan, np.nan, np.inf
    y = np.concatenate([[1, 2, -1, -100, 4, 776], np.full(T - 6, 7)])
    code, tdt, _ = DT[dtype]
    t = on_gpu(l, tdt)
    d = taw.make_loss_desc(code, T, V, grad_dtype=DT[grad][0])
    loss, rows, lse = torch.zeros(2, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
    out = torch.zeros((T, V), dtype=DT[grad][1], device="cuda")
    for f, extra in ((taw.taw_loss_fwd, ()), (taw.taw_loss_fwd_bwd, (out,))):
        f(d, t, on_gpu(y, IDS[ldt]), loss, rows, lse, *extra, scratch(taw.taw_loss_workspace_bytes(d)))
        assert np.isnan(f64(rows)[:2]).all() and np.isnan(f64(lse)[:2]).all() and not f64(rows)[2:4].any() and np.isfinite(f64(rows)[4:]).all()
        assert np.isnan(f64(loss)[0]) and f64(loss)[1] == T - 2
    g = f64(out)
    assert np.isnan(g[:2]).all() and not g[2:4].any()
    r, e, n = M.loss_fwd(f64(t)[4:], y[4:])
    assert np.allclose(g[4:], M.loss_bwd(f64(t)[4:], y[4:], e, np.full(T - 4, 1 / (T - 2))), rtol=u8 + 1e-4, atol=1e-7)


@pytest.mark.parametrize("T", [1, 5, 3000])
def test_loss_with_nothing_counted(taw, T):
    V = 130
    l = torch.full((T, V), float("nan"), dtype=torch.bfloat16, device="cuda")
    y = torch.full((T,), -100, device="cuda")
    d = taw.make_loss_desc(taw.TAW_BF16, T, V)
    loss, out = torch.full((2,), 5.0, device="cuda"), torch.full((T, V), 9.0, dtype=torch.bfloat16, device="cuda")
    taw.taw_loss_fwd_bwd(d, l, y, loss, None, None, out, scratch(taw.taw_loss_workspace_bytes(d)))
    assert f64(loss).tolist() == [0.0, 0.0] and not out.any()
    none = taw.make_loss_desc(taw.TAW_BF16, 0, V)
    loss.fill_(5.0)
    taw.taw_loss_fwd(none, None, None, loss, None, None, scratch(taw.taw_loss_workspace_bytes(none)))
    assert f64(loss).tolist() == [0.0, 0.0]


@pytest.mark.parametrize("T,V", [(1500, 9), (16384, 17), (16385, 17), (70001, 33)])
def test_loss_rows_of_several_workgroups(taw, T, V):
    """Labels counted, and losses added up, by one workgroup and by several."""
    check_loss(taw, T, V, "bf16", "bf16", "i64", eps=0.1)
    check_loss(taw, T, V, "f32", "f32", "i32", mean=False)


@pytest.mark.parametrize("T,V", [(2500, 70), (5000, 33)])
def test_loss_many_rows(taw, T, V):
    check_loss(taw, T, V, "bf16", "bf16", "i32")
    check_loss(taw, T, V, "f32", "f32", "i64", eps=0.1, mean=False)


# ----------------------------------------------------------------------------- norm and clipping
def fresh(rng, sizes, dtypes, std=1.0):
    """tensors in one buffer, and a guard behind each"""
    out = []
    for n, dt in zip(sizes, dtypes):
        b = torch.full((n + 64,), 123.0, dtype=DT[dt][1], device="cuda")
        b[:n] = on_gpu(rng.normal(0, std, n), DT[dt][1])
        out.append(b)
    return out


SIZES = [[1], [3, 0, 5], [64] * 9, [4099, 1, 70000], [16384, 16385, 16383, 33000], [7] * 130, [100 + 37 * i for i in range(300)], [5_000_003, 2]]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("kind", ["f32", "bf16", "both"])
def test_norm_and_clip(taw, sizes, kind):
    rng = np.random.default_rng(len(sizes))
    dts = [("f32", "bf16")[i % 2] if kind == "both" else kind for i in range(len(sizes))]
    bufs = fresh(rng, sizes, dts)
    gs = [b[:n] for b, n in zip(bufs, sizes)]
    was = [f64(g) for g in gs]
    lst, st = taw.make_tensor_list(gs), taw.new_clip_state()
    ws = scratch(taw.taw_grad_norm_workspace_bytes(lst))
    total = math.sqrt(sum(float(np.sum(w * w)) for w in was))
    for max_norm, s in ((0.5 * total * 0.25, -0.25), (2.0 * total, 1.0), (math.inf, 1.0)):
        norm, coef, bad = M.clip(was, max_norm, s)
        taw.taw_grad_norm(lst, max_norm, s, st, ws)
        # fp64 sums; the norm and the coefficient are rounded once, the coefficient from the rounded norm
        assert abs(float(st.sumsq) - total ** 2) <= 1e-12 * total ** 2 and abs(float(st.norm) - norm) <= 2 * u * norm
        assert abs(float(st.coef) - coef) <= 4 * u * coef and int(st.nonfinite) == bad == 0
        taw.taw_grad_clip(lst, st)
        c = float(st.coef)
        for g, w, dt, b, n in zip(gs, was, dts, bufs, sizes):
            assert np.all(np.abs(f64(g) - c * w) <= (0 if c == 1.0 else u + (u8 if dt == "bf16" else 0)) * np.abs(w))
            assert bool((b[n:] == 123.0).all())
            g.copy_(on_gpu(w, g.dtype))


def test_norm_in_two_halves_and_over_owners(taw):
    """Shards on several owners: sums of squares added up, then the coefficient; the same state as one call over all of them, and its bits over repeats."""
    rng = np.random.default_rng(3)
    bufs = fresh(rng, [70001, 12, 333], ["f32", "f32", "bf16"])
    gs = [b[:-64] for b in bufs]
    whole, parts = taw.new_clip_state(), taw.new_clip_state()
    lists = [taw.make_tensor_list([g]) for g in gs]
    for rep in range(3):
        lst = taw.make_tensor_list(gs)
        taw.taw_grad_norm(lst, 3.0, 0.5, whole, scratch(taw.taw_grad_norm_workspace_bytes(lst)))
        for i, l in enumerate(lists):
            taw.taw_grad_sumsq(l, i > 0, parts, scratch(taw.taw_grad_norm_workspace_bytes(l)))
        taw.taw_clip_coef(parts, 3.0, 0.5)
        a, b = whole.buffer.cpu(), parts.buffer.cpu()
        assert abs(float(a[0] - b[0])) <= 1e-14 * float(a[0]) and abs(float(whole.coef) - float(parts.coef)) <= 2 * u
        if rep:
            assert torch.equal(a, last)
        last = a
    empty = taw.make_tensor_list([])
    taw.taw_grad_norm(empty, 1.0, 1.0, whole, scratch(taw.taw_grad_norm_workspace_bytes(empty)))
    taw.taw_grad_clip(empty, whole)
    assert float(whole.norm) == 0.0 and float(whole.coef) == 1.0 and float(whole.sumsq) == 0.0


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("where", [0, 16384, 70000])
def test_a_gradient_that_is_not_finite(taw, bad, where):
    rng = np.random.default_rng(9)
    gs = [b[:-64] for b in fresh(rng, [40, 70001], ["bf16", "f32"])]
    gs[1][where] = bad
    was = [g.clone() for g in gs]
    lst, st = taw.make_tensor_list(gs), taw.new_clip_state()
    taw.taw_grad_norm(lst, 1.0, 1.0, st, scratch(taw.taw_grad_norm_workspace_bytes(lst)))
    assert int(st.nonfinite) == 1 and float(st.coef) == 0.0 and not math.isfinite(float(st.norm))
    taw.taw_grad_clip(lst, st)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(gs, was))
    gs[1][where] = 1e25                    # its square is more than fp32 holds, its norm is not
    taw.taw_grad_norm(lst, 1.0, 1.0, st, scratch(taw.taw_grad_norm_workspace_bytes(lst)))
    assert int(st.nonfinite) == 0 and abs(float(st.norm) / 1e25 - 1) < 1e-6
    taw.taw_grad_clip(lst, st)
    assert abs(float(gs[1][where]) - 1.0) < 1e-6


@pytest.mark.parametrize("n", [1, 3, 4, 1023, 70003])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", ["clipped", "untouched", "skipped"])
@pytest.mark.parametrize("zero", [False, True])
def test_clipped_step(taw, n, dtype, case, zero):
    """The clipped step is the plain step with grad_scale * coef, bit for bit; a gradient that is not finite leaves weights and moments alone."""
    rng = np.random.default_rng(n)
    code, tdt, _ = DT[dtype]
    w = on_gpu(rng.normal(0, 0.02, n), torch.float32)
    m, v, G = on_gpu(rng.normal(0, 1e-3, n), torch.float32), on_gpu(rng.normal(0, 1e-3, n) ** 2, torch.float32), on_gpu(rng.normal(0, 1, n), torch.float32)
    chunk = w.to(tdt)
    if case == "skipped":
        G[n // 2] = float("inf")
    lst, st = taw.make_tensor_list([G]), taw.new_clip_state()
    s = 0.25
    norm = s * math.sqrt(float((f64(G) ** 2).sum()))
    taw.taw_grad_norm(lst, 0.3 * norm if case == "clipped" else 1e30, s, st, scratch(taw.taw_grad_norm_workspace_bytes(lst)))
    a = [t.clone() for t in (chunk, w, m, v, G)]
    b = [t.clone() for t in (chunk, w, m, v, G)]
    kw = dict(step=3, lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, zero_grad=zero)
    taw.taw_optimizer_step_clipped(st, a[0], code, *a[1:], n, grad_scale=s, **kw)
    if case == "skipped":
        assert all(torch.equal(x, y) for x, y in zip(a[:4], b[:4]))
        assert not a[4].any() if zero else torch.equal(a[4], b[4])
        return
    coef = np.float32(float(st.coef))
    assert coef == 1.0 if case == "untouched" else abs(coef - 0.3) < 1e-5
    taw.taw_optimizer_step(b[0], code, *b[1:], n, grad_scale=float(np.float32(s) * coef), **kw)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


# ----------------------------------------------------------------------------- together
def plain_step(ids, labels, E, W, Ws, head, gam, cfg):
    """embedding, layers, last norm, head, loss and back, in fp64: (loss, gradients)"""
    x = M.embed_fwd(ids, E).reshape(cfg.B, cfg.S, cfg.H)
    caches = []
    for w in Ws:
        x, cache = O.layer_fwd(w, x, cfg.n_heads, cfg.rope_theta, cfg.rms_eps)
        caches.append(cache)
    z = x.reshape(-1, cfg.H)
    xn, r = O.rmsnorm_fwd(z, gam, cfg.rms_eps)
    rows, lse, counted = M.loss_fwd(xn @ head.T, labels)
    total, n = M.loss_total(rows, counted)
    d = M.loss_bwd(xn @ head.T, labels, lse, np.full(len(labels), 1.0 / n))
    dz, dgam = O.rmsnorm_bwd(d @ head, z, r, gam)
    dx, Gs = dz.reshape(cfg.B, cfg.S, cfg.H), []
    for w, cache in zip(reversed(Ws), reversed(caches)):
        dx, G = O.layer_bwd(w, cache, dx)
        Gs.insert(0, G)
    return total, {"embed": M.embed_bwd(ids, dx.reshape(-1, cfg.H), E.shape[0]), "head": d.T @ xn, "gamma": dgam, "layers": Gs}


@pytest.mark.parametrize("cfg,V", [(I.LayerConfig("small-f32", I.F32, 2, 48, 64, 4, 16, 176), 203), (I.LayerConfig("small-bf16", I.BF16, 2, 80, 256, 2, 128, 392), 504)])
def test_a_training_step(taw, cfg, V):
    """embed -> two layers -> norm -> head -> loss -> back -> norm over all shards -> clipped AdamW, against the same in fp64; the bars are the layer's
    own (1e-4 and 2e-2 of a tensor's largest value)."""
    H, T, f32, tdt = cfg.H, cfg.T, torch.float32, torch.bfloat16 if cfg.dtype == I.BF16 else torch.float32
    rng = np.random.default_rng(12)
    ids, labels = rng.integers(0, V, T), rng.integers(0, V, T)
    ids[-5:], labels[-6:] = -1, -100
    E = on_gpu(rng.normal(0, 1.0, (V, H)), tdt)
    head, gam = on_gpu(rng.normal(0, 0.05, (V, H)), tdt), on_gpu(1 + 0.1 * rng.normal(size=H), tdt)
    ws_ = [I.make_weights(cfg, 100 + i) for i in range(2)]
    layers = [U.DeviceLayer(taw, cfg) for _ in ws_]
    for L, w in zip(layers, ws_):
        L.set_weights(w)
    yd = on_gpu(labels, torch.int64)
    idd = on_gpu(ids, torch.int32)
    # forward
    ed = taw.make_embed_desc(cfg.dtype, T, H, V)
    x = torch.empty((T, H), dtype=tdt, device="cuda")
    taw.taw_embed_fwd(ed, idd, E, x)
    xs = [x.view(cfg.B, cfg.S, H)]
    for L in layers:
        xs.append(L.fwd(xs[-1]))
    xn, r = torch.empty((T, H), dtype=tdt, device="cuda"), torch.empty(T, device="cuda")
    taw.taw_op_rmsnorm_fwd(cfg.dtype, T, H, xs[-1], gam, cfg.rms_eps, xn, r)
    logits = torch.empty((T, V), device="cuda")
    taw.taw_op_gemm(cfg.dtype, taw.TAW_GEMM_NT, T, V, H, xn, H, head, H, logits, V, taw.TAW_F32)
    ld = taw.make_loss_desc(taw.TAW_F32, T, V, grad_dtype=cfg.dtype)
    loss, dlogits = torch.empty(2, device="cuda"), torch.empty((T, V), dtype=tdt, device="cuda")
    taw.taw_loss_fwd_bwd(ld, logits, yd, loss, None, None, dlogits, scratch(taw.taw_loss_workspace_bytes(ld)))
    # backward
    Gh, dg, dxn, dz = torch.empty((V, H), device="cuda"), torch.empty(H, device="cuda"), torch.empty_like(xn), torch.empty_like(xn)
    taw.taw_op_linear_bwd(cfg.dtype, T, V, H, dlogits, head, xn, dxn, Gh)
    taw.taw_op_rmsnorm_bwd(cfg.dtype, T, H, dxn, xs[-1], r, gam, None, dz, dg, 0, torch.empty(taw.taw_op_rmsnorm_bwd_scratch_floats(H), device="cuda"))
    dx = dz.view(cfg.B, cfg.S, H)
    for i in (1, 0):
        dx = layers[i].bwd(xs[i], dx)
    Ge = torch.empty((V, H), device="cuda")
    taw.taw_embed_bwd(ed, idd, dx, Ge, scratch(taw.taw_embed_bwd_workspace_bytes(ed)))
    # the same in fp64
    total, ref = plain_step(ids, labels, f64(E), None, [I.weights_to_f64(w, cfg.dtype) for w in ws_], f64(head), f64(gam), cfg)
    tol = U.TOL[cfg.dtype]
    errs = {"loss": abs(float(loss[0]) - total) / total, "embed": U.tensor_scale_err(f64(Ge), ref["embed"]), "head": U.tensor_scale_err(f64(Gh), ref["head"]),
            "gamma": U.tensor_scale_err(f64(dg), ref["gamma"])}
    for i, L in enumerate(layers):
        errs.update({f"{i}.{k}": U.tensor_scale_err(g, ref["layers"][i][k]) for k, g in L.grads().items()})
    print(errs, flush=True)
    assert float(loss[1]) == T - 6 and max(errs.values()) <= tol, errs
    # norm over everything, and the owner's update of one shard
    lst, st = taw.make_tensor_list([Ge, Gh, dg] + [L.G for L in layers]), taw.new_clip_state()
    taw.taw_grad_norm(lst, 0.1, 1.0, st, scratch(taw.taw_grad_norm_workspace_bytes(lst)))
    norm, coef, _ = M.clip([ref["embed"], ref["head"], ref["gamma"]] + [g for G in ref["layers"] for g in G.values()], 0.1)
    assert abs(float(st.norm) / norm - 1) <= tol and coef < 1
    master = E.float().reshape(-1)
    m, v, chunk = torch.zeros_like(master), torch.zeros_like(master), E.clone().reshape(-1)
    w0 = f64(master)
    taw.taw_optimizer_step_clipped(st, chunk, cfg.dtype, master, m, v, Ge, Ge.numel(), step=1, lr=1e-2, weight_decay=0.1, zero_grad=True)
    assert U.tensor_scale_err(f64(m), 0.1 * coef * ref["embed"].reshape(-1)) <= 2 * tol and not Ge.any()
    unnamed = np.setdiff1d(np.arange(V), ids)
    assert np.allclose(f64(master).reshape(V, H)[unnamed], w0.reshape(V, H)[unnamed] * (1 - 1e-3), rtol=1e-6, atol=0)


# ----------------------------------------------------------------------------- as a program uses them
class Pieces:
    """Every operation on buffers of its own, at sizes that take the kernels for many tokens (embedding: the sort) and for a few."""

    def __init__(self, T, H, V, seed):
        rng = np.random.default_rng(seed)
        self.T, self.V = T, V
        self.ids = on_gpu(zipf_ids(rng, T + 1, V), torch.int32)
        self.labels = self.ids[1:]                       # the next token: aligned to its type, not to 16 bytes
        self.ids = self.ids[:-1]
        self.E, self.dx = on_gpu(rng.normal(size=(V, H)), torch.bfloat16), on_gpu(rng.normal(size=(T, H)), torch.bfloat16)
        self.logits = on_gpu(rng.normal(0, 2, (T, V)), torch.float32)
        self.ed, self.ld = taw.make_embed_desc(taw.TAW_BF16, T, H, V), taw.make_loss_desc(taw.TAW_F32, T, V, grad_dtype=taw.TAW_BF16)
        self.x, self.G, self.dlogits = torch.empty_like(self.dx), torch.empty((V, H), device="cuda"), torch.empty((T, V), dtype=torch.bfloat16, device="cuda")
        self.loss, self.lse = torch.empty(2, device="cuda"), torch.empty(T, device="cuda")
        self.lst, self.state = taw.make_tensor_list([self.G]), taw.new_clip_state()
        self.w, self.m, self.v, self.chunk = self.E.float(), torch.zeros_like(self.G), torch.zeros_like(self.G), self.E.clone()
        self.ws = [scratch(n) for n in (taw.taw_embed_bwd_workspace_bytes(self.ed), taw.taw_loss_workspace_bytes(self.ld), taw.taw_grad_norm_workspace_bytes(self.lst))]
        torch.cuda.synchronize()

    def outs(self):
        return [self.x, self.G, self.dlogits, self.loss, self.lse, self.state.buffer, self.w, self.m, self.v, self.chunk]

    def run(self, stream):
        taw.taw_embed_fwd(self.ed, self.ids, self.E, self.x, stream)
        taw.taw_loss_fwd_bwd(self.ld, self.logits, self.labels, self.loss, None, self.lse, self.dlogits, self.ws[1], stream=stream)
        taw.taw_embed_bwd(self.ed, self.ids, self.dx, self.G, self.ws[0], stream=stream)
        taw.taw_grad_norm(self.lst, 1.0, 1.0, self.state, self.ws[2], stream=stream)
        taw.taw_grad_clip(self.lst, self.state, stream)
        taw.taw_optimizer_step_clipped(self.state, self.chunk, taw.TAW_BF16, self.w, self.m, self.v, self.G, self.G.numel(), step=1, stream=stream)

    def reset(self):
        self.w.copy_(self.E.float()), self.m.zero_(), self.v.zero_()


@pytest.mark.parametrize("T,H,V", [(3000, 256, 1000), (100, 64, 70003)])
def test_captured_and_replayed(taw, T, H, V):
    """Recorded into a graph and replayed with other work between, every replay has the eager results' bits, also with new inputs in the same buffers."""
    p = Pieces(T, H, V, 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            p.run(torch.cuda.current_stream())
    for rep in range(4):
        if rep == 2:
            p.logits.mul_(0.5), p.dx.add_(1.0)
            p.ids.copy_(torch.flip(p.ids, [0]))
        p.reset()
        torch.cuda.synchronize()
        p.run(torch.cuda.current_stream())
        torch.cuda.synchronize()
        want = [t.clone() for t in p.outs()]
        for t in p.outs():
            if t is not p.w and t is not p.m and t is not p.v:
                t.view(torch.uint8).fill_(0x5A)
        for w in p.ws:
            w.fill_(rep)
        p.reset()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(p.outs(), want)), rep
        torch.randn(1000, 1000, device="cuda").sum().item()


def test_two_streams_at_once(taw):
    """Calls that overlap on two streams, each with its own workspace, do not meet."""
    ps = [Pieces(2500, 512, 3001, 2), Pieces(700, 128, 40001, 3)]
    want = []
    for p in ps:
        p.run(torch.cuda.current_stream())
        torch.cuda.synchronize()
        want.append([t.clone() for t in p.outs()])
        p.reset()
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    for _ in range(3):
        for p, s in zip(ps, streams):
            with torch.cuda.stream(s):
                p.reset()
            p.run(s)
    torch.cuda.synchronize()
    for p, w in zip(ps, want):
        assert all(torch.equal(a, b) for a, b in zip(p.outs(), w))


def test_offsets_past_32_bits(taw):
    """A table, logits and a gradient of more than 2^31 elements: their last rows."""
    V, H, T = 300_000, 8192, 700
    G = torch.zeros((V, H), device="cuda")
    ids = torch.full((T,), V - 1, dtype=torch.int64, device="cuda")
    ids[::3] = V - 2
    dx = torch.ones((T, H), dtype=torch.bfloat16, device="cuda")
    d = taw.make_embed_desc(taw.TAW_BF16, T, H, V)
    taw.taw_embed_bwd(d, ids, dx, G, scratch(taw.taw_embed_bwd_workspace_bytes(d)))
    n = (T + 2) // 3
    assert bool((G[V - 1] == T - n).all()) and bool((G[V - 2] == n).all()) and not G[:V - 2].any()
    lst, st = taw.make_tensor_list([G.reshape(-1)]), taw.new_clip_state()
    taw.taw_grad_norm(lst, 1.0, 1.0, st, scratch(taw.taw_grad_norm_workspace_bytes(lst)))
    assert float(st.sumsq) == H * ((T - n) ** 2 + n ** 2)
    taw.taw_grad_clip(lst, st)
    assert torch.allclose(G[V - 1], (T - n) * st.coef.expand(H), rtol=1e-6)
    del G
    table = torch.zeros((V, H), dtype=torch.bfloat16, device="cuda")
    table[V - 1], table[V - 2] = 3.0, 5.0
    x = torch.empty((T, H), dtype=torch.bfloat16, device="cuda")
    taw.taw_embed_fwd(d, ids, table, x)
    assert bool((x[::3] == 5.0).all()) and bool((x[1::3] == 3.0).all())
    del table, x
    T, V = 40_000, 65_541
    l = torch.empty((T, V), dtype=torch.bfloat16, device="cuda").normal_()
    y = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    d = taw.make_loss_desc(taw.TAW_BF16, T, V, flags=0)
    loss, rows, lse, ws = torch.empty(2, device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), scratch(taw.taw_loss_workspace_bytes(d))
    tail = l[-3:].double().cpu().numpy()
    taw.taw_loss_fwd_bwd(d, l, y, loss, rows, lse, l, ws)
    r, e, _ = M.loss_fwd(tail, f64(y[-3:]).astype(np.int64))
    assert np.allclose(f64(rows[-3:]), r, rtol=1e-5) and np.allclose(f64(lse[-3:]), e, rtol=1e-6)
    g = M.loss_bwd(tail, f64(y[-3:]).astype(np.int64), e, np.ones(3))
    assert np.all(np.abs(f64(l[-3:]) - g) <= (u8 + 1e-5) * np.abs(g) + 1e-9)


def test_embed_bwd_very_many_tokens(taw):
    T, H, V = 300_001, 8, 1000
    rng = np.random.default_rng(4)
    ids = zipf_ids(rng, T, V)
    dx = on_gpu(rng.integers(-3, 4, (T, H)), torch.float32)          # whole numbers: every sum is exact
    d = taw.make_embed_desc(taw.TAW_F32, T, H, V)
    G = torch.empty((V, H), device="cuda")
    taw.taw_embed_bwd(d, on_gpu(ids, torch.int64), dx, G, scratch(taw.taw_embed_bwd_workspace_bytes(d)))
    assert np.array_equal(f64(G), M.embed_bwd(ids, f64(dx), V))


def test_loss_of_the_most_rows(taw):
    """2^24 rows: more threads than one dimension of a launch has."""
    T, V = 1 << 24, 8
    l, y = torch.randn((T, V), device="cuda").bfloat16(), torch.randint(-1, V, (T,), device="cuda", dtype=torch.int32)
    d = taw.make_loss_desc(taw.TAW_BF16, T, V, grad_scale=float(T))
    loss, rows, lse, out = torch.zeros(2, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda"), torch.empty_like(l)
    taw.taw_loss_fwd_bwd(d, l, y, loss, rows, lse, out, scratch(taw.taw_loss_workspace_bytes(d)))
    live, L = y >= 0, l.double()
    n = int(live.sum())
    ref = torch.logsumexp(L, 1)
    want = torch.where(live, ref - L.gather(1, y.clamp(min=0).long()[:, None])[:, 0], 0.0)
    # values below 8: 2^-20 is over ten roundings of them
    assert float((rows - want).abs().max()) < 2 ** -20 and float((lse - torch.where(live, ref, 0.0)).abs().max()) < 2 ** -20
    assert float(loss[1]) == n and abs(float(loss[0]) - float(want.sum()) / n) < 2 ** -20
    g = (torch.exp(L - ref[:, None]) - torch.nn.functional.one_hot(y.clamp(min=0).long(), V)) * live[:, None] * (T / n)
    near = g.abs() * u8 + 2.0 ** -18
    assert bool(((out.double() - g).abs() <= near).all())
    out.fill_(9.0)
    taw.taw_loss_bwd(d, l, y, lse, torch.full((T,), T / n, device="cuda"), out)
    assert bool(((out.double() - g).abs() <= near).all())


def test_embed_of_the_most_threads(taw):
    """Rows of odd length, a thread an element: more threads than one dimension of a launch has."""
    T, H, V = (1 << 20) + 3, 8193, 7
    table, ids = torch.randn((V, H), device="cuda").bfloat16(), torch.randint(0, V, (T,), device="cuda")
    x = torch.empty((T, H), dtype=torch.bfloat16, device="cuda")
    taw.taw_embed_fwd(taw.make_embed_desc(taw.TAW_BF16, T, H, V), ids, table, x)
    for t in range(0, T, 1 << 16):
        assert torch.equal(x[t:t + (1 << 16)], table[ids[t:t + (1 << 16)]])
    del x
    T, H, V = 3000, 4097, (1 << 20) + 5
    ids, dx = torch.randint(0, V, (T,), device="cuda"), torch.ones((T, H), dtype=torch.bfloat16, device="cuda")
    ids[:100] = V - 1
    d = taw.make_embed_desc(taw.TAW_BF16, T, H, V)
    G = torch.full((V, H), float("nan"), device="cuda")
    taw.taw_embed_bwd(d, ids, dx, G, scratch(taw.taw_embed_bwd_workspace_bytes(d)))
    count = torch.bincount(ids, minlength=V).float()
    for v in range(0, V, 1 << 16):
        assert bool((G[v:v + (1 << 16)] == count[v:v + (1 << 16), None]).all())
