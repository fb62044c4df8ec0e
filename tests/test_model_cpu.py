"""What stands around the layers (include/model/taw_model.h), without a GPU: the oracle's pins, the exported symbols, sizes, and every
refusal before a launch."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

import paper_2511_09741_amd.binding as taw
from oracle import model_ops as M

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK = 0x10000          # a 16-byte aligned address that no call below gets as far as using


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(taw.LIB_PATH):
        from paper_2511_09741_amd.build import build
        build()
    return taw.load()


# ----------------------------------------------------------------------------- oracle
def _logits(T, V, seed):
    return np.random.default_rng(seed).normal(0.0, 2.0, (T, V))


@pytest.mark.parametrize("eps,z", [(0.0, 0.0), (0.1, 0.0), (0.0, 0.05), (0.2, 0.03)])
def test_loss_gradient_against_differences(eps, z):
    T, V = 4, 9
    l, y = _logits(T, V, 1), np.array([0, 8, -100, 3])
    w = np.array([0.7, -1.3, 5.0, 0.2])
    f = lambda a: float(np.sum(w * M.loss_fwd(a, y, eps, z)[0]))
    _, lse, _ = M.loss_fwd(l, y, eps, z)
    d = M.loss_bwd(l, y, lse, w, eps, z)
    h = 1e-6
    for t in range(T):
        for v in range(V):
            up, down = l.copy(), l.copy()
            up[t, v] += h
            down[t, v] -= h
            assert abs((f(up) - f(down)) / (2 * h) - d[t, v]) < 1e-8


def test_loss_closed_forms():
    V = 7
    rows, lse, n = M.loss_fwd(np.full((2, V), 3.0), np.array([2, -1]))
    assert np.allclose(rows, [np.log(V), 0.0]) and np.allclose(lse, [3.0 + np.log(V), 0.0]) and list(n) == [True, False]
    assert M.loss_total(rows, n) == (pytest.approx(np.log(V)), 1)
    assert M.loss_total(np.zeros(2), np.array([False, False])) == (0.0, 0)
    l = _logits(3, V, 2)
    l[0, :] = -np.inf
    l[1, 4] = -np.inf
    rows, lse, _ = M.loss_fwd(l, np.array([1, 0, 0]))
    assert rows[0] == np.inf and lse[0] == -np.inf and np.isfinite(rows[1:]).all()
    d = M.loss_bwd(l, np.array([1, 0, 0]), lse, np.ones(3), V_pad=9)
    assert not d[0].any() and d[1, 4] == 0 and not d[:, V:].any() and np.allclose(d[1:].sum(1), 0)


@pytest.mark.parametrize("eps", [0.0, 0.1])
def test_loss_against_a_library(eps):
    l, y = _logits(6, 11, 3), np.array([0, 3, -100, 10, 5, -100])
    t = torch.tensor(l, requires_grad=True)
    ref = torch.nn.functional.cross_entropy(t, torch.tensor(y), label_smoothing=eps)
    ref.backward()
    rows, lse, n = M.loss_fwd(l, y, eps)
    assert M.loss_total(rows, n)[0] == pytest.approx(ref.item(), abs=1e-12)
    assert np.allclose(M.loss_bwd(l, y, lse, np.full(6, 1 / 4), eps), t.grad.numpy(), atol=1e-14)
    assert not np.allclose(M.loss_bwd(l, y, lse, np.full(6, 1 / 6), eps), t.grad.numpy(), atol=1e-3)     # a planted mistake: the mean over all rows


def test_embedding_against_a_library_and_differences():
    rng = np.random.default_rng(4)
    E, ids, dx = rng.normal(size=(5, 3)), np.array([4, 0, 4, -1, 2, 4, 5]), rng.normal(size=(7, 3))
    x = M.embed_fwd(ids, E, 1.5)
    assert not x[3].any() and not x[6].any() and np.array_equal(x[0], 1.5 * E[4])
    G = M.embed_bwd(ids, dx, 5, 1.5)
    t = torch.tensor(E, requires_grad=True)
    ok = torch.tensor((ids >= 0) & (ids < 5))
    (1.5 * torch.nn.functional.embedding(torch.tensor(ids).clamp(0, 4), t) * torch.tensor(dx) * ok[:, None]).sum().backward()
    assert np.allclose(G, t.grad.numpy(), atol=1e-14)
    h = 1e-6
    for v in range(5):
        up, down = E.copy(), E.copy()
        up[v, 1] += h
        down[v, 1] -= h
        assert abs(float(np.sum(dx * (M.embed_fwd(ids, up, 1.5) - M.embed_fwd(ids, down, 1.5)))) / (2 * h) - G[v, 1]) < 1e-8
    assert np.allclose(M.embed_bwd(ids, dx, 5, 1.5, np.ones((5, 3))), G + 1)


def test_clip_against_a_library():
    rng = np.random.default_rng(5)
    gs = [rng.normal(size=n) for n in (1, 7, 100)]
    ps = [torch.nn.Parameter(torch.zeros(len(g), dtype=torch.float64)) for g in gs]
    for p, g in zip(ps, gs):
        p.grad = torch.tensor(2.0 * g)
    norm, coef, bad = M.clip(gs, 3.0, 2.0)
    assert torch.nn.utils.clip_grad_norm_(ps, 3.0).item() == pytest.approx(norm) and bad == 0
    assert np.allclose(ps[2].grad.numpy(), 2.0 * gs[2] * coef, rtol=1e-5)        # the library adds 1e-6 to the norm
    assert M.clip(gs, 1e9)[1] == 1.0
    assert M.clip(gs + [np.array([np.inf])], 1.0)[1:] == (0.0, 1) and M.clip(gs + [np.array([np.nan])], 1.0)[1:] == (0.0, 1)


# ----------------------------------------------------------------------------- the boundary
def test_every_declared_symbol_is_exported(lib):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "model", "taw_model.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(taw_[a-z0-9_]+)\s*\(", src))
    assert names == set(taw.MODEL_EXPORTS) and not names & set(taw.EXPORTS)
    for n in names:
        assert hasattr(lib, n)


def test_clip_state_layout():
    s = taw.new_clip_state("cpu")
    raw = s.buffer.numpy().tobytes()
    assert len(raw) == 32
    s.sumsq.fill_(2.0), s.norm.fill_(3.0), s.coef.fill_(0.5), s.nonfinite.fill_(1)
    b = s.buffer.numpy().tobytes()
    assert np.frombuffer(b[:8], "f8")[0] == 2.0 and list(np.frombuffer(b[8:16], "f4")) == [3.0, 0.5] and np.frombuffer(b[16:20], "i4")[0] == 1


def refuse(code, f, *a, **kw):
    with pytest.raises(taw.TawError) as e:
        f(*a, **kw)
    assert e.value.status == code, e.value
    assert str(e.value)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), taw.TAW_ERR_DTYPE), (dict(T=-1), taw.TAW_ERR_SHAPE), (dict(H=0), taw.TAW_ERR_SHAPE), (dict(V=0), taw.TAW_ERR_SHAPE),
    (dict(T=2**24 + 1), taw.TAW_ERR_SHAPE), (dict(V=2**24 + 1), taw.TAW_ERR_SHAPE), (dict(ld_table=63), taw.TAW_ERR_SHAPE), (dict(ld_x=63), taw.TAW_ERR_SHAPE),
    (dict(scale=float("nan")), taw.TAW_ERR_SHAPE), (dict(scale=float("inf")), taw.TAW_ERR_SHAPE), (dict(flags=2), taw.TAW_ERR_SHAPE)])
def test_bad_embedding_descriptors(lib, kw, code):
    d = taw.make_embed_desc(**{**dict(dtype=taw.TAW_BF16, T=8, H=64, V=100), **kw})
    refuse(code, taw.taw_embed_fwd, d, OK, OK, OK + (1 << 20))
    refuse(code, taw.taw_embed_bwd, d, OK, OK, OK + (1 << 20), OK + (1 << 24), 1 << 30)
    assert taw.taw_embed_bwd_workspace_bytes(d) == 0


def test_embedding_refusals(lib):
    d = taw.make_embed_desc(taw.TAW_BF16, 8, 64, 100)
    far = OK + (1 << 20)
    ws = taw.taw_embed_bwd_workspace_bytes(d)
    for i in range(3):
        a = [OK + (1 << 22), OK, far]
        a[i] = None
        refuse(taw.TAW_ERR_NULL, taw.taw_embed_fwd, d, *a)
    refuse(taw.TAW_ERR_ALIGN, taw.taw_embed_fwd, d, OK + 4, OK, far, id_type=taw.TAW_I64)
    refuse(taw.TAW_ERR_ALIGN, taw.taw_embed_fwd, d, OK + 2, OK, far, id_type=taw.TAW_I32)
    refuse(taw.TAW_ERR_ALIGN, taw.taw_embed_fwd, d, OK, OK + 8, far)
    refuse(taw.TAW_ERR_DTYPE, taw.taw_embed_fwd, d, OK, OK, far, id_type=2)
    refuse(taw.TAW_ERR_SHAPE, taw.taw_embed_fwd, d, far + (1 << 20), OK, OK + 128)                  # x inside the table
    refuse(taw.TAW_ERR_SHAPE, taw.taw_embed_fwd, d, far + 16, OK, far)                              # x over the ids
    refuse(taw.TAW_ERR_SHAPE, taw.taw_embed_bwd, d, far, OK, OK, far + (1 << 20), ws)               # G over dx
    refuse(taw.TAW_ERR_SHAPE, taw.taw_embed_bwd, d, OK, far, OK + 16, far + (1 << 20), ws)          # G over the ids
    assert ws == 0                                                                                  # a few tokens need none
    more = taw.make_embed_desc(taw.TAW_BF16, 5000, 64, 100)
    ws = taw.taw_embed_bwd_workspace_bytes(more)
    assert ws > 0
    refuse(taw.TAW_ERR_WORKSPACE, taw.taw_embed_bwd, more, OK, far, far + (1 << 20), far + (1 << 22), ws - 1)
    refuse(taw.TAW_ERR_NULL, taw.taw_embed_bwd, more, OK, far, far + (1 << 20), None, ws)
    refuse(taw.TAW_ERR_ALIGN, taw.taw_embed_bwd, more, OK, far, far + (1 << 20), far + (1 << 22) + 8, ws)
    refuse(taw.TAW_ERR_SHAPE, taw.taw_embed_bwd, more, OK, far, far + (1 << 20), far, ws)
    none = taw.make_embed_desc(taw.TAW_BF16, 0, 64, 100, flags=taw.TAW_ACCUMULATE)
    taw.taw_embed_fwd(none, None, None, None)                                                       # no tokens: nothing to do
    taw.taw_embed_bwd(none, None, None, None, None)
    refuse(taw.TAW_ERR_NULL, taw.taw_embed_bwd, taw.make_embed_desc(taw.TAW_BF16, 0, 64, 100), None, None, None, None)     # but the shard is to be zeroed
    refuse(taw.TAW_ERR_DTYPE, taw.taw_embed_fwd, d, torch.zeros(8, dtype=torch.int16), OK, far)
    refuse(taw.TAW_ERR_SHAPE, taw.taw_embed_fwd, d, torch.zeros(16, dtype=torch.int64)[::2], OK, far)
    refuse(taw.TAW_ERR_UNSUPPORTED, taw.taw_embed_fwd, d, torch.zeros(8, dtype=torch.int64), OK, far)      # in host memory


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=5), taw.TAW_ERR_DTYPE), (dict(grad_dtype=taw.TAW_F32), taw.TAW_ERR_DTYPE), (dict(T=-1), taw.TAW_ERR_SHAPE), (dict(V=0), taw.TAW_ERR_SHAPE),
    (dict(V_pad=99), taw.TAW_ERR_SHAPE), (dict(ld=99), taw.TAW_ERR_SHAPE), (dict(V_pad=128, ld_grad=127), taw.TAW_ERR_SHAPE),
    (dict(label_smoothing=1.0), taw.TAW_ERR_SHAPE), (dict(label_smoothing=-0.1), taw.TAW_ERR_SHAPE), (dict(label_smoothing=float("nan")), taw.TAW_ERR_SHAPE),
    (dict(z_loss=-1.0), taw.TAW_ERR_SHAPE), (dict(z_loss=float("inf")), taw.TAW_ERR_SHAPE), (dict(grad_scale=float("nan")), taw.TAW_ERR_SHAPE),
    (dict(flags=2), taw.TAW_ERR_SHAPE), (dict(T=2**24 + 1), taw.TAW_ERR_SHAPE), (dict(V=2**24 + 1), taw.TAW_ERR_SHAPE)])
def test_bad_loss_descriptors(lib, kw, code):
    d = taw.make_loss_desc(**{**dict(dtype=taw.TAW_BF16, T=8, V=100), **kw})
    far = OK + (1 << 24)
    refuse(code, taw.taw_loss_fwd, d, OK, far, far, far, far, far, 1 << 30)
    refuse(code, taw.taw_loss_fwd_bwd, d, OK, far, far, far, far, OK, far, 1 << 30)
    refuse(code, taw.taw_loss_bwd, d, OK, far, far, far, OK)
    assert taw.taw_loss_workspace_bytes(d) == 0


def test_loss_refusals(lib):
    d = taw.make_loss_desc(taw.TAW_F32, 8, 100, grad_dtype=taw.TAW_BF16)
    ws = taw.taw_loss_workspace_bytes(d)
    L, Y, S, R, E, D, W = (OK + (i << 16) for i in range(7))
    good = [L, Y, S, R, E, D, W, ws]
    for i in (0, 1, 2, 5, 6):
        a = list(good)
        a[i] = None
        refuse(taw.TAW_ERR_NULL, taw.taw_loss_fwd_bwd, d, *a)
    for i in (0, 2, 3, 4, 5, 6):
        a = list(good)
        a[i] += 8
        refuse(taw.TAW_ERR_ALIGN, taw.taw_loss_fwd_bwd, d, *a)
    refuse(taw.TAW_ERR_WORKSPACE, taw.taw_loss_fwd_bwd, d, *good[:-1], ws - 1)
    refuse(taw.TAW_ERR_SHAPE, taw.taw_loss_fwd_bwd, d, L, Y, S, R, E, L, W, ws)            # in place needs one type
    same = taw.make_loss_desc(taw.TAW_F32, 8, 100, ld=128)
    refuse(taw.TAW_ERR_SHAPE, taw.taw_loss_bwd, same, L, Y, R, E, L)                       # ... and one row stride
    refuse(taw.TAW_ERR_SHAPE, taw.taw_loss_bwd, taw.make_loss_desc(taw.TAW_F32, 8, 100), L, Y, R, E, L + 16)
    for i, k in ((2, 0), (2, 1), (2, 3), (3, 0), (3, 4), (3, 5), (4, 1), (4, 5), (6, 0), (6, 1), (6, 2), (6, 3), (6, 5), (1, 5)):
        a = list(good)
        a[i] = a[k]                                                                        # two of the buffers are one
        refuse(taw.TAW_ERR_SHAPE, taw.taw_loss_fwd_bwd, d, *a)
    for i in (1, 2, 3):
        a = [L, Y, R, E, D]
        a[i] = D
        refuse(taw.TAW_ERR_SHAPE, taw.taw_loss_bwd, d, *a)
    for i in range(5):
        a = [L, Y, R, E, D]
        a[i] = None
        refuse(taw.TAW_ERR_NULL, taw.taw_loss_bwd, d, *a)
    refuse(taw.TAW_ERR_DTYPE, taw.taw_loss_fwd, d, L, Y, S, R, E, W, ws, label_type=3)
    refuse(taw.TAW_ERR_ALIGN, taw.taw_loss_fwd, d, L, Y + 4, S, R, E, W, ws, label_type=taw.TAW_I64)
    taw.taw_loss_bwd(taw.make_loss_desc(taw.TAW_F32, 0, 100), None, None, None, None, None)      # no rows: nothing to do


def test_norm_and_clip_refusals(lib):
    def lst(*entries):
        class L:
            array = (taw.taw_tensor * max(1, len(entries)))(*[taw.taw_tensor(*e) for e in entries])
            count = len(entries)
        return L
    ok, far = lst((OK, 64, 0)), OK + (1 << 20)
    ws = taw.taw_grad_norm_workspace_bytes(ok)
    assert ws > 0 and taw.taw_grad_norm_workspace_bytes(lst((OK, 64, 7))) == 0
    for bad in (0.0, -1.0, float("nan")):
        refuse(taw.TAW_ERR_SHAPE, taw.taw_grad_norm, ok, bad, 1.0, far, far + 4096, ws)
        refuse(taw.TAW_ERR_SHAPE, taw.taw_clip_coef, far, bad)
    refuse(taw.TAW_ERR_SHAPE, taw.taw_grad_norm, ok, 1.0, float("inf"), far, far + 4096, ws)
    refuse(taw.TAW_ERR_WORKSPACE, taw.taw_grad_norm, ok, 1.0, 1.0, far, far + 4096, ws - 1)
    refuse(taw.TAW_ERR_NULL, taw.taw_grad_norm, ok, 1.0, 1.0, None, far + 4096, ws)
    refuse(taw.TAW_ERR_NULL, taw.taw_grad_sumsq, ok, 0, far, None, ws)
    refuse(taw.TAW_ERR_NULL, taw.taw_grad_sumsq, lst((None, 4, 0)), 0, far, far + 4096, ws)
    refuse(taw.TAW_ERR_ALIGN, taw.taw_grad_sumsq, lst((OK + 8, 4, 0)), 0, far, far + 4096, ws)
    refuse(taw.TAW_ERR_DTYPE, taw.taw_grad_sumsq, lst((OK, 4, 2)), 0, far, far + 4096, ws)
    refuse(taw.TAW_ERR_SHAPE, taw.taw_grad_sumsq, lst((OK, 2**48 + 1, 0)), 0, far, far + 4096, 1 << 40)
    refuse(taw.TAW_ERR_SHAPE, taw.taw_grad_norm, ok, 1.0, 1.0, far, far + 16, 1 << 20)                # the workspace over the state
    refuse(taw.TAW_ERR_SHAPE, taw.taw_grad_norm, ok, 1.0, 1.0, OK + 240, far, ws)
    refuse(taw.TAW_ERR_SHAPE, taw.taw_grad_norm, ok, 1.0, 1.0, far, OK, ws)
    refuse(taw.TAW_ERR_NULL, taw.taw_clip_coef, None, 1.0)
    refuse(taw.TAW_ERR_ALIGN, taw.taw_clip_coef, far + 8, 1.0)
    refuse(taw.TAW_ERR_NULL, taw.taw_grad_clip, ok, None)
    refuse(taw.TAW_ERR_SHAPE, taw.taw_grad_clip, ok, OK + 32)                                         # the state inside a tensor
    refuse(taw.TAW_ERR_SHAPE, taw.taw_grad_clip, lst((OK, 64, 0), (OK, 64, 0)), far)                  # the same tensor twice
    refuse(taw.TAW_ERR_SHAPE, taw.taw_grad_clip, lst((OK + 512, 8, 0), (OK, 64, 0), (OK + 240, 8, 0)), far)
    n = lst()
    n.count = -1
    refuse(taw.TAW_ERR_SHAPE, taw.taw_grad_clip, n, far)
    refuse(taw.TAW_ERR_DTYPE, taw.make_tensor_list, [torch.zeros(4, dtype=torch.float16)])
    refuse(taw.TAW_ERR_SHAPE, taw.make_tensor_list, [torch.zeros(4, 3).t()])
    refuse(taw.TAW_ERR_UNSUPPORTED, taw.make_tensor_list, [torch.zeros(4)])


def test_clipped_step_refusals(lib):
    W, A, M_, V, G = (OK + (i << 16) for i in range(5))
    far = OK + (1 << 20)
    step = lambda state, **kw: taw.taw_optimizer_step_clipped(state, W, taw.TAW_BF16, A, M_, V, kw.pop("G", G), 64, kw.pop("step", 1), **kw)
    refuse(taw.TAW_ERR_NULL, step, None)
    refuse(taw.TAW_ERR_ALIGN, step, far + 8)
    refuse(taw.TAW_ERR_SHAPE, step, G + 128)                # the state inside the gradients
    refuse(taw.TAW_ERR_SHAPE, step, W + 96)
    refuse(taw.TAW_ERR_SHAPE, step, far, step=0)
    refuse(taw.TAW_ERR_NULL, step, far, G=None)
    refuse(taw.TAW_ERR_SHAPE, step, far, beta2=1.0)
