"""What stands around the decoder layers in a training step, as timed cases: the embedding and its gradient, the loss over the
vocabulary with its gradient, and the global gradient norm with clipping.

A program that trains with the layer calls has token ids, an embedding table and its fp32 gradient shard, the logits that the
product with the head's weights gave, labels, and a list of gradient shards with the optimizer's state beside them.  Then
  op "embed_fwd"   taw_embed_fwd                            rows of the table by token id, scaled
  op "embed_bwd"   taw_embed_bwd                            its gradient: rows of dx summed by token id into the shard
  op "loss_train"  taw_loss_fwd_bwd                         cross entropy and the gradient of the logits in one pass
  op "loss_eval"   taw_loss_fwd                             the loss alone
  op "loss_bwd"    taw_loss_bwd                             the gradient from a saved lse and a gradient of every row's loss
  op "clip"        taw_grad_norm + taw_grad_clip            norm over many tensors, gradients scaled in place
  op "step"        taw_grad_norm + taw_optimizer_step_clipped   the same inside the owner's update: no pass for the scaling
Outside `own` the same is computed in elementary torch operations in 32 bits (sums of squares, and of the rows' losses, in 64).
"""
import math

import numpy as np
import torch

own = False

BETA1, BETA2, ADAM_EPS, DECAY, LR, STEP = 0.9, 0.95, 1e-8, 0.1, 3e-4, 10


def _embed(name, op, dtype, T, H, V, ids, scale=1.0, padding="none", accumulate=False):
    return {"name": name, "op": op, "dtype": dtype, "T": T, "H": H, "V": V, "ids": ids, "scale": scale, "padding": padding,
            "accumulate": accumulate}


def _loss(name, op, dtype, grad, T, V, rows, labels, smoothing=0.0, z=0.0, mean=True, masked=False):
    return {"name": name, "op": op, "dtype": dtype, "grad": grad, "T": T, "V": V, "rows": rows, "labels": labels,
            "smoothing": smoothing, "z": z, "mean": mean, "masked": masked}


def listed():
    return [
        # the tiny fp32 model that a user runs first: 128 tokens, 64 wide; the launch is all it costs
        _embed("embed_fwd_f32_t128_h64", "embed_fwd", "f32", 128, 64, 509, "i64"),
        # the 2048-wide model of the paper's table at its own micro-batch (65536 tokens), rows scaled by sqrt(H)
        _embed("embed_fwd_h2048_t65536", "embed_fwd", "bf16", 65536, 2048, 32000, "i32", scale=math.sqrt(2048)),
        # the 1024-wide model on three sequences of 1501 that were padded with one row of the table, an odd vocabulary; one of
        # several micro-batches into one shard
        _embed("embed_bwd_h1024_t4503_padded", "embed_bwd", "bf16", 4503, 1024, 32001, "i64", padding="row", accumulate=True),
        # the 4096-wide model at long context, the first micro-batch: the shard is overwritten
        _embed("embed_bwd_h4096_t32768", "embed_bwd", "bf16", 32768, 4096, 32000, "i32"),
        # a training step's loss at 8192 tokens
        _loss("loss_train_v32000_t8192", "loss_train", "bf16", "bf16", 8192, 32000, "tight", "i32"),
        # a large vocabulary; fp32 logits as the product's epilogue leaves them, a bf16 gradient for the next product, z-loss
        _loss("loss_train_v131072_t4096_f32", "loss_train", "f32", "bf16", 4096, 131072, "tight", "i64", z=1e-4),
        # evaluation on one short sequence, an odd vocabulary whose rows start anywhere
        _loss("loss_eval_v50001_t333", "loss_eval", "bf16", "bf16", 333, 50001, "tight", "i64"),
        # weights of its own for every token (what a policy gradient gives), label smoothing, rows padded to a multiple of 64
        _loss("loss_bwd_v32003_t2048", "loss_bwd", "bf16", "bf16", 2048, 32003, "padded", "i32", smoothing=0.1, z=1e-4, mean=False),
        # the tiny fp32 model's gradients, one tensor for each weight
        {"name": "clip_h64_9_tensors", "op": "clip", "dtype": "f32", "layers": 1, "H": 64, "I": 176, "V": 509, "split": True,
         "max_norm": 1.0, "grad_scale": 1.0},
        # the whole 1024-wide model: 24 layers' shards, embedding, head and the last norm's gain
        {"name": "clip_h1024_24_layers", "op": "clip", "dtype": "f32", "layers": 24, "H": 1024, "I": 2816, "V": 32000, "split": True,
         "max_norm": 1.0, "grad_scale": 0.25},
        # the owner's update of a small bf16 layer, where nothing is clipped
        {"name": "step_h256", "op": "step", "dtype": "bf16", "layers": 1, "H": 256, "I": 392, "V": 0, "split": False,
         "max_norm": 1e6, "grad_scale": 1.0},
        # the owner's update of the 7B-wide layer, gradients of four micro-batches
        {"name": "step_h4096", "op": "step", "dtype": "bf16", "layers": 1, "H": 4096, "I": 11008, "V": 0, "split": False,
         "max_norm": 1.0, "grad_scale": 0.25},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: tokens from 1 to 65536, rows of 8 to 8192, vocabularies of 2 to 262144, models of one to forty layers."""
    op = rng.choice(["embed_fwd", "embed_bwd", "loss_train", "loss_train", "loss_eval", "loss_bwd", "clip", "step"])
    while True:
        if op.startswith("embed"):
            dtype = rng.choice(["bf16", "bf16", "f32"])
            H = rng.choice([128 * _log_int(rng, 1, 64), 8 * _log_int(rng, 1, 512), _log_int(rng, 8, 2000)])
            c = _embed("", op, dtype, _log_int(rng, 1, 65536), H, _log_int(rng, 100, 262144), rng.choice(["i32", "i64"]),
                       rng.choice([1.0, 1.0, math.sqrt(H)]), rng.choice(["none", "none", "row", "outside"]), rng.random() < 0.5)
        elif op.startswith("loss"):
            dtype, grad = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
            V = rng.choice([64 * _log_int(rng, 1, 4096), _log_int(rng, 2, 262144), _log_int(rng, 20000, 160000)])
            c = _loss("", op, dtype, grad, _log_int(rng, 1, 65536), V, rng.choice(["tight", "padded"]), rng.choice(["i32", "i64"]),
                      rng.choice([0.0, 0.0, 0.1]), rng.choice([0.0, 1e-4]), rng.random() < 0.7, rng.random() < 0.15)
            if c["masked"]:
                c["smoothing"] = 0.0      # a masked class with a share of the target has an infinite loss
        else:
            H = 64 * _log_int(rng, 1, 128)
            c = {"op": op, "dtype": "f32" if H < 256 else rng.choice(["f32", "bf16"]), "layers": _log_int(rng, 1, 40) if op == "clip" else 1,
                 "H": H, "I": 8 * _log_int(rng, max(1, H // 4), H // 2), "V": _log_int(rng, 100, 131072) if op == "clip" else 0,
                 "split": op == "clip" and rng.random() < 0.6, "max_norm": math.exp(rng.uniform(math.log(0.1), math.log(1e5))),
                 "grad_scale": rng.choice([1.0, 0.25])}
        c.pop("name", None)
        if work(c)["bytes"] <= 6.0e9:
            return c


# ----------------------------------------------------------------------------- states
def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _stride(c):
    """elements from row to row of the logits, and classes in a row of their gradient: V, or V rounded up to 64"""
    return c["V"] if c["rows"] == "tight" else -(-c["V"] // 64) * 64


def _tensor_sizes(c):
    """elements of the gradient tensors of a model: the layers' weights one by one or as one shard each, embedding, head, last gain"""
    H, I, V = c["H"], c["I"], c["V"]
    parts = [H, 3 * H * H, H * H, H, 2 * I * H, H * I]
    sizes = (parts if c["split"] else [sum(-(-n // 128) * 128 for n in parts)]) * c["layers"]
    return sizes + ([V * H, V * H, H] if V else [])


def _token_ids(c, gen):
    """ids as text has them: the n-th most frequent token about 1/n as often as the first"""
    T, V = c["T"], c["V"]
    u = torch.rand(T, generator=gen, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
    if c["padding"] != "none":            # the last third of the tokens
        ids[T - T // 3:] = V - 1 if c["padding"] == "row" else -1
    return ids.to(torch.int32 if c["ids"] == "i32" else torch.int64)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(shape, std, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)

    s = {"case": c, "stream": torch.cuda.current_stream()}
    if c["op"].startswith("embed"):
        dt = _dt(c["dtype"])
        s["ids"] = _token_ids(c, gen)
        if c["op"] == "embed_fwd":
            s["table"] = normal((c["V"], c["H"]), 0.02, dt)
            s["x"] = torch.empty((c["T"], c["H"]), dtype=dt, device="cuda")
        else:
            s["dx"] = normal((c["T"], c["H"]), 1.0, dt)
            s["G"] = normal((c["V"], c["H"]), 1.0, torch.float32)
    elif c["op"].startswith("loss"):
        dt, T, V, ld = _dt(c["dtype"]), c["T"], c["V"], _stride(c)
        logits = normal((T, ld), 1.5, dt)
        labels = torch.randint(0, V, (T,), generator=gen, device="cuda")
        right = torch.rand(T, generator=gen, device="cuda") < 0.6
        if c["masked"]:                   # a grammar that allows a tenth of the classes, and always the label
            logits[:, :V].masked_fill_(torch.rand((T, V), generator=gen, device="cuda") < 0.9, -math.inf)
            logits.scatter_(1, labels[:, None], torch.zeros((T, 1), dtype=dt, device="cuda"))
        logits.scatter_add_(1, labels[:, None], (right * 8.0).to(dt)[:, None])      # what a trained model gives most labels
        labels[torch.rand(T, generator=gen, device="cuda") < 0.1] = -100            # prompts and padding
        s["logits"], s["labels"] = logits, labels.to(torch.int32 if c["labels"] == "i32" else torch.int64)
        s["loss"] = torch.empty(2, dtype=torch.float32, device="cuda")
        s["rows"] = torch.empty(T, dtype=torch.float32, device="cuda")
        s["lse"] = torch.empty(T, dtype=torch.float32, device="cuda")
        if c["op"] != "loss_eval":
            s["dlogits"] = torch.empty((T, ld), dtype=_dt(c["grad"]), device="cuda")
        if c["op"] == "loss_bwd":         # what the forward of these logits left
            l = logits[:, :V].double()
            s["lse"] = torch.logsumexp(l, 1).float()
            s["dloss"] = normal((T,), 1.0, torch.float32)
    else:
        sizes = _tensor_sizes(c)
        starts = np.concatenate([[0], np.cumsum([-(-n // 128) * 128 for n in sizes])])
        s["G"] = normal((int(starts[-1]),), 1e-2, torch.float32)
        if c["op"] == "clip" and c["dtype"] == "bf16":
            s["G"] = s["G"].to(torch.bfloat16)
        s["grads"] = [s["G"][int(a):int(a) + n] for a, n in zip(starts, sizes)]
        if c["op"] == "step":
            n = s["G"].numel()
            s.update(master=normal(n, 0.02, torch.float32), m=normal(n, 1e-3, torch.float32), v=normal(n, 1e-3, torch.float32).square_())
            s["chunk"] = s["master"].to(_dt(c["dtype"]))
    if own:
        _handles(s)
    return s


def _handles(s):
    """the descriptors and workspaces that a training program makes once"""
    import paper_2511_09741_amd.binding as taw
    c = s["case"]
    code = {"f32": taw.TAW_F32, "bf16": taw.TAW_BF16}
    s["taw"] = taw

    def buffer(nbytes):
        return torch.empty(max(16, nbytes), dtype=torch.uint8, device="cuda")

    if c["op"].startswith("embed"):
        s["desc"] = taw.make_embed_desc(code[c["dtype"]], c["T"], c["H"], c["V"], scale=c["scale"],
                                        flags=taw.TAW_ACCUMULATE if c["accumulate"] else 0)
        if c["op"] == "embed_bwd":
            s["ws"] = buffer(taw.taw_embed_bwd_workspace_bytes(s["desc"]))
    elif c["op"].startswith("loss"):
        s["desc"] = taw.make_loss_desc(code[c["dtype"]], c["T"], c["V"], grad_dtype=code[c["grad"]], ld=_stride(c), ld_grad=_stride(c),
                                       V_pad=_stride(c), label_smoothing=c["smoothing"], z_loss=c["z"], grad_scale=1.0,
                                       flags=taw.TAW_LOSS_MEAN if c["mean"] else 0)
        s["ws"] = buffer(taw.taw_loss_workspace_bytes(s["desc"]))
    else:
        if c["op"] == "step" and c["dtype"] == "f32":
            s["chunk"] = s["master"].clone()      # a buffer of its own also where the types are the same
        s["list"] = taw.make_tensor_list(s["grads"])
        s["state"] = taw.new_clip_state()
        s["ws"] = buffer(taw.taw_grad_norm_workspace_bytes(s["list"]))


# ----------------------------------------------------------------------------- one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    taw, c, st = s["taw"], s["case"], s["stream"]
    op = c["op"]
    if op == "embed_fwd":
        taw.taw_embed_fwd(s["desc"], s["ids"], s["table"], s["x"], st)
        return {"x": s["x"]}
    if op == "embed_bwd":
        taw.taw_embed_bwd(s["desc"], s["ids"], s["dx"], s["G"], s["ws"], stream=st)
        return {"G": s["G"]}
    if op == "loss_train":
        taw.taw_loss_fwd_bwd(s["desc"], s["logits"], s["labels"], s["loss"], s["rows"], s["lse"], s["dlogits"], s["ws"], stream=st)
        return {k: s[k] for k in ("loss", "rows", "lse", "dlogits")}
    if op == "loss_eval":
        taw.taw_loss_fwd(s["desc"], s["logits"], s["labels"], s["loss"], s["rows"], s["lse"], s["ws"], stream=st)
        return {k: s[k] for k in ("loss", "rows", "lse")}
    if op == "loss_bwd":
        taw.taw_loss_bwd(s["desc"], s["logits"], s["labels"], s["lse"], s["dloss"], s["dlogits"], st)
        return {"dlogits": s["dlogits"]}
    taw.taw_grad_norm(s["list"], c["max_norm"], c["grad_scale"], s["state"], s["ws"], stream=st)
    if op == "clip":
        taw.taw_grad_clip(s["list"], s["state"], st)
        return {"G": s["G"], "norm": s["state"].norm, "coef": s["state"].coef, "nonfinite": s["state"].nonfinite}
    taw.taw_optimizer_step_clipped(s["state"], s["chunk"], taw.TAW_BF16 if c["dtype"] == "bf16" else taw.TAW_F32, s["master"], s["m"], s["v"],
                                   s["G"], s["G"].numel(), step=STEP, lr=LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=DECAY,
                                   grad_scale=c["grad_scale"], zero_grad=False, stream=st)
    return {**{k: s[k] for k in ("chunk", "master", "m", "v")}, "norm": s["state"].norm, "coef": s["state"].coef, "nonfinite": s["state"].nonfinite}


def _run_plain(s):
    c = s["case"]
    op, dt = c["op"], _dt(c["dtype"])
    if op.startswith("embed"):
        ids = s["ids"]
        inside = (ids >= 0) & (ids < c["V"])
        at = torch.where(inside, ids, 0).long()
        if op == "embed_fwd":
            x = s["table"][at].float() * c["scale"]
            return {"x": torch.where(inside[:, None], x, 0.0).to(dt)}
        rows = torch.where(inside[:, None], s["dx"].float(), 0.0)
        dw = torch.zeros_like(s["G"]).index_add_(0, at, rows) * c["scale"]
        if c["accumulate"]:
            s["G"] += dw
        else:
            s["G"].copy_(dw)
        return {"G": s["G"]}
    if op.startswith("loss"):
        return _loss_plain(s)
    scale = c["grad_scale"]
    squares = torch.stack([g.float().square().sum(dtype=torch.float64) for g in s["grads"]]).sum()
    norm = (squares.sqrt() * abs(scale)).float()
    nonfinite = ~torch.isfinite(norm)
    coef = torch.where(nonfinite, 0.0, torch.where(norm > c["max_norm"], c["max_norm"] / norm, 1.0))
    told = {"norm": norm, "coef": coef, "nonfinite": nonfinite.to(torch.int32)}
    if op == "clip":
        for g in s["grads"]:
            g.copy_(torch.where(nonfinite, g.float(), g.float() * coef))
        return {"G": s["G"], **told}
    g = s["G"] * (scale * coef)
    m, v, w = s["m"], s["v"], s["master"]
    m1 = BETA1 * m + (1 - BETA1) * g
    v1 = BETA2 * v + (1 - BETA2) * g * g
    w1 = w - LR * ((m1 / (1 - BETA1 ** STEP)) / ((v1 / (1 - BETA2 ** STEP)).sqrt() + ADAM_EPS) + DECAY * w)
    s["m"], s["v"], s["master"] = torch.where(nonfinite, m, m1), torch.where(nonfinite, v, v1), torch.where(nonfinite, w, w1)
    s["chunk"] = s["master"].to(dt)
    return {**{k: s[k] for k in ("chunk", "master", "m", "v")}, **told}


def _loss_plain(s):
    c = s["case"]
    V, eps, z = c["V"], c["smoothing"], c["z"]
    l = s["logits"][:, :V].float()
    labels = s["labels"]
    counted = (labels >= 0) & (labels < V)
    at = torch.where(counted, labels, 0).long()[:, None]
    if c["op"] == "loss_bwd":
        lse, upstream = s["lse"], torch.where(counted, s["dloss"], 0.0)
    else:
        top = l.max(1, keepdim=True).values
        lse = (top + torch.log(torch.exp(l - top).sum(1, keepdim=True)))[:, 0]
        rows = lse - (1 - eps) * l.gather(1, at)[:, 0]
        if eps:
            rows = rows - eps * l.mean(1)
        if z:
            rows = rows + z * lse.square()
        rows = torch.where(counted, rows, 0.0)
        count = counted.sum()
        share = 1.0 / torch.clamp(count, min=1) if c["mean"] else torch.ones((), device=l.device)
        loss = rows.sum(dtype=torch.float64) * share
        out = {"loss": torch.stack([loss.float(), count.float()]), "rows": rows, "lse": torch.where(counted, lse, 0.0)}
        if c["op"] == "loss_eval":
            return out
        upstream = torch.where(counted, share.float(), 0.0)
    d = torch.exp(l - lse[:, None])
    if z:
        d = d * (1 + 2 * z * lse)[:, None]
    if eps:
        d = d - eps / V
    d.scatter_add_(1, at, torch.full_like(at, -(1 - eps), dtype=torch.float32))
    d = (d * upstream[:, None]).to(_dt(c["grad"]))
    d = torch.nn.functional.pad(d, (0, _stride(c) - V))
    if c["op"] == "loss_bwd":
        return {"dlogits": d}
    return {**out, "dlogits": d}


# ----------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    global own
    c, was = case, own
    own = False
    s = prepare(case, seed)
    own = was
    if c["op"].startswith("embed"):
        ids = s["ids"].long()
        order = torch.argsort(ids, stable=True)
        order = order[(ids[order] >= 0) & (ids[order] < c["V"])]
        if c["op"] == "embed_fwd":
            x = torch.zeros((c["T"], c["H"]), dtype=torch.float64, device="cuda")
            x[order] = s["table"].double()[ids[order]] * c["scale"]
            return {"x": x}
        G = s["G"].double() if c["accumulate"] else torch.zeros(s["G"].shape, dtype=torch.float64, device="cuda")
        tokens, counts = torch.unique_consecutive(ids[order], return_counts=True)
        if not tokens.numel():
            return {"G": G}
        ends = torch.cumsum(counts, 0)
        for a in range(0, c["H"], 512):                     # differences of running sums, some columns at a time
            run_ = torch.cumsum(s["dx"][:, a:a + 512].double()[order], 0)
            sums = run_[ends - 1]
            sums[1:] = sums[1:] - run_[ends[:-1] - 1]
            G[tokens, a:a + 512] += c["scale"] * sums
        return {"G": G}
    if c["op"].startswith("loss"):
        T, V, ld, eps, z = c["T"], c["V"], _stride(c), c["smoothing"], c["z"]
        labels = s["labels"].long()
        counted = torch.isin(labels, torch.arange(V, device="cuda"))
        n = int(counted.sum())
        lse = torch.zeros(T, dtype=torch.float64, device="cuda")
        rows = torch.zeros(T, dtype=torch.float64, device="cuda")
        d = None if c["op"] == "loss_eval" else torch.zeros((T, ld), dtype=torch.float64, device="cuda")
        for a in range(0, T, 1024):
            b = min(a + 1024, T)
            l = s["logits"][a:b, :V].double()
            k = counted[a:b]
            target = torch.full_like(l, eps / V)
            target[k, labels[a:b][k]] += 1 - eps
            logp = torch.log_softmax(l, 1)
            lse[a:b] = torch.logsumexp(l, 1)
            along = torch.where(target > 0, target * logp, 0.0).sum(1)
            rows[a:b] = torch.where(k, -along + z * lse[a:b] ** 2, 0.0)
            if d is not None:
                if c["op"] == "loss_bwd":
                    w = torch.where(k, s["dloss"][a:b].double(), 0.0)
                    p = torch.exp(l - s["lse"][a:b].double()[:, None])
                    zl = s["lse"][a:b].double()
                else:
                    w, p, zl = k.double() / (max(n, 1) if c["mean"] else 1), torch.exp(logp), lse[a:b]
                d[a:b, :V] = w[:, None] * (p * (1 + 2 * z * zl)[:, None] - target)
        if c["op"] == "loss_bwd":
            return {"dlogits": d}
        total = rows.sum() / (max(n, 1) if c["mean"] else 1)
        out = {"loss": torch.stack([total, torch.tensor(float(n), dtype=torch.float64, device="cuda")]), "rows": rows, "lse": torch.where(counted, lse, 0.0)}
        return out if d is None else {**out, "dlogits": d}
    norm = abs(c["grad_scale"]) * math.sqrt(sum(float(torch.linalg.vector_norm(g, dtype=torch.float64)) ** 2 for g in s["grads"]))
    coef = min(1.0, c["max_norm"] / norm) if norm else 1.0
    told = {"norm": torch.tensor(norm, dtype=torch.float64), "coef": torch.tensor(coef, dtype=torch.float64), "nonfinite": None}
    if c["op"] == "clip":
        G = s["G"].double()
        at = 0
        for n in _tensor_sizes(c):
            G[at:at + n] *= coef
            at += -(-n // 128) * 128
        return {"G": G, **told}
    g = s["G"].double() * (c["grad_scale"] * coef)
    m = s["m"].double().lerp_(g, 1 - BETA1)
    v = s["v"].double().lerp_(g.square_(), 1 - BETA2)
    w = s["master"].double()
    w = w * (1 - LR * DECAY) - LR * (m / (1 - BETA1 ** STEP)) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + ADAM_EPS)
    return {"chunk": w, "master": w, "m": m, "v": v, **told}


# ----------------------------------------------------------------------------- what a pass cannot do without
def _distinct(c):
    """how many different rows of the table T such ids are expected to name"""
    tokens = c["T"] - (c["T"] // 3 if c["padding"] != "none" else 0)
    v = np.arange(1, c["V"] + 1, dtype=np.float64)
    p = np.log1p(1.0 / v) / math.log(c["V"] + 1.0)
    return float(np.sum(-np.expm1(tokens * np.log1p(-p)))) if c["V"] > 1 else 1.0


def work(case):
    c = case
    if c["op"].startswith("embed"):
        e, T, H = (2 if c["dtype"] == "bf16" else 4), c["T"], c["H"]
        used = T - T // 3 if c["padding"] == "outside" else T
        ids = T * (4 if c["ids"] == "i32" else 8)
        if c["op"] == "embed_fwd":        # the rows that are named in, x out
            return {"bytes": float(ids + e * H * (_distinct(c) + T)), "flops": float(T * H)}
        shard = 8 * H * _distinct(c) if c["accumulate"] else 4 * H * c["V"]      # the rows that are named read and written, or all written
        return {"bytes": float(ids + e * H * used + shard), "flops": float(used * H)}
    if c["op"].startswith("loss"):
        T, V = c["T"], c["V"]
        rows = T * (4 if c["labels"] == "i32" else 8) + 8 * T
        out = 0 if c["op"] == "loss_eval" else T * _stride(c) * (2 if c["grad"] == "bf16" else 4)
        return {"bytes": float(T * V * (2 if c["dtype"] == "bf16" else 4) + out + rows), "flops": float(T * V * (4 if out else 3))}
    n = float(sum(_tensor_sizes(c)))
    if c["op"] == "clip":                 # each gradient read, and written again
        return {"bytes": n * (8 if c["dtype"] == "f32" else 4), "flops": 3 * n}
    # G, m, v, master read; m, v, master and the chunk written
    return {"bytes": n * (16 + 12 + (2 if c["dtype"] == "bf16" else 4)), "flops": 16 * n}
