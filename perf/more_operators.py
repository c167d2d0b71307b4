"""A decoder's operators beside its linear layers, as cases that can be timed and compared: the output layer
with its loss, norms, and the token embedding.

A case is one pass, called as a training step or a server calls it:

* ``xent``   the cross entropy of z = x W^T, x [m, k], W [n, k], against targets [m]: per-row losses
             ``lse_i - z_i,t_i``, lse_i = log sum_j exp z_ij (0 for a row whose target is -100), with ``mean`` their
             mean over the other rows, and the lse; with ``grad`` the gradients dx and dW of that mean, or of the losses weighted by
             a number per row;
* ``norm``   y = (x - mean) / sqrt(var + eps) w + b per row (``layer``), or x / sqrt(mean x^2 + eps) w (``rms``); with
             ``grad`` also dx, dw and db from dy;
* ``embed``  y_i = scale T[id_i] for ids [m] and a table [n, k]; with ``grad`` also dT, whose rows are
             scale times the sums of the dy_i of their id (zeros where no id, and for a padding id).

The plain forms compute in fp32 and round each output once.  Widths and vocabularies are those of the workloads'
stacks (768/50304, 1024, 1536/151936, 2048/128256, 4096/128256), or odd ones.
"""
from __future__ import annotations

import math

import torch

own = False     # False: the plain forms; True: the framework's operators

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
EPS = {"layer": 1e-5, "rms": 1e-6}
IGNORE = -100
MAX_XENT = 4096 * 128256 * 2048
MAX_NORM = 16384 * 4096
MAX_EMBED = 128256 * 2048


# ---------------------------------------------------------------- the cases
def _case(op, name=None, **kw):
    c = dict(op=op, dtype="bf16", wdtype="bf16", m=1, n=1, k=1, grad=False, mean=False, ignored=0.0, kind="rms",
             bias=False, scale=1.0, padding=-1)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one token's log probability under the 768-wide stack: the head's bytes bound it
        _case("xent", "xent_token", m=1, n=50304, k=768),
        # an evaluation batch scored by the 1536-wide decoder: losses alone
        _case("xent", "xent_score", m=512, n=151936, k=1536),
        # a training step of the 2048-wide decoder, 8 x 512 tokens, mean loss: the largest
        _case("xent", "xent_train", m=4096, n=128256, k=2048, grad=True, mean=True),
        # the 4096-wide decoder's fine-tuning batch: half of the rows are prompts without a target, the others weighted
        _case("xent", "xent_prompts", m=2048, n=128256, k=4096, grad=True, ignored=0.5),
        # an fp32 model of odd sizes
        _case("xent", "xent_odd_f32", dtype="f32", wdtype="f32", m=515, n=32003, k=769, grad=True, mean=True, ignored=0.1),
        # the next token's row before a product of the 4096-wide decoder: one launch's latency
        _case("norm", "norm_token", m=1, n=4096, wdtype="f32"),
        # the vision tower's layer norm over eight images of 257 patches, forward and backward
        _case("norm", "norm_layer", m=2056, n=1024, kind="layer", bias=True, grad=True),
        # the 4096-wide decoder's norm over 16384 tokens, weights kept in fp32
        _case("norm", "norm_rms_large", m=16384, n=4096, wdtype="f32", grad=True),
        # odd sizes in fp32: rows off any vector boundary
        _case("norm", "norm_odd_f32", dtype="f32", wdtype="f32", m=1999, n=1537, kind="layer", bias=True, grad=True),
        # next tokens of four sequences
        _case("embed", "embed_tokens", m=4, n=128256, k=4096),
        # a training step of the 2048-wide decoder: rows in, the whole table's gradient out
        _case("embed", "embed_train", m=4096, n=128256, k=2048, grad=True),
        # an fp32 table of odd sizes read as bf16, scaled, with a padding id
        _case("embed", "embed_odd", wdtype="f32", m=5003, n=32003, k=1025, grad=True, scale=32.0, padding=0),
    ]


def _size(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if v >= 64 and rng.random() < 0.5:
        v -= v % 32        # half of the sizes are a layer's, half are odd
    return min(max(v, lo), hi)


def draw(rng):
    op = rng.choice(("xent", "xent", "norm", "embed"))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    c = _case(op, dtype=dtype, wdtype=dtype, grad=rng.random() < 0.7)
    if op == "xent":
        n, k = _size(rng, 500, 151936), _size(rng, 64, 4096)
        most = MAX_XENT // (n * k) // (4 if dtype == "f32" else 1)
        c.update(m=max(1, min(_size(rng, 1, 8192), most)), n=n, k=k, mean=rng.random() < 0.5,
                 ignored=rng.choice((0.0, 0.1, 0.6)))
        return c
    if rng.random() < 0.4:
        c["wdtype"] = rng.choice(("f32", "bf16"))
    if op == "norm":
        n = _size(rng, 1, 16384)
        kind = rng.choice(("layer", "rms"))
        c.update(n=n, m=max(1, min(_size(rng, 1, 16384), MAX_NORM // n)), kind=kind, bias=kind == "layer" and rng.random() < 0.7)
        return c
    k = _size(rng, 16, 4096)
    n = max(64, min(_size(rng, 64, 151936), MAX_EMBED // k))
    c.update(k=k, n=n, m=max(1, min(_size(rng, 1, 65536), MAX_EMBED // k)), scale=rng.choice((1.0, math.sqrt(k))),
             padding=rng.choice((-1, 0)))
    return c


def work(case):
    op, m, n, k, b, wb = case["op"], case["m"], case["n"], case["k"], BYTES[case["dtype"]], BYTES[case["wdtype"]]
    if op == "xent":
        nbytes = b * (m * k + n * k) * (2 if case["grad"] else 1) + 8 * m + 4 * (1 + m if case["mean"] else 2 * m)
        if case["grad"] and not case["mean"]:
            nbytes += 4 * m
        return {"bytes": nbytes, "flops": 2 * m * n * k * (3 if case["grad"] else 1)}
    if op == "norm":
        params = wb * n * (1 + case["bias"])
        return {"bytes": (b * m * n * 4 + 2 * params) if case["grad"] else b * m * n * 2 + params, "flops": 0}
    rows = min(m, n)
    nbytes = wb * rows * k + b * m * k + 8 * m
    return {"bytes": nbytes + (b * m * k + wb * n * k if case["grad"] else 0), "flops": 0}


# ---------------------------------------------------------------- the inputs
def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    dt, wdt, m, n, k, op = DTYPES[case["dtype"]], DTYPES[case["wdtype"]], case["m"], case["n"], case["k"], case["op"]

    def normal(rows, cols, std, wide=False):
        x = torch.randn(rows, cols, generator=gen, device=DEV, dtype=torch.float32).mul_(std)
        if wide:
            x[:, ::97] *= 12.0      # some channels of a residual stream are far larger than the others
        return x

    def uniform(size):
        return torch.rand(size, generator=gen, device=DEV)

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device=DEV)

    s = dict(case=case)
    if op == "xent":
        w = normal(n, k, 0.02).to(wdt)
        t = torch.randint(0, n, (m,), generator=gen, device=DEV)
        # rows lean towards their target's row of W, some hardly and some so far that its probability is near one
        lean = uniform((m, 1)) * (1.3 * math.log(n) / (0.02 ** 2 * k))
        x = (normal(m, k, 0.9) + lean * w[t].float()).to(dt)
        ignored = uniform(m) < case["ignored"]
        ignored[0] = False
        t = torch.where(ignored, torch.full_like(t, IGNORE), t)
        s.update(x=x, w=w, t=t, loss=empty(m), lse=empty(m), totals=empty(3) if case["mean"] else None, weight=None, dx=None, dw=None)
        if case["grad"]:
            s.update(dx=empty(m, k, dtype=dt), dw=empty(n, k, dtype=wdt))
            if not case["mean"]:
                s["weight"] = uniform(m) + 0.5
    elif op == "norm":
        s.update(x=normal(m, n, 1.0, wide=True).add_(0.1).to(dt), w=(normal(1, n, 0.05).view(n) + 1.0).to(wdt), b=None,
                 y=empty(m, n, dtype=dt), mean=None, rstd=None)
        if case["bias"]:
            s["b"] = normal(1, n, 0.02).view(n).to(wdt)
        if case["grad"]:
            s.update(dy=normal(m, n, 1e-3).to(dt), rstd=empty(m), dx=empty(m, n, dtype=dt), dw=empty(n, dtype=wdt),
                     mean=empty(m) if case["kind"] == "layer" else None, db=empty(n, dtype=wdt) if case["bias"] else None)
    else:
        # ids as they occur in text: the r-th most frequent one about as often as 1 / r
        ids = torch.exp(uniform(m).double() * math.log(n)).long().sub_(1).clamp_(0, n - 1)
        s.update(table=normal(n, k, 0.02).to(wdt), ids=ids, y=empty(m, k, dtype=dt))
        if case["grad"]:
            s.update(dy=normal(m, k, 1e-3).to(dt), dtable=empty(n, k, dtype=wdt))
    return s


# ---------------------------------------------------------------- the plain forms
def _plain_xent(s, case):
    x, w, t = s["x"].float(), s["w"].float(), s["t"]
    z = x @ w.t()
    has = t != IGNORE
    at = torch.where(has, t, torch.zeros_like(t))[:, None]
    top = z.amax(dim=1, keepdim=True)
    p = torch.exp(z - top)
    total = p.sum(dim=1, keepdim=True)
    lse = torch.log(total) + top
    loss = torch.where(has, (lse - z.gather(1, at))[:, 0], torch.zeros_like(top[:, 0]))
    del z
    count = has.sum()
    out = {"loss": loss.sum() / count if case["mean"] else loss, "lse": lse[:, 0]}
    if not case["grad"]:
        return out
    p /= total
    p[torch.arange(p.shape[0], device=p.device), at[:, 0]] -= 1.0
    g = has.float() / count if case["mean"] else has.float() * s["weight"]
    p *= g[:, None]
    out["dx"] = (p @ w).to(s["x"].dtype)
    out["dw"] = (p.t() @ x).to(s["w"].dtype)
    return out


def _plain_norm(s, case):
    x, w = s["x"].float(), s["w"].float()
    if case["kind"] == "layer":
        x = x - x.mean(dim=1, keepdim=True)
    r = 1.0 / torch.sqrt((x * x).mean(dim=1, keepdim=True) + EPS[case["kind"]])
    xh = x * r
    y = xh * w
    if s["b"] is not None:
        y = y + s["b"].float()
    out = {"y": y.to(s["x"].dtype)}
    if not case["grad"]:
        return out
    dy = s["dy"].float()
    d = dy * w
    dx = d - xh * (d * xh).mean(dim=1, keepdim=True)
    if case["kind"] == "layer":
        dx = dx - d.mean(dim=1, keepdim=True)
    out["dx"] = (dx * r).to(s["x"].dtype)
    out["dw"] = (dy * xh).sum(dim=0).to(s["w"].dtype)
    if s["b"] is not None:
        out["db"] = dy.sum(dim=0).to(s["w"].dtype)
    return out


def _plain_embed(s, case):
    ids, dt, wdt = s["ids"], s["y"].dtype, s["table"].dtype
    out = {"y": (s["table"][ids].float() * case["scale"]).to(dt)}
    if case["grad"]:
        dy = s["dy"].float() * (ids != case["padding"])[:, None]
        dtable = torch.zeros(s["table"].shape, dtype=torch.float32, device=dy.device).index_add_(0, ids, dy)
        out["dtable"] = (dtable * case["scale"]).to(wdt)
    return out


def _plain(s):
    case = s["case"]
    return {"xent": _plain_xent, "norm": _plain_norm, "embed": _plain_embed}[case["op"]](s, case)


# ---------------------------------------------------------------- the framework's operators
def _own(s):
    import paper_2609_33437_amd as smat

    case, op = s["case"], s["case"]["op"]
    if op == "xent":
        smat.smat_linear_xent(s["x"], s["w"], s["t"], s["loss"], s["lse"], totals=s["totals"], ignore_index=IGNORE)
        out = {"loss": s["totals"][2] if case["mean"] else s["loss"], "lse": s["lse"]}
        if case["grad"]:
            smat.smat_linear_xent_grad(s["x"], s["w"], s["t"], s["lse"], dx=s["dx"], dw=s["dw"], row_scale=s["weight"],
                                       totals=s["totals"], ignore_index=IGNORE)
            out.update(dx=s["dx"], dw=s["dw"])
        return out
    if op == "norm":
        kind = smat.SMAT_NORM_LAYER if case["kind"] == "layer" else smat.SMAT_NORM_RMS
        smat.smat_norm(s["x"], s["y"], weight=s["w"], bias=s["b"], kind=kind, eps=EPS[case["kind"]], mean=s["mean"],
                       rstd=s["rstd"])
        out = {"y": s["y"]}
        if case["grad"]:
            smat.smat_norm_grad(s["dy"], s["x"], s["rstd"], weight=s["w"], mean=s["mean"], kind=kind, dx=s["dx"],
                                dw=s["dw"], db=s["db"])
            out.update(dx=s["dx"], dw=s["dw"])
            if s["db"] is not None:
                out["db"] = s["db"]
        return out
    smat.smat_embed(s["table"], s["ids"], s["y"], scale=case["scale"])
    out = {"y": s["y"]}
    if case["grad"]:
        smat.smat_embed_grad(s["dy"], s["ids"], s["dtable"], scale=case["scale"], padding_idx=case["padding"])
        out["dtable"] = s["dtable"]
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- the definition in 64 bits
def _exact_xent(case, s):
    x, w, t = s["x"].double(), s["w"].double(), s["t"]
    z = torch.mm(x, w.t())
    rows = torch.nonzero(t >= 0)[:, 0]
    lse = torch.logsumexp(z, dim=1)
    loss = torch.zeros(case["m"], dtype=torch.float64, device=DEV)
    loss[rows] = lse[rows] - z[rows, t[rows]]
    out = {"loss": loss.sum() / rows.numel() if case["mean"] else loss, "lse": lse}
    if case["grad"]:
        g = torch.zeros_like(loss)
        g[rows] = 1.0 / rows.numel() if case["mean"] else s["weight"].double()[rows]
        dz = z.sub_(lse[:, None]).exp_().mul_(g[:, None])
        dz[rows, t[rows]] -= g[rows]
        out.update(dx=torch.mm(dz, w), dw=torch.mm(dz.t(), x))
    return out


def _exact_norm(case, s):
    x, w = s["x"].double(), s["w"].double()
    layer, n = case["kind"] == "layer", case["n"]
    mu = x.sum(1, keepdim=True) / n if layer else torch.zeros(case["m"], 1, dtype=torch.float64, device=DEV)
    sigma = torch.sqrt(((x - mu) ** 2).sum(1, keepdim=True) / n + EPS[case["kind"]])
    unit = (x - mu) / sigma
    out = {"y": unit * w + (s["b"].double() if case["bias"] else 0.0)}
    if case["grad"]:
        dy = s["dy"].double()
        du = dy * w
        along = (du * unit).sum(1, keepdim=True) / n
        dx = du - unit * along - (du.sum(1, keepdim=True) / n if layer else 0.0)
        out.update(dx=dx / sigma, dw=(dy * unit).sum(0))
        if case["bias"]:
            out["db"] = dy.sum(0)
    return out


def _exact_embed(case, s):
    ids, scale = s["ids"], case["scale"]
    out = {"y": s["table"].double().index_select(0, ids) * scale}
    if case["grad"]:
        keep = torch.nonzero(ids != case["padding"])[:, 0]
        dtable = torch.zeros(case["n"], case["k"], dtype=torch.float64, device=DEV)
        dtable.index_add_(0, ids[keep], s["dy"].double()[keep])
        out["dtable"] = dtable * scale
    return out


def exact(case, seed):
    return {"xent": _exact_xent, "norm": _exact_norm, "embed": _exact_embed}[case["op"]](case, prepare(case, seed))
