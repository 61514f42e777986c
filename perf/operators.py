"""The operators of a training step around the sampled layers, case by case.

  embed        rows of a learned table by node id, scaled (csgs_embed)
  embed_grad   the table's gradient by sorted ids: dense (csgs_embed_grad), or the rows that were looked up alone
               (csgs_embed_grad_rows)
  norm         y = beta x + alpha a(gate) .* N(h), u = N(y): a block's gated residual with the norms around it (csgs_norm_residual)
  norm_grad    its gradient (csgs_norm_residual_grad)
  clip         the global norm over all gradients of a network, and clipping by it (csgs_grad_clip)

own = False computes the same with elementary torch operations in 32 bits; own = True calls the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def _embed(name, rows, F, tokens, dist, table, out, scale=1.0, pad=0.0, count=0):
    return dict(name=name, op="embed", rows=rows, F=F, tokens=tokens, dist=dist, table=table, out=out, scale=float(scale), pad=float(pad),
                count=count)


def _embed_grad(name, rows, F, tokens, dist, compact, g, d, scale=1.0, pad=0.0, count=0):
    return dict(name=name, op="embed_grad", rows=rows, F=F, tokens=tokens, dist=dist, compact=compact, g=g, d=d, scale=float(scale),
                pad=float(pad), count=count)


def _norm(name, M, F, post, pre, act, gate, stream="f32", block="f32", bias=False, beta=1.0, alpha=1.0, grad=False, count=0, dy=True):
    return dict(name=name, op="norm_grad" if grad else "norm", M=M, F=F, post=post, pre=pre, act=act, gate=gate, stream=stream, block=block,
                bias=bias, beta=float(beta), alpha=float(alpha), count=count, dy=dy)


def _clip(name, layers, feat, hidden, classes, table_rows, table_dim, table="f32", count=0, kind="l2", max_norm=1.0):
    return dict(name=name, op="clip", layers=layers, feat=feat, hidden=hidden, classes=classes, table_rows=table_rows, table_dim=table_dim,
                table=table, count=count, kind=kind, max_norm=float(max_norm))


def listed():
    return [
        # the batch of a toy graph looks its rows up: latency
        _embed("lookup_tiny", 4096, 64, 256, "uniform", "f32", "f32", scale=8.0),
        # the rows of a mini-batch of almost a whole partition, out of the large graph's table in bfloat16
        _embed("lookup_large", 2_449_029, 100, 131_072, "uniform", "bf16", "f32", scale=10.0),
        # three node sets of the toy step, whose rows' gradients come together: latency
        _embed_grad("table_grad_rows_tiny", 4096, 64, 768, "hubs", True, "f32", "f32", scale=8.0),
        # four node sets of the large step: hubs are in all of them, places behind the sets' device counts hold no node
        _embed_grad("table_grad_rows_large", 2_449_029, 100, 32_768, "hubs", True, "f32", "f32", scale=10.0, pad=0.1),
        # an attribute of many values (words of a description), some of them in most of the nodes; the whole table's gradient
        _embed_grad("table_grad_dense", 50_021, 512, 65_536, "zipf", False, "bf16", "f32", scale=1.0, pad=0.02),
        # a block's end on the toy graph
        _norm("residual_tiny", 256, 64, "rms", "rms", "linear", "row"),
        # a block's end for almost a whole partition, a gate for every entry
        _norm("residual_large", 131_072, 256, "layer", "layer", "sigmoid", "full", bias=True, beta=0.9, alpha=0.5),
        # gradient of an ordinary block
        _norm("residual_grad_medium", 8192, 256, "rms", "rms", "silu", "full", beta=0.9, alpha=0.5, grad=True),
        # odd width in bfloat16, rows up to a device count, the residual stream ends here
        _norm("residual_grad_odd", 2048, 602, "layer", "layer", "sigmoid", "row", stream="bf16", block="bf16", bias=True, grad=True, count=1999,
              dy=False),
        # a wide network in mixed types
        _norm("residual_grad_large", 65_536, 1024, "rms", "rms", "sigmoid", "full", stream="f32", block="bf16", alpha=0.7, grad=True),
        # all gradients of the large graph's step: layers, gates and norms, and the rows that were looked up
        _clip("clip_layers", 3, 100, 256, 47, 32_768, 100, count=29_000),
        # the same with the gradient of a whole table
        _clip("clip_table", 3, 100, 256, 47, 2_449_029, 100),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    case = _draw(rng)
    del case["name"]
    return case


def _draw(rng):
    op = rng.choice(["embed", "embed_grad", "norm", "norm_grad", "clip"])
    if op in ("embed", "embed_grad"):
        tokens = _log(rng, 1, 131_072)
        F = _log(rng, 1, min(1024, max(1, 33_000_000 // tokens)))
        dist = rng.choice(["uniform", "hubs", "zipf"])
        types = (rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"]))
        scale, pad = rng.choice([1.0, math.sqrt(F)]), rng.choice([0.0, 0.05])
        count = rng.randrange(tokens + 1) if rng.random() < 0.25 else 0
        if op == "embed":
            return _embed("", _log(rng, 1, min(2_449_029, 245_000_000 // F)), F, tokens, dist, *types, scale, pad, count)
        compact = rng.random() < 0.5
        rows = _log(rng, 1, 2_449_029 if compact else min(2_449_029, 25_000_000 // F))
        return _embed_grad("", rows, F, tokens, dist, compact, *types, scale, pad, count)
    if op in ("norm", "norm_grad"):
        M = _log(rng, 1, 131_072)
        F = _log(rng, 8, min(4096, 33_000_000 // M))
        stream, block = rng.choice([("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
        count = rng.randrange(M + 1) if rng.random() < 0.25 else 0
        return _norm("", M, F, rng.choice(["rms", "layer"]), rng.choice(["rms", "layer"]), rng.choice(["linear", "sigmoid", "silu"]),
                     rng.choice(["none", "row", "full"]), stream, block, rng.random() < 0.5, rng.choice([1.0, 0.9]), rng.choice([1.0, 0.5]),
                     op == "norm_grad", count, rng.random() < 0.7)
    hidden, feat = _log(rng, 16, 1024), _log(rng, 16, 602)
    rows = _log(rng, 64, 200_000)
    count = rng.randrange(rows + 1) if rng.random() < 0.5 else 0
    return _clip("", rng.randrange(2, 9), feat, hidden, _log(rng, 2, 128), rows, _log(rng, 1, 256), rng.choice(["f32", "bf16"]), count,
                 rng.choice(["l2", "l2", "max"]), rng.choice([1.0, 1e6]))


# ---------------------------------------------------------------------------------------------- inputs

def _ids(case, gen):
    rows, n = case["rows"], case["tokens"]
    u = torch.rand(n, generator=gen, device=DEV, dtype=torch.float64)
    flat = (u * rows).long().clamp_(max=rows - 1)
    # log-uniform ranks, scattered over the table by a step that shares no factor with its size
    step = 1_000_003
    while math.gcd(step, rows) != 1:
        step += 2
    rank = (torch.exp(u * math.log(rows + 1.0)) - 1.0).long().clamp_(0, rows - 1)
    steep = (rank * step) % rows
    dist = case["dist"]
    ids = flat if dist == "uniform" else steep
    if dist == "hubs":
        ids = torch.where(torch.rand(n, generator=gen, device=DEV) < 0.5, flat, steep)
    if case["pad"]:
        ids = torch.where(torch.rand(n, generator=gen, device=DEV) < case["pad"], torch.full_like(ids, -1), ids)
    return ids.int()


def _clip_shapes(c):
    shapes = []
    f = c["feat"]
    for l in range(c["layers"]):
        out = c["classes"] if l == c["layers"] - 1 else c["hidden"]
        shapes += [(f, out), (1, out), (1, out), (1, out)]
        f = out
    return shapes


def _inputs(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def normal(*shape, std=1.0, dtype="f32"):
        return (torch.randn(*shape, generator=gen, device=DEV) * std).to(TYPES[dtype])

    op = case["op"]
    s = {"case": case}
    if op == "embed":
        s["ids"] = _ids(case, gen)
        s["table"] = normal(case["rows"], case["F"], std=0.1, dtype=case["table"])
    elif op == "embed_grad":
        s["ids"] = _ids(case, gen)
        s["G"] = normal(case["tokens"], case["F"], std=0.01, dtype=case["g"])
    elif op in ("norm", "norm_grad"):
        M, F = case["M"], case["F"]
        s["x"] = normal(M, F, dtype=case["stream"])
        h = normal(M, F, std=0.5)
        # rows without kept edges come out of the layer as zeros
        s["h"] = torch.where(torch.rand(M, 1, generator=gen, device=DEV) < 0.03, torch.zeros_like(h), h).to(TYPES[case["block"]])
        # a gate for every entry is the block's output, one for all rows is a parameter
        s["gate"] = normal(M, F, dtype=case["block"]) if case["gate"] == "full" else normal(F) if case["gate"] == "row" else None
        s["post_w"], s["pre_w"] = 1.0 + normal(F, std=0.1), 1.0 + normal(F, std=0.1)
        s["post_b"], s["pre_b"] = (normal(F, std=0.1), normal(F, std=0.1)) if case["bias"] else (None, None)
        if op == "norm_grad":
            s["dy"] = normal(M, F, std=0.01, dtype=case["stream"]) if case["dy"] else None
            s["du"] = normal(M, F, std=0.01, dtype=case["block"])
    else:
        s["grads"] = [normal(*shape, std=0.02) for shape in _clip_shapes(case)]
        s["grads"].append(normal(case["table_rows"], case["table_dim"], std=0.02, dtype=case["table"]))
    if case["count"]:
        s["count"] = torch.tensor([case["count"]], dtype=torch.int32, device=DEV)
    else:
        s["count"] = None
    return s


def _norm_args(s):
    from paper_2101_07706_amd import csgs
    c = s["case"]
    kinds = {"rms": csgs.NORM_RMS, "layer": csgs.NORM_LAYER}
    acts = {"linear": csgs.GATE_LINEAR, "sigmoid": csgs.GATE_SIGMOID, "silu": csgs.GATE_SILU}
    return dict(gate=s["gate"], gate_act=acts[c["act"]], post=kinds[c["post"]], post_w=s["post_w"], post_b=s["post_b"], pre=kinds[c["pre"]],
                pre_w=s["pre_w"], pre_b=s["pre_b"], eps=1e-5, alpha=c["alpha"], beta=c["beta"], M_dev=s["count"])


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    # the buffers that a training program keeps from step to step
    from paper_2101_07706_amd import csgs
    op = case["op"]
    if op == "embed":
        s["out"] = torch.zeros((case["tokens"], case["F"]), dtype=TYPES[case["out"]], device=DEV)
    elif op == "embed_grad":
        n, F, rows = case["tokens"], case["F"], case["rows"]
        s["scratch"] = torch.empty(csgs.csgs_embed_grad_scratch_bytes(n, rows, F), dtype=torch.uint8, device=DEV)
        if case["compact"]:
            s["uniq"] = torch.full((n,), -1, dtype=torch.int32, device=DEV)
            s["n_uniq"] = torch.zeros(1, dtype=torch.int32, device=DEV)
            s["d"] = torch.zeros((n, F), dtype=TYPES[case["d"]], device=DEV)
        else:
            s["d"] = torch.zeros((rows, F), dtype=TYPES[case["d"]], device=DEV)
    elif op in ("norm", "norm_grad"):
        M, F = case["M"], case["F"]
        stream, block = TYPES[case["stream"]], TYPES[case["block"]]
        if op == "norm":
            s["y"] = torch.zeros((M, F), dtype=stream, device=DEV)
            s["u"] = torch.zeros((M, F), dtype=block, device=DEV)
        else:
            s["dx"] = torch.zeros((M, F), dtype=stream, device=DEV)
            s["dh"] = torch.zeros((M, F), dtype=block, device=DEV)
            s["dgate"] = None
            if case["gate"] == "full":
                s["dgate"] = torch.zeros((M, F), dtype=block, device=DEV)
            elif case["gate"] == "row":
                s["dgate"] = torch.zeros(F, dtype=torch.float32, device=DEV)
            for k in ("dpost_w", "dpre_w"):
                s[k] = torch.zeros(F, dtype=torch.float32, device=DEV)
            for k in ("dpost_b", "dpre_b"):
                s[k] = torch.zeros(F, dtype=torch.float32, device=DEV) if case["bias"] else None
            s["scratch"] = torch.empty(csgs.csgs_norm_residual_grad_scratch_bytes(M, F), dtype=torch.uint8, device=DEV)
    else:
        s["outs"] = [torch.zeros_like(g) for g in s["grads"]]
        s["norm"] = torch.zeros(1, dtype=torch.float32, device=DEV)
        counts = [None] * (len(s["grads"]) - 1) + [s["count"]]
        s["list"] = csgs.make_grad_list(s["grads"], s["outs"], counts)
    return s


# ---------------------------------------------------------------------------------------------- one pass

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2101_07706_amd import csgs
    c = s["case"]
    op = c["op"]
    if op == "embed":
        csgs.csgs_embed(s["table"], s["ids"], s["out"], scale=c["scale"], n_dev=s["count"])
        return s["out"]
    if op == "embed_grad":
        if c["compact"]:
            csgs.csgs_embed_grad_rows(s["ids"], s["G"], c["rows"], s["uniq"], s["n_uniq"], s["d"], s["scratch"], scale=c["scale"],
                                      n_dev=s["count"])
            return s["uniq"], s["n_uniq"], s["d"]
        csgs.csgs_embed_grad(s["ids"], s["G"], s["d"], s["scratch"], scale=c["scale"], n_dev=s["count"])
        return s["d"]
    if op == "norm":
        csgs.csgs_norm_residual(s["x"], s["h"], s["y"], s["u"], **_norm_args(s))
        return s["y"], s["u"]
    if op == "norm_grad":
        csgs.csgs_norm_residual_grad(s["x"], s["h"], s["dy"], s["du"], s["dx"], s["dh"], s["dgate"], s["dpost_w"], s["dpost_b"], s["dpre_w"],
                                     s["dpre_b"], s["scratch"], **_norm_args(s))
        return [t for t in (s["dx"], s["dh"], s["dgate"], s["dpost_w"], s["dpost_b"], s["dpre_w"], s["dpre_b"]) if t is not None]
    csgs.csgs_grad_clip(s["list"], csgs.GRAD_L2 if c["kind"] == "l2" else csgs.GRAD_MAX, c["max_norm"], s["norm"])
    return [s["norm"]] + s["outs"]


def _within(s, n):
    return None if s["count"] is None else (torch.arange(n, device=DEV) < s["count"]).unsqueeze(1)


def _valid(s):
    ids = s["ids"].long()
    ok = (ids >= 0) & (ids < s["case"]["rows"])
    if s["count"] is not None:
        ok = ok & (torch.arange(ids.numel(), device=DEV) < s["count"])
    return ids, ok


def _run_plain(s):
    c = s["case"]
    op = c["op"]
    if op == "embed":
        ids, ok = _valid(s)
        picked = s["table"][ids.clamp(0, c["rows"] - 1)].float() * c["scale"]
        return torch.where(ok.unsqueeze(1), picked, torch.zeros_like(picked)).to(TYPES[c["out"]])
    if op == "embed_grad":
        ids, ok = _valid(s)
        rows, n, F = c["rows"], c["tokens"], c["F"]
        g = s["G"].float() * c["scale"]
        if not c["compact"]:
            d = torch.zeros((rows + 1, F), dtype=torch.float32, device=DEV)
            d.index_add_(0, torch.where(ok, ids, torch.full_like(ids, rows)), g)
            return d[:rows].to(TYPES[c["d"]])
        met = torch.zeros(rows + 1, dtype=torch.int32, device=DEV)
        met[torch.where(ok, ids, torch.full_like(ids, rows))] = 1
        rank = torch.cumsum(met[:rows], 0, dtype=torch.int32)
        at = torch.where(ok, rank[ids.clamp(0, rows - 1)].long() - 1, torch.full_like(ids, n))
        uniq = torch.full((n + 1,), -1, dtype=torch.int32, device=DEV)
        uniq[at] = s["ids"]
        d = torch.zeros((n + 1, F), dtype=torch.float32, device=DEV)
        d.index_add_(0, at, g)
        return uniq[:n].clone(), rank[-1:].clone(), d[:n].to(TYPES[c["d"]])
    if op == "norm":
        _, n, a, _, _ = _plain_post(s)
        y = c["beta"] * s["x"].float() + c["alpha"] * (n if a is None else a * n)
        hat, _ = _plain_hat(y, c["pre"])
        u = hat * s["pre_w"]
        if s["pre_b"] is not None:
            u = u + s["pre_b"]
        inside = _within(s, c["M"])
        if inside is not None:
            y, u = torch.where(inside, y, torch.zeros_like(y)), torch.where(inside, u, torch.zeros_like(u))
        return y.to(TYPES[c["stream"]]), u.to(TYPES[c["block"]])
    if op == "norm_grad":
        return _plain_norm_grad(s)
    live = [g.float() for g in s["grads"]]
    inside = _within(s, c["table_rows"])
    if inside is not None:
        live[-1] = torch.where(inside, live[-1], torch.zeros_like(live[-1]))
    if c["kind"] == "l2":
        total = torch.sqrt(sum((g * g).sum() for g in live))
    else:
        total = torch.stack([g.abs().max() for g in live]).max()
    coef = torch.clamp(c["max_norm"] / (total + 1e-6), max=1.0)
    return [total.reshape(1)] + [(g * coef).to(src.dtype) for g, src in zip(live, s["grads"])]


def _plain_hat(v, kind):
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    r = torch.rsqrt((v * v).mean(1, keepdim=True) + 1e-5)
    return v * r, r


def _plain_post(s):
    c = s["case"]
    hat, r = _plain_hat(s["h"].float(), c["post"])
    n = hat * s["post_w"]
    if s["post_b"] is not None:
        n = n + s["post_b"]
    if s["gate"] is None:
        return hat, n, None, None, r
    g = s["gate"].float()
    if c["act"] == "linear":
        return hat, n, g, torch.ones_like(g), r
    sig = 1.0 / (1.0 + torch.exp(-g))
    if c["act"] == "sigmoid":
        return hat, n, sig, sig * (1.0 - sig), r
    return hat, n, g * sig, sig * (1.0 + g * (1.0 - sig)), r


def _plain_hat_grad(t, hat, r, kind):
    """Gradient through v -> hat(v), t the gradient of hat."""
    g = t - hat * (t * hat).mean(1, keepdim=True)
    if kind == "layer":
        g = g - t.mean(1, keepdim=True)
    return g * r


def _plain_norm_grad(s):
    c = s["case"]
    hat, n, a, da, r = _plain_post(s)
    y = c["beta"] * s["x"].float() + c["alpha"] * (n if a is None else a * n)
    yhat, yr = _plain_hat(y, c["pre"])
    du = s["du"].float()
    inside = _within(s, c["M"])
    if inside is not None:
        du = torch.where(inside, du, torch.zeros_like(du))
    d = _plain_hat_grad(du * s["pre_w"], yhat, yr, c["pre"])
    if s["dy"] is not None:
        dy = s["dy"].float()
        d = d + (dy if inside is None else torch.where(inside, dy, torch.zeros_like(dy)))
    t = c["alpha"] * d
    dn = t if a is None else t * a
    dh = _plain_hat_grad(dn * s["post_w"], hat, r, c["post"])
    out = [(c["beta"] * d).to(TYPES[c["stream"]]), dh.to(TYPES[c["block"]])]
    if a is not None:
        dg = t * n * da
        out.append(dg.to(TYPES[c["block"]]) if c["gate"] == "full" else dg.sum(0))
    out.append((dn * hat).sum(0))
    if c["bias"]:
        out.append(dn.sum(0))
    out.append((du * yhat).sum(0))
    if c["bias"]:
        out.append(du.sum(0))
    return out


# ---------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "embed":
        live = case["count"] or case["tokens"]
        out = torch.zeros((case["tokens"], case["F"]), dtype=torch.float64, device=DEV)
        ids = s["ids"][:live].long()
        at = torch.nonzero((ids >= 0) & (ids < case["rows"])).flatten()
        out[at] = case["scale"] * s["table"][ids[at]].double()
        return out
    if op == "embed_grad":
        live = case["count"] or case["tokens"]
        ids = s["ids"][:live].cpu().numpy().astype(np.int64)
        at = np.flatnonzero((ids >= 0) & (ids < case["rows"]))
        order = at[np.argsort(ids[at], kind="stable")]
        keys, first = np.unique(ids[order], return_index=True)
        G = s["G"].cpu().double().numpy()
        sums = np.add.reduceat(G[order], first, axis=0) * case["scale"] if len(keys) else np.zeros((0, case["F"]))
        if not case["compact"]:
            d = np.zeros((case["rows"], case["F"]))
            d[keys] = sums
            return torch.from_numpy(d).to(DEV)
        d = np.zeros((case["tokens"], case["F"]))
        d[:len(keys)] = sums
        uniq = np.full(case["tokens"], -1, np.int32)
        uniq[:len(keys)] = keys
        return torch.from_numpy(uniq).to(DEV), torch.tensor([len(keys)], dtype=torch.int32, device=DEV), torch.from_numpy(d).to(DEV)
    if op in ("norm", "norm_grad"):
        live = case["count"] or case["M"]
        leaf = {k: s[k].double().requires_grad_(op == "norm_grad") for k in ("x", "h", "gate", "post_w", "post_b", "pre_w", "pre_b")
                if s[k] is not None}

        def norm(v, kind, w, b):
            mean = v.sum(-1, keepdim=True) / v.shape[-1] if kind == "layer" else 0.0
            power = ((v - mean) ** 2).sum(-1, keepdim=True) / v.shape[-1]
            out = (v - mean) / torch.sqrt(power + 1e-5) * leaf[w]
            return out + leaf[b] if b in leaf else out

        x, h = leaf["x"][:live], leaf["h"][:live]
        n = norm(h, case["post"], "post_w", "post_b")
        if "gate" in leaf:
            g = leaf["gate"][:live] if case["gate"] == "full" else leaf["gate"]
            n = n * {"linear": lambda v: v, "sigmoid": torch.sigmoid, "silu": lambda v: v * torch.sigmoid(v)}[case["act"]](g)
        y = case["beta"] * x + case["alpha"] * n
        u = norm(y, case["pre"], "pre_w", "pre_b")
        if op == "norm":
            pad = torch.zeros((case["M"] - live, case["F"]), dtype=torch.float64, device=DEV)
            return torch.cat([y, pad]), torch.cat([u, pad])
        loss = (u * s["du"][:live].double()).sum()
        if s["dy"] is not None:
            loss = loss + (y * s["dy"][:live].double()).sum()
        names = [k for k in ("x", "h", "gate", "post_w", "post_b", "pre_w", "pre_b") if k in leaf]
        return list(torch.autograd.grad(loss, [leaf[k] for k in names]))
    live = [g.double() for g in s["grads"]]
    if case["count"]:
        live[-1][case["count"]:] = 0.0
    if case["kind"] == "l2":
        total = math.sqrt(sum(float(torch.dot(g.flatten(), g.flatten())) for g in live))
    else:
        total = max(float(torch.maximum(g.max(), -g.min())) for g in live)
    coef = min(1.0, case["max_norm"] / (total + 1e-6))
    return [torch.tensor([total], dtype=torch.float64, device=DEV)] + [g * coef for g in live]


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def _distinct(case):
    """Expected number of different rows among the ids."""
    rows, n = case["rows"], (case["count"] or case["tokens"]) * (1.0 - case["pad"])
    k = np.arange(1, rows + 1, dtype=np.float64)
    steep = np.log1p(1.0 / k) / math.log(rows + 1.0)
    flat = np.full(rows, 1.0 / rows)
    p = {"uniform": flat, "zipf": steep, "hubs": 0.5 * flat + 0.5 * steep}[case["dist"]]
    return float(-np.expm1(n * np.log1p(-np.minimum(p, 1.0 - 1e-12))).sum())


def work(case):
    op = case["op"]
    if op == "embed":
        n, F = case["count"] or case["tokens"], case["F"]
        return {"bytes": 4 * n + _distinct(case) * F * SIZE[case["table"]] + n * F * SIZE[case["out"]], "flops": n * F}
    if op == "embed_grad":
        n, F = case["count"] or case["tokens"], case["F"]
        live = n * (1.0 - case["pad"])
        written = _distinct(case) * (F * SIZE[case["d"]] + 4) if case["compact"] else case["rows"] * F * SIZE[case["d"]]
        return {"bytes": 4 * n + live * F * SIZE[case["g"]] + written, "flops": 2 * live * F}
    if op in ("norm", "norm_grad"):
        n = (case["count"] or case["M"]) * case["F"]
        stream, block = SIZE[case["stream"]], SIZE[case["block"]]
        gate = block if case["gate"] == "full" else 0
        if op == "norm":
            return {"bytes": n * (2 * stream + 2 * block + gate), "flops": n * 20}
        return {"bytes": n * (2 * stream + 3 * block + 2 * gate + (stream if case["dy"] else 0)), "flops": n * 50}
    small = sum(a * b for a, b in _clip_shapes(case))
    table = (case["count"] or case["table_rows"]) * case["table_dim"]
    return {"bytes": 2 * (4 * small + SIZE[case["table"]] * table), "flops": 3 * (small + table)}
