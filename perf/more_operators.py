"""The operators of a feed-forward block on the rows of a sampled layer, and of the step that trains it, case by case.

  linear       y = alpha act(a w + b) + beta r (csgs_linear)
  linear_grad  its gradient (csgs_linear_grad)
  gated        h = act(x wg + bg) .* (x wu + bu), both projections in one kernel (csgs_gated)
  gated_grad   its gradient (csgs_gated_grad)
  adamw        one step over all tensors of a network, clipped by the global norm, states in 32 or in 8 bits (csgs_adamw)

own = False computes the same with elementary torch operations in 32 bits (states that are held in 8 bits, whose values may lie next to a
border between two codes, and the norm over all gradients in 64); own = True calls the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
ACTS = ["none", "relu", "sigmoid", "silu", "gelu"]
BETA1, BETA2, EPS, LR, DECAY = 0.9, 0.999, 1e-8, 1e-3, 0.01
BLOCK = 256      # entries of a row that share a scale where states are held in 8 bits


def _linear(name, M, K, N, block, stream, act="none", bias=True, residual=True, alpha=1.0, beta=1.0, count=0, grad=False):
    return dict(name=name, op="linear_grad" if grad else "linear", M=M, K=K, N=N, block=block, stream=stream, act=act, bias=bias,
                residual=residual, alpha=float(alpha), beta=float(beta), count=count)


def _gated(name, M, K, N, block, act="silu", bias=False, count=0, grad=False):
    return dict(name=name, op="gated_grad" if grad else "gated", M=M, K=K, N=N, block=block, act=act, bias=bias, count=count)


def _adamw(name, layers, width, ffn, classes, table_rows, table_dim, positions=0, count=0, state="f32", g="f32", p="f32", copies=False,
           max_norm=1.0, step=10):
    return dict(name=name, op="adamw", layers=layers, width=width, ffn=ffn, classes=classes, table_rows=table_rows, table_dim=table_dim,
                positions=positions, count=count, state=state, g=g, p=p, copies=copies, max_norm=float(max_norm), step=step)


def listed():
    return [
        # the classifier of a toy graph's batch: latency
        _linear("linear_tiny", 256, 64, 4, "f32", "f32", residual=False),
        # the block's second product for a wide network, onto a residual stream in float32
        _linear("linear_large", 65_536, 4096, 1024, "bf16", "f32", alpha=0.5),
        # gradient of a layer on raw features with an activation: odd widths, rows up to a device count
        _linear("linear_grad_odd", 8192, 602, 47, "f32", "f32", act="gelu", residual=False, count=7999, grad=True),
        # gradient of the block's second product
        _linear("linear_grad_large", 65_536, 4096, 1024, "bf16", "f32", alpha=0.5, grad=True),
        # one node is asked for: latency
        _gated("gated_single", 1, 1024, 4096, "bf16"),
        # the block's first half for a wide network
        _gated("gated_large", 65_536, 1024, 4096, "bf16"),
        # gradient for a mini-batch's rows in float32, odd widths
        _gated("gated_grad_odd", 4096, 602, 1111, "f32", act="gelu", bias=True, count=4001, grad=True),
        # gradient of the block's first half
        _gated("gated_grad_large", 65_536, 1024, 4096, "bf16", grad=True),
        # the step of a toy network with a learned vector per node, of which a mini-batch looked some up: latency
        _adamw("adamw_tiny", 2, 64, 0, 4, 4096, 64, positions=768, count=700),
        # the same on the large graph: rows of a long table
        _adamw("adamw_rows", 2, 256, 1024, 47, 2_449_029, 100, positions=131_072, count=120_000),
        # a wide network whose products read weights in bfloat16
        _adamw("adamw_wide", 2, 2048, 8192, 47, 0, 0, g="bf16", copies=True),
        # a whole table with states in 8 bits
        _adamw("adamw_8bit", 1, 256, 1024, 47, 500_009, 100, state="8bit"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    case = _draw(rng)
    del case["name"]
    return case


def _draw(rng):
    op = rng.choice(["linear", "linear_grad", "gated", "gated_grad", "adamw"])
    if op == "adamw":
        layers, width = rng.randrange(1, 3), _log(rng, 8, 1024)
        ffn = rng.choice([0, 2 * width, 4 * width, _log(rng, 8, 4096)])
        rows, dim = _log(rng, 16, 200_000), _log(rng, 1, 256)
        positions = rng.choice([0, rng.randrange(1, rows + 1)])
        count = rng.randrange(1, positions + 1) if positions and rng.random() < 0.7 else 0
        return _adamw("", layers, width, ffn, _log(rng, 2, 128), rows, dim, positions, count, rng.choice(["f32", "8bit"]),
                      rng.choice(["f32", "bf16"]), rng.choice(["f32", "f32", "bf16"]), rng.random() < 0.3, rng.choice([1.0, 1e6]),
                      rng.choice([0, 10, 1000]))
    M = _log(rng, 1, 65_536)
    most = 2 ** 36 // M if M > 64 else 2 ** 24
    K = _log(rng, 8, min(4096, most // 8))
    N = _log(rng, 2, min(4096, most // K))
    if rng.random() < 0.5:
        K, N = (K + 7) // 8 * 8, (N + 7) // 8 * 8
    count = rng.randrange(1, M + 1) if rng.random() < 0.25 else 0
    if op in ("gated", "gated_grad"):
        return _gated("", M, K, N, rng.choice(["f32", "bf16"]), rng.choice(ACTS), rng.random() < 0.5, count, op == "gated_grad")
    block, stream = rng.choice([("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
    return _linear("", M, K, N, block, stream, rng.choice(ACTS), rng.random() < 0.5, rng.random() < 0.5, rng.choice([1.0, 0.5]),
                   rng.choice([1.0, 0.9]), count, op == "linear_grad")


# ---------------------------------------------------------------------------------------------- inputs

def _shapes(c):
    """(rows, columns, whether weight decay applies) of a network's tensors but the table."""
    D, F = c["width"], c["ffn"]
    shapes = []
    for _ in range(c["layers"]):
        shapes += [(D, F, True), (D, F, True), (F, D, True)] if F else [(D, D, True)]
        shapes += [(1, D, False), (1, D, False)]
    return shapes + [(D, c["classes"], True)]


def _state_blocks(t):
    """A matrix's rows in blocks of BLOCK entries, the last one filled up with zeros, and the shape to come back to."""
    rows, cols = t.shape
    nb = (cols + BLOCK - 1) // BLOCK
    return torch.nn.functional.pad(t, (0, nb * BLOCK - cols)).reshape(rows, nb, BLOCK)


def _two_to(k):
    """2^k as float32, k an int32 tensor."""
    return ((k + 127).clamp(1, 254) << 23).view(torch.float32)


def _encode(t, second):
    """Float32 values as 8-bit codes and a block's exponent, plainly: (codes, exponents), uint8 both."""
    cols = t.shape[1]
    x = _state_blocks(t)
    e = x.view(torch.int32).bitwise_and(0x7FFFFFFF).amax(2, keepdim=True) >> 23          # (exponent field of the largest)
    if second:
        # 5 bits of exponent and 3 of mantissa, from 1.25 * 2^-31 to 2 of the block's power of two, what is not zero never rounded to zero
        bits = (x * _two_to(127 - e)).view(torch.int32)
        code = ((bits + 0x7FFFF + ((bits >> 20) & 1)) >> 20) - 769
        code = torch.where((x > 0) & (e > 0), code.clamp(1, 255), torch.zeros_like(code)).to(torch.uint8)
    else:
        # 4 bits of exponent and 3 of mantissa and a sign, the block's power of two at 128
        code = torch.where(e > 0, x * _two_to(134 - e), torch.zeros_like(x)).to(torch.float8_e4m3fn).view(torch.uint8)
    return code.reshape(t.shape[0], -1)[:, :cols].contiguous(), e.squeeze(2).to(torch.uint8)


def _decode(code, e, second):
    """What such codes stand for, as float32."""
    x = _state_blocks(code)
    e = e.to(torch.int32).unsqueeze(2)
    if second:
        c = x.to(torch.int32)
        v = torch.where(c > 0, ((c + 769) << 20).view(torch.float32) * _two_to(e - 127), torch.zeros((), device=x.device))
    else:
        v = x.view(torch.float8_e4m3fn).float() * _two_to(e - 134)
    return v.reshape(code.shape[0], -1)[:, :code.shape[1]].contiguous()


def _inputs(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def normal(*shape, std=1.0, dtype="f32"):
        return (torch.randn(*shape, generator=gen, device=DEV) * std).to(TYPES[dtype])

    s = {"case": case, "count": None}
    if case["count"]:
        s["count"] = torch.tensor([case["count"]], dtype=torch.int32, device=DEV)
    if case["op"] != "adamw":
        M, K, N, block = case["M"], case["K"], case["N"], case["block"]
        s["x"] = normal(M, K, dtype=block)
        std = 1.0 / math.sqrt(K)
        s["b"] = normal(N, std=0.1) if case["bias"] else None
        if case["op"] in ("gated", "gated_grad"):
            s["wg"], s["wu"] = normal(K, N, std=std, dtype=block), normal(K, N, std=std, dtype=block)
            s["bu"] = normal(N, std=0.1) if case["bias"] else None
            if case["op"] == "gated_grad":
                s["d"] = normal(M, N, std=0.01, dtype=block)
        else:
            s["w"] = normal(K, N, std=std, dtype=block)
            s["r"] = normal(M, N, dtype=case["stream"]) if case["residual"] else None
            if case["op"] == "linear_grad":
                s["d"] = normal(M, N, std=0.01, dtype=case["stream"])
        return s
    s["step"] = torch.full((1,), case["step"], dtype=torch.int32, device=DEV)
    s["norm"] = torch.zeros(1, dtype=torch.float32, device=DEV)
    s["entries"] = []
    shapes = _shapes(case)
    if case["table_rows"]:
        shapes.append((case["table_rows"], case["table_dim"], False))
    for k, (rows, cols, decay) in enumerate(shapes):
        table = case["table_rows"] and k == len(shapes) - 1
        n = case["positions"] if table and case["positions"] else rows
        e = {"decay": DECAY if decay else 0.0, "ids": None, "n": None, "second": None}
        e["p"] = normal(rows, cols, std=0.1, dtype=case["p"])
        e["copy"] = e["p"].to(torch.bfloat16) if case["copies"] and decay else None
        e["g"] = normal(n, cols, std=0.02, dtype=case["g"])
        m = normal(rows, cols, std=0.005)
        v = (m * m + 1e-8) * torch.exp(torch.randn(rows, cols, generator=gen, device=DEV))
        e["m_exp"] = e["v_exp"] = None
        if case["state"] == "8bit" and rows > 1:
            m, e["m_exp"] = _encode(m, False)
            v, e["v_exp"] = _encode(v, True)
        e["m"], e["v"] = m, v
        if table and case["positions"]:
            # the different rows that a mini-batch looked up, ascending; places behind their number hold none
            e["ids"] = torch.sort(torch.randperm(rows, generator=gen, device=DEV)[:n])[0].int()
            e["n"] = s["count"]
            if case["count"]:
                e["ids"][case["count"]:] = -1
        s["entries"].append(e)
    return s


def _empty(*shape, dtype="f32"):
    return torch.zeros(*shape, dtype=TYPES[dtype], device=DEV)


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    # the buffers and lists that a training program keeps from step to step
    from paper_2101_07706_amd import csgs
    op = case["op"]
    if op == "adamw":
        es = s["entries"]
        s["clip"] = csgs.make_grad_list([e["g"] for e in es], [None] * len(es), [e["n"] for e in es])
        s["list"] = csgs.make_adamw_list([csgs.adamw_entry(e["p"], e["g"], e["m"], e["v"], m_exp=e["m_exp"], v_exp=e["v_exp"],
                                                           copy=None if e["copy"] is e["p"] else e["copy"], ids=e["ids"], n_dev=e["n"], weight_decay=e["decay"]) for e in es])
        for e in es:
            if e["m_exp"] is not None:
                e["m_out"], e["v_out"] = _empty(*e["m"].shape), _empty(*e["v"].shape)
        return s
    M, K, N, block = case["M"], case["K"], case["N"], case["block"]
    elem = {"f32": csgs.F32, "bf16": csgs.BF16}[block]
    if op == "linear":
        s["y"] = _empty(M, N, dtype=case["stream"])
    elif op == "gated":
        s["y"] = _empty(M, N, dtype=block)
    else:
        s["dx"] = _empty(M, K, dtype=block)
        s["db"] = _empty(N) if case["bias"] else None
        if op == "linear_grad":
            s["dw"] = _empty(K, N, dtype=block)
            s["dr"] = _empty(M, N, dtype=case["stream"]) if case["residual"] else None
            s["scratch"] = torch.empty(csgs.csgs_linear_grad_scratch_bytes(M, K, N, elem), dtype=torch.uint8, device=DEV)
        else:
            s["dwg"], s["dwu"] = _empty(K, N, dtype=block), _empty(K, N, dtype=block)
            s["dbu"] = _empty(N) if case["bias"] else None
            s["scratch"] = torch.empty(csgs.csgs_gated_grad_scratch_bytes(M, K, N, elem), dtype=torch.uint8, device=DEV)
    return s


# ---------------------------------------------------------------------------------------------- one pass

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2101_07706_amd import csgs
    c = s["case"]
    op = c["op"]
    if op == "adamw":
        csgs.csgs_adamw(s["list"], LR, s["step"], beta1=BETA1, beta2=BETA2, eps=EPS, clip=s["clip"], kind=csgs.GRAD_L2, max_norm=c["max_norm"],
                        norm=s["norm"])
        for e in s["entries"]:
            if e["m_exp"] is not None:
                csgs.csgs_state_read(e["m"], e["m_exp"], csgs.STATE_FIRST, e["m_out"])
                csgs.csgs_state_read(e["v"], e["v_exp"], csgs.STATE_SECOND, e["v_out"])
        return _adamw_outputs(s)
    act = {"none": csgs.ACT_NONE, "relu": csgs.ACT_RELU, "sigmoid": csgs.ACT_SIGMOID, "silu": csgs.ACT_SILU, "gelu": csgs.ACT_GELU}[c["act"]]
    if op == "linear":
        csgs.csgs_linear(s["x"], s["w"], s["y"], bias=s["b"], r=s["r"], act=act, alpha=c["alpha"], beta=c["beta"], M_dev=s["count"])
        return s["y"]
    if op == "linear_grad":
        csgs.csgs_linear_grad(s["x"], s["w"], s["d"], s["dx"], s["dw"], s["db"], s["dr"], s["scratch"], bias=s["b"], act=act, alpha=c["alpha"],
                              beta=c["beta"], M_dev=s["count"])
        return [t for t in (s["dx"], s["dw"], s["db"], s["dr"]) if t is not None]
    if op == "gated":
        csgs.csgs_gated(s["x"], s["wg"], s["wu"], s["y"], bg=s["b"], bu=s["bu"], act=act, M_dev=s["count"])
        return s["y"]
    csgs.csgs_gated_grad(s["x"], s["wg"], s["wu"], s["d"], s["dx"], s["dwg"], s["dwu"], s["db"], s["dbu"], s["scratch"], bg=s["b"], bu=s["bu"],
                         act=act, M_dev=s["count"])
    return [t for t in (s["dx"], s["dwg"], s["dwu"], s["db"], s["dbu"]) if t is not None]


def _adamw_outputs(s):
    out = [s["norm"], s["step"]]
    for e in s["entries"]:
        out += [e["p"], e.get("m_out", e["m"]), e.get("v_out", e["v"])]
        if e["copy"] is not None:
            out.append(e["copy"])
    return out


def _live(s, t):
    """Rows behind the device count count for nothing."""
    if s["count"] is None:
        return t
    inside = (torch.arange(t.shape[0], device=DEV) < s["count"]).unsqueeze(1)
    return torch.where(inside, t, torch.zeros((), dtype=t.dtype, device=DEV))


def _plain_act(name, g):
    """act(g) and its derivative."""
    if name == "none":
        return g, torch.ones_like(g)
    if name == "relu":
        on = (g > 0).to(g.dtype)
        return g * on, on
    if name == "gelu":
        phi = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    sig = 1.0 / (1.0 + torch.exp(-g))
    if name == "sigmoid":
        return sig, sig * (1.0 - sig)
    return g * sig, sig * (1.0 + g * (1.0 - sig))


def _product(x, w, b):
    y = x @ w
    return y if b is None else y + b


def _run_plain(s):
    c = s["case"]
    op = c["op"]
    if op == "adamw":
        return _plain_adamw(s)
    x, block = s["x"].float(), TYPES[c["block"]]
    if op in ("linear", "linear_grad"):
        w, stream = s["w"].float(), TYPES[c["stream"]]
        if op == "linear":
            y = c["alpha"] * _plain_act(c["act"], _product(x, w, s["b"]))[0]
            if s["r"] is not None:
                y = y + c["beta"] * s["r"].float()
            return _live(s, y).to(stream)
        d = _live(s, s["d"].float())
        t = c["alpha"] * d
        if c["act"] != "none":
            t = t * _plain_act(c["act"], _product(x, w, s["b"]))[1]
        out = [(t @ w.t()).to(block), (_live(s, x).t() @ t).to(block)]
        if c["bias"]:
            out.append(t.sum(0))
        if c["residual"]:
            out.append((c["beta"] * d).to(stream))
        return out
    wg, wu = s["wg"].float(), s["wu"].float()
    g, u = _product(x, wg, s["b"]), _product(x, wu, s["bu"])
    a, da = _plain_act(c["act"], g)
    if op == "gated":
        return _live(s, a * u).to(block)
    d = _live(s, s["d"].float())
    tg, tu = d * u * da, d * a
    xl = _live(s, x).t()
    out = [(tg @ wg.t() + tu @ wu.t()).to(block), (xl @ tg).to(block), (xl @ tu).to(block)]
    if c["bias"]:
        out += [tg.sum(0), tu.sum(0)]
    return out


def _plain_adamw(s):
    c = s["case"]
    total = None
    for e in s["entries"]:
        g = e["g"].double()
        if e["n"] is not None:
            g = torch.where((torch.arange(g.shape[0], device=DEV) < e["n"]).unsqueeze(1), g, torch.zeros((), dtype=g.dtype, device=DEV))
        part = (g * g).sum()
        total = part if total is None else total + part
    norm = torch.sqrt(total)
    coef = torch.clamp(c["max_norm"] / (norm + 1e-6), max=1.0)
    s["norm"].copy_(norm.reshape(1))
    s["step"] += 1
    t = s["step"].double()
    root, first = torch.sqrt(1.0 - BETA2 ** t).float(), (1.0 - BETA1 ** t).float()
    for e in s["entries"]:
        at = None
        if e["ids"] is not None:
            at = torch.arange(e["ids"].numel(), device=DEV)
            if e["n"] is not None:
                at = torch.where(at < e["n"], at, torch.zeros_like(at))      # (the first row again, with the same result)
            rows = e["ids"].long()[at]
        pick = (lambda x: x) if at is None else (lambda x: x[rows])
        p, g = pick(e["p"]).float(), e["g"] if at is None else e["g"][at]
        if e["m_exp"] is None:
            g = g.float() * coef.float()
            m = BETA1 * pick(e["m"]) + (1.0 - BETA1) * g
            v = BETA2 * pick(e["v"]) + (1.0 - BETA2) * g * g
        else:
            g = g.double() * coef
            m = (BETA1 * _decode(pick(e["m"]), pick(e["m_exp"]), False).double() + (1.0 - BETA1) * g).float()
            v = (BETA2 * _decode(pick(e["v"]), pick(e["v_exp"]), True).double() + (1.0 - BETA2) * (g * g)).float()
        p = p - LR * ((m / first) / (torch.sqrt(v) / root + EPS) + e["decay"] * p)
        put = (lambda x, y: x.copy_(y)) if at is None else (lambda x, y: x.index_copy_(0, rows, y.to(x.dtype)))
        put(e["p"], p)
        if e["copy"] is not None:
            put(e["copy"], p)
        if e["m_exp"] is None:
            put(e["m"], m)
            put(e["v"], v)
        else:
            for k, x, second in (("m", m, False), ("v", v, True)):
                code, exp = _encode(x, second)
                put(e[k], code)
                put(e[k + "_exp"], exp)
                e[k + "_out"] = _decode(e[k], e[k + "_exp"], second)
    return _adamw_outputs(s)


# ---------------------------------------------------------------------------------------------- in 64 bits

def _in_64(codes, exps, second):
    """What 8-bit codes stand for, by the fields' own arithmetic."""
    c = codes.long()
    scale = torch.repeat_interleave(exps.double(), BLOCK, dim=1)[:, :codes.shape[1]]
    if second:
        f = c + 1                                                # (code 255 is 2, a step is an eighth of an octave)
        value = (1.0 + (f % 8).double() / 8.0) * torch.pow(2.0, torch.div(f, 8, rounding_mode="floor").double() - 31.0)
        return torch.where(c == 0, torch.zeros_like(value), value * torch.pow(2.0, scale - 127.0))
    field, mantissa = (c >> 3) & 15, (c & 7).double() / 8.0
    value = torch.where(field == 0, mantissa * 2.0 ** -6, (1.0 + mantissa) * torch.pow(2.0, field.double() - 7.0))
    return torch.where(c >= 128, -value, value) * torch.pow(2.0, scale - 134.0)


def _held_64(x, second):
    """The values that 8-bit states keep of these."""
    x = x.float().double()
    rows, cols = x.shape
    nb = (cols + BLOCK - 1) // BLOCK
    full = torch.zeros(rows, nb * BLOCK, dtype=torch.float64, device=x.device)
    full[:, :cols] = x
    full = full.reshape(rows, nb, BLOCK)
    top = full.abs().amax(2, keepdim=True)
    power = torch.frexp(top)[1].double() - 1.0
    y = full * torch.pow(2.0, -power)                            # the largest in [1, 2)
    octave = torch.frexp(y.abs())[1].double() - 1.0
    if second:
        step = torch.pow(2.0, octave - 3.0)
        q = torch.where(y > 0, (torch.round(y / step) * step).clamp(1.25 * 2.0 ** -31, 2.0), torch.zeros_like(y))
    else:
        step = torch.pow(2.0, torch.clamp(octave + 7.0, min=-6.0) - 10.0)
        q = torch.round(y / step) * step
    return (q * torch.pow(2.0, power)).reshape(rows, -1)[:, :cols]


def exact(case, seed):
    s = _inputs(case, seed)
    c, op = case, case["op"]
    if op == "adamw":
        return _exact_adamw(s)
    live = c["count"] or c["M"]
    need = op in ("linear_grad", "gated_grad")
    leaf = {k: s[k].double().requires_grad_(need) for k in ("x", "w", "wg", "wu", "b", "bu", "r") if s.get(k) is not None}
    act = {"none": lambda g: g, "relu": torch.relu, "sigmoid": torch.sigmoid, "silu": lambda g: g * torch.sigmoid(g),
           "gelu": lambda g: 0.5 * g * torch.erfc(-g / math.sqrt(2.0))}[c["act"]]

    def project(w, b):
        y = torch.mm(leaf["x"][:live], leaf[w])
        return y + leaf[b] if b in leaf else y

    if op in ("gated", "gated_grad"):
        y = act(project("wg", "b")) * project("wu", "bu")
    else:
        y = c["alpha"] * act(project("w", "b"))
        if "r" in leaf:
            y = y + c["beta"] * leaf["r"][:live]
    if not need:
        return torch.cat([y, torch.zeros(c["M"] - live, c["N"], dtype=torch.float64, device=DEV)])
    names = [k for k in ("x", "w", "wg", "wu", "b", "bu", "r") if k in leaf]
    return list(torch.autograd.grad((y * s["d"][:live].double()).sum(), [leaf[k] for k in names]))


def _exact_adamw(s):
    c = s["case"]
    square = 0.0
    for e in s["entries"]:
        g = e["g"][:c["count"]] if e["n"] is not None else e["g"]
        square += float(torch.linalg.vector_norm(g.double())) ** 2
    norm = math.sqrt(square)
    coef = min(1.0, c["max_norm"] / (norm + 1e-6))
    t = c["step"] + 1
    out = [torch.tensor([norm], dtype=torch.float64, device=DEV), torch.tensor([t], dtype=torch.int32, device=DEV)]
    for e in s["entries"]:
        g = coef * (e["g"][:c["count"]] if e["n"] is not None else e["g"]).double()
        rows = slice(None) if e["ids"] is None else e["ids"][:g.shape[0]].long()
        p = e["p"].double()
        small = e["m_exp"] is not None
        m, v = (_in_64(e["m"], e["m_exp"], False), _in_64(e["v"], e["v_exp"], True)) if small else (e["m"].double(), e["v"].double())
        m1, v1 = BETA1 * m[rows] + (1.0 - BETA1) * g, BETA2 * v[rows] + (1.0 - BETA2) * g ** 2
        p[rows] = p[rows] - LR * e["decay"] * p[rows] - LR * (m1 / -math.expm1(t * math.log(BETA1))) / (
            torch.sqrt(v1 / -math.expm1(t * math.log(BETA2))) + EPS)
        m[rows], v[rows] = (_held_64(m1, False), _held_64(v1, True)) if small else (m1, v1)
        out += [p, m, v]
        if e["copy"] is not None:
            out.append(p)
    return out


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    c, op = case, case["op"]
    if op == "adamw":
        total = flops = 0.0
        shapes = _shapes(c) + ([(c["table_rows"], c["table_dim"], False)] if c["table_rows"] else [])
        for k, (rows, cols, decay) in enumerate(shapes):
            table = c["table_rows"] and k == len(shapes) - 1
            n = (c["count"] or c["positions"]) if table and c["positions"] else rows
            if table and c["positions"]:
                total += 4 * n
            small = c["state"] == "8bit" and rows > 1
            total += n * cols * (2 * SIZE[c["p"]] + SIZE[c["g"]] + (2 if c["copies"] and decay else 0) + (4 if small else 16))
            if small:
                total += 4 * n * ((cols + BLOCK - 1) // BLOCK) + 8 * rows * cols      # (the states' values are outputs too)
            flops += 20 * n * cols
        return {"bytes": total, "flops": flops}
    M, K, N = c["count"] or c["M"], c["K"], c["N"]
    b = SIZE[c["block"]]
    gated = op in ("gated", "gated_grad")
    weights = K * N * b * (2 if gated else 1)
    product = 2.0 * M * K * N * (2 if gated else 1)
    if op == "linear":
        return {"bytes": M * K * b + weights + M * N * SIZE[c["stream"]] * (2 if c["residual"] else 1), "flops": product}
    if op == "gated":
        return {"bytes": M * K * b + weights + M * N * b, "flops": product}
    d = b if gated else SIZE[c["stream"]]
    again = product if gated or c["act"] != "none" else 0.0          # (what the activation was given is formed again)
    return {"bytes": 2 * M * K * b + 2 * weights + M * N * d * (2 if not gated and c["residual"] else 1), "flops": 2 * product + again}
