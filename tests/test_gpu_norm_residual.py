"""A block's gated residual with the norms around it, and its gradient, against 64 bits."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import plain_operators as plain

TYPES = {"f32": (torch.float32, torch.float32), "bf16": (torch.bfloat16, torch.bfloat16), "mixed": (torch.float32, torch.bfloat16)}
SHAPES = [(1, 1), (1, 64), (3, 2), (5, 17), (256, 64), (77, 100), (300, 256), (130, 602), (23, 333), (40, 512), (41, 1024), (9, 1500), (65, 2047), (4, 4096), (3, 9001), (2, 40000)]


@pytest.fixture(scope="module")
def env():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2101_07706_amd import csgs
    csgs.lib()
    return csgs, torch.device("cuda:0")


def roundings(F, rows=0):
    """Roundings on the longest chain to a result: sums over a row go through at most F / 64 entries of a lane and a tree, five of them one after the
    other (two means, two deviations, the gradient's), each with some operations around it; `rows` more where rows are summed."""
    return 5 * (F / 64 + 24) + rows


def matrix(M, F, extra, shift, dtype, dev, values=None):
    raw = torch.full((M * (F + extra) + shift + 8,), float("nan"), dtype=dtype, device=dev)
    m = raw[shift:shift + M * (F + extra)].view(M, F + extra)[:, :F]
    if values is not None:
        m.copy_(values)
    return m


class Case:
    def __init__(self, csgs, dev, M, F, types, post="rms", pre="rms", act="linear", gate="full", bias=True, weights=True, x=True, h=True, dy=True, du=True,
                 extra=0, shift=0, alpha=0.7, beta=0.9, eps=1e-5, seed=0, spread=1.0, count=None):
        self.csgs, self.dev, self.M, self.F, self.count = csgs, dev, M, F, count
        self.stream, self.block = TYPES[types]
        self.kw = dict(post=post, pre=pre, act=act)
        g = torch.Generator().manual_seed(seed + 1000 * M + F)
        mk = lambda dt, s=1.0, off=0.0: matrix(M, F, extra, shift, dt, dev, torch.randn(M, F, generator=g) * s + off)
        vec = lambda s, off=0.0: (torch.randn(F, generator=g) * s + off).to(dev)
        self.x = mk(self.stream, spread, 0.3) if x else None
        self.h = mk(self.block, 0.5 * spread, -0.2) if h else None
        if h and M > 2:
            self.h[1].zero_()          # a row without kept edges
        self.gate = None if gate == "none" or not h else mk(self.block, 1.5) if gate == "full" else vec(1.0)
        self.pw, self.qw = (vec(0.2, 1.0), vec(0.2, 1.0)) if weights else (None, None)
        self.pb, self.qb = (vec(0.3), vec(0.3)) if bias else (None, None)
        self.dy = mk(self.stream) if dy else None
        self.du = mk(self.block) if du and pre != "none" else None
        self.alpha, self.beta, self.eps = (float(torch.tensor(v, dtype=torch.float32)) for v in (alpha, beta, eps))
        self.new = lambda dt: matrix(M, F, extra, shift, dt, dev)
        self.M_dev = None if count is None else torch.tensor([count], dtype=torch.int32, device=dev)

    def args(self):
        n = {"none": self.csgs.NORM_NONE, "rms": self.csgs.NORM_RMS, "layer": self.csgs.NORM_LAYER}
        a = {"linear": self.csgs.GATE_LINEAR, "sigmoid": self.csgs.GATE_SIGMOID, "silu": self.csgs.GATE_SILU}
        return dict(gate=self.gate, gate_act=a[self.kw["act"]], post=n[self.kw["post"]], post_w=self.pw, post_b=self.pb, pre=n[self.kw["pre"]], pre_w=self.qw,
                    pre_b=self.qb, eps=self.eps, alpha=self.alpha, beta=self.beta, M_dev=self.M_dev)

    def rows(self):
        return self.M if self.count is None else max(0, min(self.count, self.M))

    def plain_args(self):
        m = self.rows()
        d = lambda t: None if t is None else (t[:m] if t.dim() == 2 else t).double().cpu()
        none = self.kw["post"] == "none"
        return (d(self.x), d(self.h), d(self.gate), self.kw["post"], self.kw["pre"], self.kw["act"], None if none else d(self.pw), None if none else d(self.pb),
                d(self.qw), d(self.qb), self.eps, self.alpha, self.beta)

    def forward(self):
        y, u = self.new(self.stream), self.new(self.block) if self.kw["pre"] != "none" else None
        self.csgs.csgs_norm_residual(self.x, self.h, y, u, **self.args())
        return y, u

    def backward(self):
        F, dev = self.F, self.dev
        vec = lambda: torch.full((F,), float("nan"), device=dev)
        o = dict(dx=self.new(self.stream) if self.x is not None else None, dh=self.new(self.block) if self.h is not None else None, dgate=None, dpost_w=None,
                 dpost_b=None, dpre_w=None, dpre_b=None)
        if self.gate is not None:
            o["dgate"] = self.new(self.block) if self.gate.dim() == 2 else vec()
        if self.h is not None and self.kw["post"] != "none":
            o["dpost_w"], o["dpost_b"] = vec(), vec()
        if self.du is not None:
            o["dpre_w"], o["dpre_b"] = vec(), vec()
        scratch = torch.full((self.csgs.csgs_norm_residual_grad_scratch_bytes(self.M, F),), 0xFF, dtype=torch.uint8, device=dev)
        self.csgs.csgs_norm_residual_grad(self.x, self.h, self.dy, self.du, *o.values(), scratch, **self.args())
        return o

    def check(self):
        m, F = self.rows(), self.F
        y, u = self.forward()
        want = plain.residual(*self.plain_args())
        plain.check(y[:m], want.y, want.y_mag, roundings(F), "y")
        if u is not None:
            plain.check(u[:m], want.u, want.u_mag, roundings(F), "u")
            assert bool(torch.isnan(u[m:].float()).all())
        assert bool(torch.isnan(y[m:].float()).all()), "wrote past the count"
        if self.dy is None and self.du is None:
            return
        o = self.backward()
        d = lambda t: None if t is None else t[:m].double().cpu()
        z = plain.residual_grad(*self.plain_args(), d(self.dy), d(self.du))
        for k in ("dx", "dh"):
            if o[k] is not None:
                plain.check(o[k][:m], *getattr(z, k), roundings(F), k)
                assert bool(torch.isnan(o[k][m:].float()).all()), "wrote past the count"
        if self.gate is not None:
            if self.gate.dim() == 2:
                plain.check(o["dgate"][:m], *z.dg, roundings(F), "dgate")
            else:
                plain.check(o["dgate"], *z.dg_sum, roundings(F, m), "dgate")
        for k in ("dpost_w", "dpost_b", "dpre_w", "dpre_b"):
            if o[k] is not None:
                plain.check(o[k], *getattr(z, k), roundings(F, m), k)
        again = self.backward()
        for k in o:
            if o[k] is not None:
                assert torch.equal(torch.nan_to_num(o[k].float(), 3.0), torch.nan_to_num(again[k].float(), 3.0)), f"{k}: two calls differ"


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("M,F", SHAPES)
def test_shapes(env, M, F, norm, types):
    Case(*env, M, F, types, post=norm, pre=norm, act="sigmoid", gate="full").check()


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("M,F,extra,shift", [(33, 100, 4, 0), (33, 100, 1, 1), (20, 256, 3, 5), (20, 602, 0, 1), (7, 1024, 7, 2), (3, 9001, 1, 1)])
def test_rows_that_start_anywhere(env, M, F, extra, shift, types):
    Case(*env, M, F, types, post="layer", pre="rms", act="silu", gate="row", extra=extra, shift=shift).check()


@pytest.mark.parametrize("post", ["none", "rms", "layer"])
@pytest.mark.parametrize("pre", ["none", "rms", "layer"])
@pytest.mark.parametrize("act", ["linear", "sigmoid", "silu"])
@pytest.mark.parametrize("gate", ["none", "row", "full"])
def test_kinds(env, post, pre, act, gate):
    Case(*env, 21, 72, "mixed", post=post, pre=pre, act=act, gate=gate, bias=act != "silu", weights=act != "linear").check()


@pytest.mark.parametrize("F", [48, 130, 5000])
@pytest.mark.parametrize("x,h,dy,du", [(True, False, True, True), (False, True, True, True), (True, True, True, False), (True, True, False, True), (True, False, False, True),
                                       (False, True, False, True)])
def test_absent_parts(env, F, x, h, dy, du):
    Case(*env, 19, F, "f32", post="layer", pre="layer", act="sigmoid", gate="full" if h else "none", x=x, h=h, dy=dy, du=du).check()


@pytest.mark.parametrize("M", [1, 2, 255, 3000, 20000])
def test_many_rows(env, M):
    for F, gate in ((64, "row"), (33, "full"), (256, "row")):
        Case(*env, M, F, "f32", post="rms", pre="layer", act="sigmoid", gate=gate).check()


@pytest.mark.parametrize("M,count", [(40, 0), (40, 1), (40, 39), (40, 400), (40, -5), (5000, 2500)])
def test_rows_up_to_a_device_count(env, M, count):
    for F in (100, 6000):
        Case(*env, M, F, "f32", post="layer", pre="rms", act="silu", gate="row", count=count).check()


@pytest.mark.parametrize("spread,eps", [(1e-4, 1e-5), (1e3, 1e-5), (1e-12, 1e-12), (1.0, 0.0)])
def test_sizes_of_values(env, spread, eps):
    c = Case(*env, 12, 96, "f32", post="rms", pre="layer", act="sigmoid", gate="full", spread=spread, eps=eps)
    c.h[1].fill_(0.01 * spread)     # (eps = 0 has no value for a row of zeros)
    c.check()


def test_a_row_depends_on_itself_alone(env):
    """NaN and infinities stay in their row; sums over rows show them."""
    csgs, dev = env
    c = Case(csgs, dev, 70, 128, "f32", act="sigmoid", gate="full")
    y0, u0 = c.forward()
    o0 = c.backward()
    c.h[7, 3], c.x[11, 100], c.dy[20, 1], c.gate[30, 2] = float("nan"), float("inf"), float("nan"), float("-inf")
    y1, u1 = c.forward()
    o1 = c.backward()
    keep = torch.ones(70, dtype=torch.bool, device=dev)
    keep[[7, 11, 20, 30]] = False
    assert torch.equal(y0[keep], y1[keep]) and torch.equal(u0[keep], u1[keep])
    for k in ("dx", "dh", "dgate"):
        assert torch.equal(o0[k][keep], o1[k][keep]), k
    assert bool(torch.isnan(y1[7]).all()) and bool(torch.isnan(u1[11]).any()) and bool(torch.isfinite(u1[20]).all())
    assert bool(torch.isfinite(y1[30]).all())          # the logistic function of -infinity is 0
    assert bool(torch.isnan(o1["dpost_w"]).any())


@pytest.mark.parametrize("F", [100, 256, 6001])
def test_in_place(env, F):
    csgs, dev = env
    c = Case(csgs, dev, 50, F, "bf16", post="layer", pre="rms", act="silu", gate="full")
    y, u = c.forward()
    o = c.backward()
    h, x = c.h.clone(), c.x.clone()
    csgs.csgs_norm_residual(x, h, x, h, **c.args())
    assert torch.equal(x, y) and torch.equal(h, u)
    dy, du, gate = c.dy.clone(), c.du.clone(), c.gate.clone()
    scratch = torch.empty(csgs.csgs_norm_residual_grad_scratch_bytes(50, F), dtype=torch.uint8, device=dev)
    kw = c.args()
    kw["gate"] = gate
    csgs.csgs_norm_residual_grad(c.x, c.h, dy, du, dy, du, gate, None, None, None, None, scratch, **kw)
    assert torch.equal(dy, o["dx"]) and torch.equal(du, o["dh"]) and torch.equal(gate, o["dgate"])


def test_single_outputs(env):
    """u alone and y alone are what both give together."""
    csgs, dev = env
    c = Case(csgs, dev, 30, 200, "f32")
    y, u = c.forward()
    y1, u1 = c.new(torch.float32), c.new(torch.float32)
    csgs.csgs_norm_residual(c.x, c.h, y1, None, **c.args())
    csgs.csgs_norm_residual(c.x, c.h, None, u1, **c.args())
    assert torch.equal(y, y1) and torch.equal(u, u1)


@pytest.mark.parametrize("post,pre,act,gate", [("rms", "layer", "sigmoid", "full"), ("layer", "rms", "silu", "row")])
def test_gradient_against_differences(env, post, pre, act, gate):
    """The kernel's gradients against central differences of the 64-bit forward pass."""
    c = Case(*env, 6, 10, "f32", post=post, pre=pre, act=act, gate=gate)
    o = c.backward()
    args = list(c.plain_args())
    dy, du = c.dy.double().cpu(), c.du.double().cpu()

    def loss(a):
        f = plain.residual(*a)
        return float((f.y * dy).sum() + (f.u * du).sum())

    step = 1e-5     # error of a central difference: step^2 times a third derivative, and 2^-53 L / step
    for name, k in (("dx", 0), ("dh", 1), ("dgate", 2), ("dpost_w", 6), ("dpost_b", 7), ("dpre_w", 8), ("dpre_b", 9)):
        got, base = o[name].double().cpu(), args[k]
        for at in [(0,) * base.dim(), tuple(s - 1 for s in base.shape), tuple(s // 2 for s in base.shape)]:
            v = []
            for sign in (1, -1):
                moved = base.clone()
                moved[at] += sign * step
                v.append(loss(args[:k] + [moved] + args[k + 1:]))
            want = (v[0] - v[1]) / (2 * step)
            if base.dim() == 2 and at[0] == 1 and name == "dh":
                continue     # the row of zeros bends within the step
            assert abs(float(got[at]) - want) <= 1e-5 * max(1.0, abs(want)), (name, at, float(got[at]), want)


def test_rows_past_32_bits(env):
    csgs, dev = env
    M, F, ld = 70_001, 40, 1 << 16
    assert (M - 1) * ld > 1 << 32
    big = torch.empty(M * ld, dtype=torch.bfloat16, device=dev).view(M, ld)
    cols = [big[:, k * 64:k * 64 + F] for k in range(7)]
    g = torch.Generator().manual_seed(1)
    for k in range(4):
        cols[k].copy_(torch.randn(M, F, generator=g))
    x, h, dy, du, y, u, dh = cols
    kw = dict(post=csgs.NORM_RMS, pre=csgs.NORM_LAYER)
    csgs.csgs_norm_residual(x, h, y, u, **kw)
    scratch = torch.empty(csgs.csgs_norm_residual_grad_scratch_bytes(M, F), dtype=torch.uint8, device=dev)
    csgs.csgs_norm_residual_grad(x, h, dy, du, None, dh, None, None, None, None, None, scratch, **kw)
    torch.cuda.synchronize()
    last = slice(M - 5, M)
    d = lambda t: t[last].double().cpu()
    a = (d(x), d(h), None, "rms", "layer", "linear", None, None, None, None, float(torch.tensor(1e-5)), 1.0, 1.0)
    want = plain.residual(*a)
    plain.check(y[last], want.y, want.y_mag, roundings(F), "y")
    plain.check(u[last], want.u, want.u_mag, roundings(F), "u")
    plain.check(dh[last], *plain.residual_grad(*a, d(dy), d(du)).dh, roundings(F), "dh")


def test_on_another_stream_and_replayed(env):
    csgs, dev = env
    c = Case(csgs, dev, 500, 96, "f32", act="silu", gate="row")
    y, u = c.new(torch.float32), c.new(torch.float32)
    dx, dh = c.new(torch.float32), c.new(torch.float32)
    vs = [torch.empty(96, device=dev) for _ in range(5)]
    scratch = torch.empty(csgs.csgs_norm_residual_grad_scratch_bytes(500, 96), dtype=torch.uint8, device=dev)

    def step(stream):
        csgs.csgs_norm_residual(c.x, c.h, y, u, stream=stream, **c.args())
        csgs.csgs_norm_residual_grad(c.x, c.h, c.dy, c.du, dx, dh, *vs, scratch, stream=stream, **c.args())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    first = [t.clone() for t in [y, u, dx, dh] + vs]
    step(None)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, [y, u, dx, dh] + vs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(None)
    for k in range(3):
        for t in (c.x, c.h, c.dy, c.du):
            t.normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in [y, u, dx, dh] + vs]
        step(None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, [y, u, dx, dh] + vs)), f"replay {k}"


def test_recorded_calls(env):
    """Calls marshalled once and issued again see what the buffers hold then."""
    csgs, dev = env
    c = Case(csgs, dev, 60, 72, "mixed", act="silu", gate="row", count=50)
    y, u = c.new(torch.float32), c.new(torch.bfloat16)
    dx, dh, dw = c.new(torch.float32), c.new(torch.bfloat16), torch.empty(72, device=dev)
    scratch = torch.empty(csgs.csgs_norm_residual_grad_scratch_bytes(60, 72), dtype=torch.uint8, device=dev)
    ids, table, out = torch.arange(60, dtype=torch.int32, device=dev).flip(0).contiguous(), torch.randn(60, 72, device=dev), torch.empty(60, 72, device=dev)

    def calls():
        csgs.csgs_embed(table, ids, out, scale=2.0)
        csgs.csgs_norm_residual(c.x, c.h, y, u, **c.args())
        csgs.csgs_norm_residual_grad(c.x, c.h, c.dy, c.du, dx, dh, None, dw, None, None, None, scratch, **c.args())

    with csgs.record() as plan:
        calls()
    for _ in range(2):
        c.x.normal_()
        table.normal_()
        plan.run()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, y[:50], u[:50], dx[:50], dh[:50], dw)]
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, y[:50], u[:50], dx[:50], dh[:50], dw)))
        assert torch.equal(out, 2.0 * table.flip(0))


@pytest.mark.parametrize("F", [3, 100, 9000])
def test_without_a_norm_nothing_is_divided_by(env, F):
    """No norm before the gate: the gradient of h does not depend on h, whatever it holds."""
    csgs, dev = env
    c = Case(csgs, dev, 9, F, "f32", post="none", pre="none", act="sigmoid", gate="row", du=False)
    want = c.backward()["dh"].clone()
    c.h[2, 1], c.h[3, 0], c.h[4] = float("inf"), float("nan"), float("-inf")
    assert torch.equal(c.backward()["dh"], want)


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("gate", ["row", "full"])
@pytest.mark.parametrize("F", [2049, 2052, 2999, 3508, 4095, 4100, 6001, 6148, 8190])
def test_wide_rows(env, F, gate, bias, types):
    Case(*env, 5, F, types, post="layer", pre="rms", act="silu", gate=gate, bias=bias).check()


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("F", [2500, 4096, 5000, 8192])
def test_several_wide_rows_a_block(env, F, types):
    Case(*env, 1100, F, types, post="rms", pre="layer", act="sigmoid", gate="full", count=1060).check()


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("bias,gate", [(False, "full"), (True, "row")])
@pytest.mark.parametrize("M,F", [(5, 769), (1100, 1000), (5, 1024), (5, 1025), (2100, 1300), (5, 1531), (5, 1536), (5, 1537)])
def test_rows_of_two_wavefronts(env, M, F, bias, gate, types):
    Case(*env, M, F, types, post="rms", pre="layer", act="silu", gate=gate, bias=bias).check()


@pytest.mark.parametrize("act", ["sigmoid", "silu"])
@pytest.mark.parametrize("gate", ["row", "full"])
@pytest.mark.parametrize("F", [3, 100, 1000, 6000])
def test_gates_open_and_shut(env, F, gate, act):
    """The gate itself and its derivative, to a number of roundings of their own size (y = a(g), dgate = a'(g) for h = dy = 1 without norms): an ulp each of the
    exponential and the reciprocal, the operations between them, |g| / 20 for the constant that the exponential's argument is formed with."""
    csgs, dev = env
    special = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 8.0, -8.0, 12.0, -12.0, 16.7, -16.7, 17.5, -17.5, 20.0, -20.0, 40.0, -40.0, 80.0, -80.0, 1e4, -1e4, 1e30, -1e30])
    g = torch.randn(4096, generator=torch.Generator().manual_seed(F)) * 10
    g[:2000] = torch.linspace(-80, 80, 2000)
    g[2000:2000 + len(special)] = special
    M = (len(g) + F - 1) // F
    g = torch.cat([g, torch.zeros(M * F - len(g))]).view(M, F)
    one, y, dg = torch.ones(1, F, device=dev), [], []
    scratch = torch.empty(csgs.csgs_norm_residual_grad_scratch_bytes(M, F), dtype=torch.uint8, device=dev)
    kw = dict(gate_act=csgs.GATE_SIGMOID if act == "sigmoid" else csgs.GATE_SILU, post=csgs.NORM_NONE, pre=csgs.NORM_NONE)
    none = [None] * 4
    if gate == "full":
        one, gates = torch.ones(M, F, device=dev), [g.to(dev)]
    else:
        gates = [row.to(dev) for row in g]
    for v in gates:
        y.append(torch.empty_like(one))
        dg.append(torch.empty_like(v))
        csgs.csgs_norm_residual(None, one, y[-1], None, gate=v, **kw)
        csgs.csgs_norm_residual_grad(None, one, one, None, None, None, dg[-1], *none, scratch, gate=v, **kw)
    y, dg = torch.cat(y).double().cpu(), torch.cat([t.view(-1, F) for t in dg]).double().cpu()
    g = g.double()
    s, rest = 1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g))
    share = g.abs().clamp(max=100) / 20
    if act == "sigmoid":
        checks = [("gate", y, s, s, 8 + share), ("derivative", dg, s * rest, s * rest, 13 + share)]
    else:
        checks = [("gate", y, g * s, (g * s).abs(), 9 + share), ("derivative", dg, s * (1 + g * rest), s * (1 + g.abs() * rest), 18 + 2 * share)]
    for what, got, want, mag, roundings_ in checks:
        tol = roundings_ * 2.0 ** -24 * mag + 2e-36      # (below 2^-126, and up to |g| times that, nothing is left)
        worst = ((got - want).abs() / tol)
        at = int(worst.argmax())
        assert float(worst.max()) <= 1.0, f"{what}: error {float(worst.max()):.2f} times its bound at g = {float(g.view(-1)[at])}"


@pytest.mark.parametrize("F", [3, 100, 6000])
def test_gates_that_are_not_finite(env, F):
    csgs, dev = env
    inf = float("inf")
    g = torch.full((3, F), inf, device=dev)
    g[1], g[2] = -inf, float("nan")
    one, y, dg = torch.ones(3, F, device=dev), torch.empty(3, F, device=dev), torch.empty(3, F, device=dev)
    scratch = torch.empty(csgs.csgs_norm_residual_grad_scratch_bytes(3, F), dtype=torch.uint8, device=dev)
    kw = dict(gate=g, gate_act=csgs.GATE_SIGMOID, post=csgs.NORM_NONE, pre=csgs.NORM_NONE)
    csgs.csgs_norm_residual(None, one, y, None, **kw)
    csgs.csgs_norm_residual_grad(None, one, one, None, None, None, dg, None, None, None, None, scratch, **kw)
    assert bool((y[0] == 1).all()) and bool((y[1] == 0).all()) and bool(torch.isnan(y[2]).all())
    assert bool((dg[:2] == 0).all()) and bool(torch.isnan(dg[2]).all())


# rows of fewer columns than a piece and of more than a block's registers hold are walked over in memory
WALKED = [1, 2, 3, 8193, 9000]


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("M,count", [(40, 0), (40, 1), (40, 39), (40, 400), (40, -5), (1100, 1060)])
def test_walked_rows_up_to_a_device_count(env, M, count, types):
    for F in (3, 9000) if M < 1000 else (2, 8193):
        Case(*env, M, F, types, post="layer", pre="rms", act="silu", gate="row" if M < 1000 else "full", count=count).check()


@pytest.mark.parametrize("types", ["f32", "bf16"])
@pytest.mark.parametrize("F", WALKED)
def test_walked_rows_in_place(env, F, types):
    csgs, dev = env
    for gate in ("full", "row"):
        c = Case(csgs, dev, 50, F, types, post="layer", pre="rms", act="silu", gate=gate)
        y, u = c.forward()
        o = c.backward()
        h, x = c.h.clone(), c.x.clone()
        csgs.csgs_norm_residual(x, h, x, h, **c.args())
        assert torch.equal(x, y) and torch.equal(h, u)
        for onto in ("du", "h"):             # where the gradient of h goes
            dy, du, h, kw = c.dy.clone(), c.du.clone(), c.h.clone(), c.args()
            kw["gate"] = c.gate.clone()
            dh = du if onto == "du" else h
            scratch = torch.empty(csgs.csgs_norm_residual_grad_scratch_bytes(50, F), dtype=torch.uint8, device=dev)
            vec = [torch.empty(F, device=dev) for _ in range(4)]
            dgate = kw["gate"] if gate == "full" else torch.empty(F, device=dev)
            csgs.csgs_norm_residual_grad(c.x, h, dy, du, dy, dh, dgate, *vec, scratch, **kw)
            assert torch.equal(dy, o["dx"]) and torch.equal(dh, o["dh"]) and torch.equal(dgate, o["dgate"])
            for v, k in zip(vec, ("dpost_w", "dpost_b", "dpre_w", "dpre_b")):
                assert torch.equal(v, o[k]), k


@pytest.mark.parametrize("F", [3, 9000])
@pytest.mark.parametrize("x,h,dy,du", [(True, False, True, True), (False, True, True, True), (True, True, True, False), (True, True, False, True), (True, False, False, True),
                                       (False, True, False, True)])
def test_absent_parts_of_walked_rows(env, F, x, h, dy, du):
    for types in ("f32", "mixed"):
        Case(*env, 19, F, types, post="layer", pre="layer", act="sigmoid", gate="full" if h else "none", x=x, h=h, dy=dy, du=du).check()


@pytest.mark.parametrize("post,pre", [("none", "rms"), ("none", "layer"), ("rms", "none"), ("layer", "none"), ("none", "none")])
@pytest.mark.parametrize("F", [3, 8193])
def test_walked_rows_without_a_norm(env, F, post, pre):
    for gate in ("none", "row", "full"):
        Case(*env, 9, F, "mixed", post=post, pre=pre, act="sigmoid", gate=gate, bias=F == 3, weights=F != 3).check()
