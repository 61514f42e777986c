"""Products with an epilogue and gated feed-forward blocks, and their gradients, against 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import plain_training as plain

HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
F, B = torch.float32, torch.bfloat16
ACTS = ["none", "relu", "sigmoid", "silu", "gelu"]
# one entry; less than a piece, a tile, a wavefront's rows; whole tiles; just past them; widths that no piece divides; long sums with few outputs
SIZES = [(1, 1, 1), (1, 8, 3), (3, 5, 7), (2, 64, 300), (64, 64, 64), (65, 130, 33), (200, 31, 129), (256, 64, 4), (130, 602, 47), (17, 1000, 300), (300, 257, 260), (5, 4096, 9),
         (16, 513, 40), (9, 40, 1030)]


@pytest.fixture(scope="module")
def env():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2101_07706_amd import csgs
    csgs.lib()
    return csgs, torch.device("cuda:0")


def act_of(csgs, name):
    return {"none": csgs.ACT_NONE, "relu": csgs.ACT_RELU, "sigmoid": csgs.ACT_SIGMOID, "silu": csgs.ACT_SILU, "gelu": csgs.ACT_GELU}[name]


def elem(csgs, t):
    return csgs.F32 if t is F else csgs.BF16


class Maker:
    """Matrices with a gap behind their rows and a first row that starts `shift` entries into its memory; NaN in all that is no entry."""

    def __init__(self, dev, seed, gap=0, shift=0):
        self.dev, self.gen, self.gap, self.shift = dev, torch.Generator().manual_seed(seed), gap, shift

    def room(self, rows, cols, dtype):
        flat = torch.full((rows * (cols + self.gap) + self.shift,), math.nan, dtype=dtype, device=self.dev)
        return flat[self.shift:].view(rows, cols + self.gap)[:, :cols]

    def matrix(self, rows, cols, dtype, std=1.0):
        x = self.room(rows, cols, dtype)
        x.copy_(torch.randn(rows, cols, generator=self.gen) * std)
        return x

    def vector(self, n):
        return torch.randn(n, generator=self.gen).to(self.dev)


REFERENCE = {"device": "cpu"}      # (the largest sizes: in 64 bits on the device, plain products of two matrices)


def cpu(t):
    return None if t is None else t.detach().to(REFERENCE["device"]).double()


def within(got, want, tol, what):
    got = got.detach().to(want.device)
    off = (got.double() - want).abs()
    tol = HALF_ULP[got.dtype] * want.abs() * 1.01 + tol * (1 + 2 * HALF_ULP[got.dtype]) + 1e-37
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    worst = float((off / tol).max()) if got.numel() else 0.0
    assert worst <= 1.0, f"{what}: error {worst:.3f} times its bound"


# Bounds.  A sum of n products in float: (n + 2) roundings of the sum of their absolute values (mag).  (The matrix cores form a step's sum in their own order, and cut off once a step
# what lies below its largest term's float: counted as one more rounding for each product.)  An activation: its derivative, below 1.13, times its argument's error, and 12 + |z| roundings
# of its own (the error of the exponential's argument), of its derivative 16 + |z| and its second derivative, below 0.9 times the argument's error (0.5 for z s(z); 0.25 for s).
ULP = 2.0 ** -24


def pre(a, w, bias):
    z, mag = a @ w, a.abs() @ w.abs()
    if bias is not None:
        z, mag = z + bias, mag + bias.abs()
    return z, (2 * a.shape[1] + 3) * ULP * mag


def through(name, z, err):
    """act(z), its derivative, and bounds of their errors."""
    a, da = plain.act(name, z)
    if name == "none":
        return a, da, err, torch.zeros_like(z)
    if name == "relu":
        return a, da, err, (z.abs() <= err).double()
    size = torch.maximum(a.abs(), (z.abs() * torch.sigmoid(1.7 * z)).abs() if name != "sigmoid" else a.abs())
    grow = da.abs() + (z.abs() + 1) * (torch.sigmoid(z) if name != "gelu" else 0.4 * torch.exp(-z * z / 2)) * (1 if name != "sigmoid" else 0) + (torch.exp(-z.abs()) if name == "sigmoid" else 0)
    return a, da, 1.13 * err + (12 + z.abs()) * ULP * size, 0.9 * err + (16 + z.abs() + (z * z if name == "gelu" else 0)) * ULP * grow


def check_linear(csgs, dev, M, K, N, ts, act, bias, residual, alpha, beta, count=None, gap=0, shift=0, seed=0, in_place=False, grads=True):
    tb, ty = ts
    mk = Maker(dev, seed, gap, shift)
    a, w = mk.matrix(M, K, tb), mk.matrix(K, N, tb, 1 / math.sqrt(K))
    b = mk.vector(N) if bias else None
    r = mk.matrix(M, N, ty) if residual else None
    live = M if count is None else min(max(count, 0), M)
    a[live:] = math.nan
    if r is not None:
        r[live:] = math.nan
    n_dev = None if count is None else torch.tensor([count], dtype=torch.int32, device=dev)
    A, W, Bv, R = cpu(a)[:live], cpu(w), cpu(b), cpu(r)
    z, zerr = pre(A, W, Bv)
    v, dv, verr, dverr = through(act, z, zerr)
    want, tol = alpha * v, abs(alpha) * verr + ULP * abs(alpha) * v.abs()
    if residual:
        want, tol = want + beta * R[:live], tol + 2 * ULP * (abs(beta) * R[:live].abs() + abs(alpha) * v.abs())
    y = r if in_place else mk.room(M, N, ty)
    csgs.csgs_linear(a, w, y, bias=b, r=r, act=act_of(csgs, act), alpha=alpha, beta=beta, M_dev=n_dev)
    within(y[:live], want, tol, "y")
    assert bool(y[live:].isnan().all()), "rows past the count"
    if not grads:
        return
    dy = mk.matrix(M, N, ty)
    dy[live:] = math.nan
    D = cpu(dy)[:live]
    t = alpha * D * dv
    terr = abs(alpha) * D.abs() * dverr + 3 * ULP * t.abs()
    # (t as an operand: rounded to the operands' type)
    oerr = terr + HALF_ULP[tb] * (t.abs() + terr) * (1 if tb is B else 0)
    da, dw = mk.room(M, K, tb), mk.room(K, N, tb)
    db = torch.full((N,), math.nan, device=dev) if bias else None
    dr = (dy if in_place else mk.room(M, N, ty)) if residual else None
    nbytes = csgs.csgs_linear_grad_scratch_bytes(M, K, N, elem(csgs, tb))
    scratch = torch.full((nbytes + 256,), 170, dtype=torch.uint8, device=dev)
    csgs.csgs_linear_grad(a, w, dy, da, dw, db, dr, scratch[:nbytes], bias=b, act=act_of(csgs, act), alpha=alpha, beta=beta, M_dev=n_dev)
    assert bool((scratch[nbytes:] == 170).all())
    within(da[:live], t @ W.t(), oerr @ W.abs().t() + (2 * N + 3) * ULP * (t.abs() @ W.abs().t()), "da")
    within(dw, A.t() @ t, A.abs().t() @ oerr + (2 * live + 3) * ULP * (A.abs().t() @ t.abs()), "dw")
    assert bool(da[live:].isnan().all()), "rows past the count"
    if bias:
        within(db, t.sum(0), terr.sum(0) + (live + 3) * ULP * t.abs().sum(0), "dbias")
    if residual:
        within(dr[:live], beta * D, ULP * abs(beta) * D.abs(), "dr")
        assert bool(dr[live:].isnan().all()), "rows past the count"


@pytest.mark.parametrize("ts", [(F, F), (B, B), (B, F)], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_linear(env, size, ts):
    csgs, dev = env
    k = SIZES.index(size)
    for i in range(3):
        check_linear(csgs, dev, *size, ts, ACTS[(k + i) % 5], bias=i != 1, residual=i != 2, alpha=[1.0, 0.5, -0.3][i], beta=[1.0, 0.9, 0.0][i], gap=[0, 8, 3][i], shift=[0, 8, 5][i],
                     seed=k, in_place=i == 1)


@pytest.mark.parametrize("ts", [(F, F), (B, B), (B, F)], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("act", ACTS)
def test_linear_rows_up_to_a_device_count(env, act, ts):
    csgs, dev = env
    for k, count in enumerate((0, 1, 63, 64, 130, 201, 500, -3)):
        check_linear(csgs, dev, 201, 100, 70, ts, act, bias=k % 2 == 0, residual=k % 3 == 0, alpha=0.5, beta=2.0, count=count, gap=k % 3, seed=k)


# sizes that tiles of 128 and 256 rows and parts of long sums are taken for
LARGE = [(2053, 72, 2051), (4100, 200, 1030), (20_001, 100, 48), (40, 96, 5000), (33_000, 64, 64)]


@pytest.mark.parametrize("ts", [(F, F), (B, B), (B, F)], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("size", LARGE, ids=str)
def test_linear_large(env, size, ts):
    csgs, dev = env
    for i, act in enumerate(("none", "gelu")):
        check_linear(csgs, dev, *size, ts, act, bias=True, residual=True, alpha=0.5, beta=1.0, count=[None, size[0] - 77][i], gap=[0, 1][i], seed=i)


@pytest.fixture
def on_device():
    REFERENCE["device"] = "cuda"
    yield
    REFERENCE["device"] = "cpu"


# tiles of 256 that go straight to LDS: more rows than whole tiles, k that ends inside a chunk, columns inside a tile and a piece, rows on multiples of 4 bytes
@pytest.mark.parametrize("ts", [(B, B), (B, F)], ids=["bf16", "mixed"])
@pytest.mark.parametrize("size", [(21_007, 520, 1032), (52_000, 72, 40), (51_200, 1000, 8), (300, 8, 52_002), (300, 2056, 20_050)], ids=str)
def test_linear_straight_to_lds(env, size, ts, on_device):
    csgs, dev = env
    M = size[0]
    for i, (act, count, gap, shift) in enumerate((("none", None, 0, 0), ("silu", M - 77, 6, 2), ("none", M // 3, 8, 2), ("gelu", 0, 0, 8))):
        check_linear(csgs, dev, *size, ts, act, bias=i != 2, residual=i != 1, alpha=0.5, beta=-1.0, count=count, gap=gap, shift=shift, seed=i, in_place=i == 2)


@pytest.mark.parametrize("size", [(21_007, 520, 1032), (51_300, 72, 40), (300, 8, 26_002), (700, 2056, 10_050)], ids=str)
def test_gated_straight_to_lds(env, size, on_device):
    csgs, dev = env
    M = size[0]
    for i, (act, count, gap, shift) in enumerate((("silu", None, 0, 0), ("gelu", M - 77, 6, 2), ("none", M // 3, 8, 2), ("relu", 0, 0, 8))):
        check_gated(csgs, dev, *size, B, act, bias=i != 2, count=count, gap=gap, shift=shift, seed=i, halves=i == 2)


# tiles of 64 by one and by four groups of wavefronts, of 32 rows by eight; gradients' parts of one chunk and of many
TILES = [(8200, 520, 260), (4064, 1000, 16), (1024, 300, 70), (1000, 257, 600), (96, 2048, 130)]


@pytest.mark.parametrize("ts", [(F, F), (B, B), (B, F)], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("size", TILES, ids=str)
def test_linear_over_tiles(env, size, ts, on_device):
    csgs, dev = env
    M = size[0]
    for i, (act, count, gap) in enumerate((("none", None, 0), ("silu", M - 33, 3), ("gelu", 40, 8))):
        check_linear(csgs, dev, *size, ts, act, bias=i != 2, residual=i != 1, alpha=0.5, beta=-1.0, count=count, gap=gap, seed=i)


@pytest.mark.parametrize("tb", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", TILES, ids=str)
def test_gated_over_tiles(env, size, tb, on_device):
    csgs, dev = env
    check_gated(csgs, dev, *size, tb, "silu", bias=True, gap=0, seed=1)
    check_gated(csgs, dev, *size, tb, "gelu", bias=False, count=size[0] - 33, gap=1, seed=2)


def check_gated(csgs, dev, M, K, N, tb, act, bias, count=None, gap=0, shift=0, seed=0, halves=False):
    mk = Maker(dev, seed, gap, shift)
    x = mk.matrix(M, K, tb)
    if halves:
        both = mk.matrix(K, 2 * N, tb, 1 / math.sqrt(K))
        wg, wu = both[:, :N], both[:, N:]
    else:
        wg, wu = mk.matrix(K, N, tb, 1 / math.sqrt(K)), mk.matrix(K, N, tb, 1 / math.sqrt(K))
    bg, bu = (mk.vector(N), mk.vector(N)) if bias else (None, None)
    live = M if count is None else min(max(count, 0), M)
    x[live:] = math.nan
    n_dev = None if count is None else torch.tensor([count], dtype=torch.int32, device=dev)
    X, G, U = cpu(x)[:live], cpu(wg), cpu(wu)
    g, gerr = pre(X, G, cpu(bg))
    u, uerr = pre(X, U, cpu(bu))
    v, dv, verr, dverr = through(act, g, gerr)
    h = mk.room(M, N, tb)
    csgs.csgs_gated(x, wg, wu, h, bg=bg, bu=bu, act=act_of(csgs, act), M_dev=n_dev)
    within(h[:live], v * u, verr * (u.abs() + uerr) + uerr * v.abs() + ULP * (v * u).abs(), "h")
    assert bool(h[live:].isnan().all()), "rows past the count"
    dh = mk.matrix(M, N, tb)
    dh[live:] = math.nan
    D = cpu(dh)[:live]
    tg, tu = D * u * dv, D * v
    tgerr = D.abs() * (uerr * (dv.abs() + dverr) + u.abs() * dverr) + 3 * ULP * tg.abs()
    tuerr = D.abs() * verr + 2 * ULP * tu.abs()
    half = HALF_ULP[tb] if tb is B else 0.0
    og, ou = tgerr + half * (tg.abs() + tgerr), tuerr + half * (tu.abs() + tuerr)
    dx, dwg, dwu = mk.room(M, K, tb), mk.room(K, N, tb), mk.room(K, N, tb)
    dbg, dbu = (torch.full((N,), math.nan, device=dev) for _ in range(2)) if bias else (None, None)
    nbytes = csgs.csgs_gated_grad_scratch_bytes(M, K, N, elem(csgs, tb))
    scratch = torch.full((nbytes + 256,), 170, dtype=torch.uint8, device=dev)
    csgs.csgs_gated_grad(x, wg, wu, dh, dx, dwg, dwu, dbg, dbu, scratch[:nbytes], bg=bg, bu=bu, act=act_of(csgs, act), M_dev=n_dev)
    assert bool((scratch[nbytes:] == 170).all())
    mag = tg.abs() @ G.abs().t() + tu.abs() @ U.abs().t()
    within(dx[:live], tg @ G.t() + tu @ U.t(), og @ G.abs().t() + ou @ U.abs().t() + (4 * N + 3) * ULP * mag, "dx")
    assert bool(dx[live:].isnan().all()), "rows past the count"
    for name, d, t, o in (("dwg", dwg, tg, og), ("dwu", dwu, tu, ou)):
        within(d, X.t() @ t, X.abs().t() @ o + (2 * live + 3) * ULP * (X.abs().t() @ t.abs()), name)
    if bias:
        for name, d, t, e in (("dbg", dbg, tg, tgerr), ("dbu", dbu, tu, tuerr)):
            within(d, t.sum(0), e.sum(0) + (live + 3) * ULP * t.abs().sum(0), name)


@pytest.mark.parametrize("tb", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gated(env, size, tb):
    csgs, dev = env
    k = SIZES.index(size)
    for i in range(3):
        check_gated(csgs, dev, *size, tb, ACTS[(k + 2 * i) % 5], bias=i != 1, gap=[0, 8, 3][i], shift=[0, 8, 5][i], seed=k, halves=i == 1)


@pytest.mark.parametrize("tb", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
def test_gated_rows_up_to_a_device_count(env, act, tb):
    csgs, dev = env
    for k, count in enumerate((0, 1, 63, 64, 130, 201, 500, -3)):
        check_gated(csgs, dev, 201, 100, 70, tb, act, bias=k % 2 == 0, count=count, gap=k % 3, seed=k)


@pytest.mark.parametrize("tb", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", LARGE, ids=str)
def test_gated_large(env, size, tb):
    csgs, dev = env
    check_gated(csgs, dev, *size, tb, "silu", bias=True, gap=0, seed=1)
    check_gated(csgs, dev, *size, tb, "gelu", bias=False, count=size[0] - 77, gap=1, seed=2)


@pytest.mark.parametrize("act", ACTS)
def test_gradients_against_differences(env, act):
    """<gradient, direction> against the difference of the 64-bit forward along it."""
    csgs, dev = env
    mk = Maker(dev, 5)
    M, K, N = 33, 40, 50
    x, wg, wu, w = mk.matrix(M, K, F), mk.matrix(K, N, F, 0.2), mk.matrix(K, N, F, 0.2), mk.matrix(K, N, F, 0.2)
    bg, bu, r, d = mk.vector(N), mk.vector(N), mk.matrix(M, N, F), mk.matrix(M, N, F)
    f = lambda z: plain.act(act, z)[0]
    D = cpu(d)
    scratch = torch.empty(csgs.csgs_gated_grad_scratch_bytes(M, K, N, csgs.F32), dtype=torch.uint8, device=dev)
    dx, dwg, dwu, dw, db, dbu, dr = (torch.zeros_like(t) for t in (x, wg, wu, w, bg, bu, r))

    def compare(forward, leaves, grads):
        dirs = [torch.randn(t.shape, generator=mk.gen, dtype=torch.float64) for t in leaves]
        at = lambda s: float((forward(*[cpu(t) + s * e for t, e in zip(leaves, dirs)]) * D).sum())
        step = 1e-5
        want = (at(step) - at(-step)) / (2 * step)
        got = sum(float((cpu(g) * e).sum()) for g, e in zip(grads, dirs))
        size = sum(float((cpu(g) * e).abs().sum()) for g, e in zip(grads, dirs))
        # (differences: the third derivative and the doubles' roundings over the step; a kink within it for max(z, 0))
        assert abs(got - want) <= 1e-5 * size + (1e-3 * size if act == "relu" else 0.0), (got, want, size)
    csgs.csgs_gated_grad(x, wg, wu, d, dx, dwg, dwu, db, dbu, scratch, bg=bg, bu=bu, act=act_of(csgs, act))
    compare(lambda X, G, U, b, c: f(X @ G + b) * (X @ U + c), [x, wg, wu, bg, bu], [dx, dwg, dwu, db, dbu])
    csgs.csgs_linear_grad(x, w, d, dx, dw, db, dr, scratch, bias=bg, act=act_of(csgs, act), alpha=0.7, beta=-1.5)
    compare(lambda X, W, b, R: 0.7 * f(X @ W + b) - 1.5 * R, [x, w, bg, r], [dx, dw, db, dr])


def test_outputs_one_at_a_time_and_the_same_bits(env):
    csgs, dev = env
    for tb, ty in ((F, F), (B, B), (B, F)):
        for act in ("none", "silu"):
            mk = Maker(dev, 3)
            M, K, N = 700, 90, 130
            x, w, w2 = mk.matrix(M, K, tb), mk.matrix(K, N, tb, 0.1), mk.matrix(K, N, tb, 0.1)
            b, r, d = mk.vector(N), mk.matrix(M, N, ty), mk.matrix(M, N, ty)
            scratch = torch.empty(csgs.csgs_gated_grad_scratch_bytes(M, K, N, elem(csgs, tb)), dtype=torch.uint8, device=dev)

            def linear(want):
                out = [torch.full_like(t, math.nan) if k in want else None for k, t in enumerate((x, w, b, r))]
                csgs.csgs_linear_grad(x, w, d, *out, scratch, bias=b, act=act_of(csgs, act), alpha=0.5)
                return out

            def gated(want):
                out = [torch.full_like(t, math.nan) if k in want else None for k, t in enumerate((x, w, w2, b, b))]
                csgs.csgs_gated_grad(x, w, w2, d.to(tb), *out, scratch, bg=b, bu=b, act=act_of(csgs, act))
                return out
            for f, n in ((linear, 4), (gated, 5)):
                if f is linear:      # (dr alone says that there is a residual)
                    full = f(range(n))
                else:
                    full = f(range(n))
                again = f(range(n))
                for k in range(n):
                    assert torch.equal(full[k], again[k]) and torch.equal(f([k])[k], full[k]), (f, k)


def test_values_that_are_not_finite_stay_in_their_rows(env):
    csgs, dev = env
    for tb in (F, B):
        for N in (40, 300):
            mk = Maker(dev, 4)
            x, w = mk.matrix(70, 90, tb), mk.matrix(90, N, tb, 0.1)
            w.abs_()
            clean = torch.zeros(70, N, dtype=tb, device=dev)
            csgs.csgs_linear(x, w, clean)
            y = torch.zeros_like(clean)
            for bad in (math.nan, math.inf, -math.inf):
                z = x.clone()
                z[33, 7] = bad
                csgs.csgs_linear(z, w, y)
                keep = torch.arange(70, device=dev) != 33
                assert torch.equal(y[keep], clean[keep])
                assert bool((y[33].isnan() if math.isnan(bad) else y[33] == bad).all()), bad
                csgs.csgs_gated(z, w, w, y, act=csgs.ACT_RELU)
                assert bool(torch.isfinite(y[keep]).all())
                assert bool((y[33].isnan() if bad != math.inf else y[33] == math.inf).all()), bad      # (0 times -inf)
            # large values whose products overflow
            z = torch.full((3, 90), 1e30, dtype=tb, device=dev)
            v = torch.full((90, N), 1e30, dtype=tb, device=dev)
            out = torch.zeros(3, N, dtype=tb, device=dev)
            csgs.csgs_linear(z, v, out)
            assert bool((out == math.inf).all())
            csgs.csgs_linear(torch.full_like(z, 3e38), torch.full_like(v, 1e-3), out)
            want = 90 * float(torch.tensor(3e38, dtype=tb)) * float(torch.tensor(1e-3, dtype=tb))
            assert bool(((out.double() - want).abs() <= (2.0 ** -8 if tb is B else 1e-5) * want).all())
            csgs.csgs_linear(torch.full_like(z, 1e-36), torch.full_like(v, 1e-3), out)     # below the smallest number of full precision
            want = 90 * float(torch.tensor(1e-36, dtype=tb)) * float(torch.tensor(1e-3, dtype=tb))
            assert bool(((out.double() - want).abs() <= (2.0 ** -8 if tb is B else 1e-5) * want + 1e-41).all())


def test_rows_far_apart(env):
    """Leading dimensions whose products with a row pass 2^32 bytes and 2^31 entries."""
    csgs, dev = env
    ld, M, K, N = 1_100_000_001, 3, 70, 20
    big = torch.zeros(2 * ld + K, dtype=B, device=dev)
    a = big.as_strided((M, K), (ld, 1))
    mk = Maker(dev, 6)
    a.copy_(mk.matrix(M, K, B))
    w = mk.matrix(K, N, B, 0.1)
    near = a.contiguous()
    y, z = torch.zeros(M, N, device=dev), torch.zeros(M, N, device=dev)
    csgs.csgs_linear(a, w, y)
    csgs.csgs_linear(near, w, z)
    assert torch.equal(y, z) and float(y.abs().sum()) > 0
    d = mk.matrix(M, N, F)
    scratch = torch.empty(csgs.csgs_linear_grad_scratch_bytes(M, K, N, csgs.BF16), dtype=torch.uint8, device=dev)
    outs = []
    for left in (a, near):
        dw = torch.zeros(K, N, dtype=B, device=dev)
        csgs.csgs_linear_grad(left, w, d, None, dw, None, None, scratch)
        outs.append(dw)
    assert torch.equal(*outs)
    csgs.csgs_linear_grad(near, w, d, a, None, None, None, scratch)      # written far apart
    da = torch.zeros(M, K, dtype=B, device=dev)
    csgs.csgs_linear_grad(near, w, d, da, None, None, None, scratch)
    assert torch.equal(a, da)


def test_other_stream_and_replayed_graphs_that_share_scratch(env):
    csgs, dev = env
    side = torch.cuda.Stream()
    mk = Maker(dev, 7)
    M, K, N = 300, 120, 200
    x, wg, wu, w = mk.matrix(M, K, B), mk.matrix(K, N, B, 0.1), mk.matrix(K, N, B, 0.1), mk.matrix(N, K, B, 0.1)
    bg, bu, b = mk.vector(N), mk.vector(N), mk.vector(K)
    dy = mk.matrix(M, K, F)
    count = torch.tensor([M], dtype=torch.int32, device=dev)
    nbytes = max(csgs.csgs_gated_grad_scratch_bytes(M, K, N, csgs.BF16), csgs.csgs_linear_grad_scratch_bytes(M, N, K, csgs.BF16))
    scratch = torch.empty(nbytes, dtype=torch.uint8, device=dev)

    def buffers():
        z = lambda *s, t=B: torch.zeros(*s, dtype=t, device=dev)
        return dict(h=z(M, N), y=z(M, K, t=F), dh=z(M, N), dw=z(N, K), db=z(K, t=F), dr=z(M, K, t=F), dx=z(M, K), dwg=z(K, N), dwu=z(K, N), dbg=z(N, t=F), dbu=z(N, t=F))

    def half(o, k, stream=None):
        if k == 0:
            csgs.csgs_gated(x, wg, wu, o["h"], bg=bg, bu=bu, M_dev=count, stream=stream)
            csgs.csgs_linear(o["h"], w, o["y"], bias=b, r=dy, M_dev=count, stream=stream)
            csgs.csgs_linear_grad(o["h"], w, dy, o["dh"], o["dw"], o["db"], o["dr"], scratch, bias=b, M_dev=count, stream=stream)
        else:
            csgs.csgs_gated_grad(x, wg, wu, o["dh"], o["dx"], o["dwg"], o["dwu"], o["dbg"], o["dbu"], scratch, bg=bg, bu=bu, M_dev=count, stream=stream)
    got, want = buffers(), buffers()
    torch.cuda.synchronize()
    for k in range(2):
        half(got, k, side)
    side.synchronize()
    graphs = []
    for k in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            half(got, k, side)
        graphs.append(g)
    for i in range(5):
        x.mul_(-0.9)
        count.fill_(M - 31 * i)
        for t in list(got.values()) + list(want.values()):
            t.zero_()
        for k in range(2):
            half(want, k)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for name in got:
            assert torch.equal(got[name], want[name]), (i, name)
        assert float(want["dwg"].float().abs().sum()) > 0


@pytest.mark.parametrize("tb", [F, B], ids=["f32", "bf16"])
def test_matrices_in_the_columns_of_one_buffer(env, tb):
    """Inputs and outputs side by side in each row of one buffer, as in buffers of their own."""
    csgs, dev = env
    M, K, N = 300, 72, 40
    mk = Maker(dev, 9)
    a, dy, w, w2, b = mk.matrix(M, K, tb), mk.matrix(M, N, tb), mk.matrix(K, N, tb, 0.1), mk.matrix(K, N, tb, 0.1), mk.vector(N)
    scratch = torch.empty(csgs.csgs_gated_grad_scratch_bytes(M, K, N, elem(csgs, tb)), dtype=torch.uint8, device=dev)

    def run(cut, both):
        x, d, y, h, dx = cut
        x.copy_(a)
        d.copy_(dy)
        dwg, dwu = both
        csgs.csgs_linear(x, w, y, bias=b, r=d, act=csgs.ACT_SILU)
        csgs.csgs_gated(x, w, w2, h)
        csgs.csgs_gated_grad(x, w, w2, d, dx, dwg, dwu, None, None, scratch)
        return [t.clone() for t in (y, h, dx, dwg, dwu)]
    widths = [K, N, N, N, K]
    one = torch.full((M, sum(widths) + 3), math.nan, dtype=tb, device=dev)
    weights = torch.full((K, 2 * N), math.nan, dtype=tb, device=dev)
    got = run(one[:, 1:-2].split(widths, 1), weights.split(N, 1))
    want = run([torch.full((M, c), math.nan, dtype=tb, device=dev) for c in widths], [torch.zeros(K, N, dtype=tb, device=dev) for _ in range(2)])
    for g, t in zip(got, want):
        assert torch.equal(g, t)
    assert bool(one[:, 0].isnan().all()) and bool(one[:, -2:].isnan().all())
