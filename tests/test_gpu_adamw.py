"""A step of AdamW over many tensors, states in 32 and in 8 bits, against 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import plain_training as plain

HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def env():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2101_07706_amd import csgs
    csgs.lib()
    return csgs, torch.device("cuda:0")


def f32(x):
    return float(torch.tensor(x, dtype=torch.float32))


class Param:
    """A parameter on the device, and the same in 64 bits on the CPU."""

    def __init__(self, csgs, dev, gen, rows, cols, bits=32, p_type=torch.float32, g_type=torch.float32, gap=0, copy=False, ids=None, n_dev=None, wd=0.0,
                 lr_scale=1.0, std=0.1):
        self.csgs, self.bits, self.wd, self.lr_scale, self.ids, self.n_dev = csgs, bits, wd, lr_scale, ids, n_dev
        n = rows if ids is None else len(ids)

        def matrix(r, c, dtype, std):
            x = torch.full((r, c + gap), math.nan, dtype=dtype, device=dev)[:, :c]
            x.copy_(torch.randn(r, c, generator=gen) * std)
            return x
        self.p, self.g = matrix(rows, cols, p_type, 1.0), matrix(n, cols, g_type, std)
        self.copy = torch.full((rows, cols + gap), math.nan, dtype=torch.bfloat16, device=dev)[:, :cols] if copy else None
        m0 = torch.randn(rows, cols, generator=gen) * std / 4
        v0 = m0 * m0 * torch.exp(torch.randn(rows, cols, generator=gen)) + 1e-7
        if bits == 32:
            self.state = {"m": m0.to(dev), "v": v0.to(dev)}
        else:
            self.state = {}
            for k, x, second in (("m", m0, False), ("v", v0, True)):
                code, exps = plain.encode(x, second)
                self.state[k], self.state[k + "_exp"] = code.to(dev), exps.to(dev)
        self.ids_dev = None if ids is None else torch.tensor(ids, dtype=torch.int32, device=dev)
        self.n_dev_t = None if n_dev is None else torch.tensor([n_dev], dtype=torch.int32, device=dev)

    def entry(self):
        return self.csgs.adamw_entry(self.p, self.g, **self.state, copy=self.copy, ids=self.ids_dev, n_dev=self.n_dev_t, weight_decay=self.wd, lr_scale=self.lr_scale)

    def snapshot(self):
        s = {k: x.cpu() for k, x in self.state.items()}
        s["p"], s["g"] = self.p.cpu(), self.g.cpu()
        return s

    def live(self):
        n = self.g.shape[0]
        return n if self.n_dev is None else min(max(self.n_dev, 0), n)

    def rows(self):
        """(rows of p that a step changes, rows of g they belong to)."""
        n, rows = self.live(), self.p.shape[0]
        if self.ids is None:
            return list(range(n)), list(range(n))
        keep = [j for j in range(n) if 0 <= self.ids[j] < rows and (j == 0 or self.ids[j] > self.ids[j - 1])]
        return [self.ids[j] for j in keep], keep

    def check(self, before, t, lr, beta1, beta2, eps, c=1.0):
        rows, at = self.rows()
        old = {k: before[k][rows] for k in before if k != "g"}
        m, v = (old["m"].double(), old["v"].double()) if self.bits == 32 else (plain.decode(old["m"], old["m_exp"], False), plain.decode(old["v"], old["v_exp"], True))
        lr = f32(f32(lr) * f32(self.lr_scale))
        wp, wm, wv, change = plain.adamw(old["p"], before["g"][at], m, v, t, lr, beta1, beta2, f32(eps), f32(self.wd), c)
        got = self.snapshot()
        # double until the one rounding to float (double's own roundings: 2^-50 of it)
        if self.bits == 32:
            for k, want in (("m", wm), ("v", wv)):
                assert bool(((got[k][rows].double() - want).abs() <= (2.0 ** -24 + 2.0 ** -45) * want.abs() + 2.0 ** -149).all()), k
        else:
            for k, want, second in (("m", wm, False), ("v", wv, True)):
                code, exps = plain.encode(want.float(), second)
                assert torch.equal(got[k + "_exp"][rows], exps), k
                assert torch.equal(got[k][rows], code), k
        # the change: m and v as floats (1 and 1/2), 1 / (1 - beta1^t) and its product, the root, 1 / root and its product, eps and its sum, the quotient; the
        # decay's product, the sum, lr's products (2) and the last subtraction's operand: 14 roundings of it; one of p to its type (and one of the float before)
        half = HALF_ULP[self.p.dtype]
        tol = half * wp.abs() * 1.01 + 2.0 ** -24 * (wp.abs() + 14 * change) + 1e-38
        assert bool(((got["p"][rows].double() - wp).abs() <= tol).all()), "p"
        if self.copy is not None:
            tol = 2.0 ** -8 * wp.abs() * 1.01 + 2.0 ** -24 * (wp.abs() + 14 * change) + 1e-38
            assert bool(((self.copy.cpu()[rows].double() - wp).abs() <= tol).all()), "copy"
        rest = sorted(set(range(self.p.shape[0])) - set(rows))
        for k in got:
            if k != "g":
                assert torch.equal(got[k][rest].view(torch.uint8), before[k][rest].view(torch.uint8)), f"{k}: rows that no gradient names"
        if self.copy is not None:
            assert bool(self.copy.cpu()[rest].isnan().all())


SHAPES = [(1, 1), (1, 5), (3, 1), (2, 4), (17, 3), (5, 64), (7, 100), (4, 255), (3, 256), (3, 257), (2, 1000), (33, 47), (1, 5000), (64, 512), (300, 20)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("types", ["ff", "fb", "bf", "bb"])
def test_step_over_shapes(env, bits, types):
    csgs, dev = env
    gen = torch.Generator().manual_seed(bits)
    kind = {"f": torch.float32, "b": torch.bfloat16}
    params = [Param(csgs, dev, gen, r, c, bits, kind[types[0]], kind[types[1]], gap=(i % 3) * 3, copy=i % 2 == 0, wd=0.01 * (i % 3), lr_scale=[1.0, 0.5][i % 2])
              for i, (r, c) in enumerate(SHAPES)]
    l = csgs.make_adamw_list([p.entry() for p in params])
    step = torch.zeros(1, dtype=torch.int32, device=dev)
    for t in range(1, 4):
        before = [p.snapshot() for p in params]
        csgs.csgs_adamw(l, 1e-2, step)
        assert int(step) == t
        for p, b in zip(params, before):
            p.check(b, t, 1e-2, 0.9, 0.999, 1e-8)


@pytest.mark.parametrize("bits", [32, 8])
def test_hyperparameters_and_late_steps(env, bits):
    csgs, dev = env
    for beta1, beta2, eps, t0 in ((0.0, 0.0, 1e-3, 0), (0.0, 0.99, 0.0, 5), (0.95, 0.0, 1e-8, 1), (0.9, 0.9999, 1e-8, 99_999), (0.9, 0.999, 1e-8, 2_000_000_000)):
        p = Param(csgs, dev, torch.Generator().manual_seed(1), 9, 70, bits, wd=0.1)
        l = csgs.make_adamw_list([p.entry()])
        step = torch.full((1,), t0, dtype=torch.int32, device=dev)
        half = torch.full((1,), 0.5, device=dev)
        before = p.snapshot()
        csgs.csgs_adamw(l, 2e-2, step, beta1=beta1, beta2=beta2, eps=eps, lr_dev=half)
        p.check(before, t0 + 1, 1e-2, beta1, beta2, eps)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("cols", [1, 33, 100, 300])
def test_rows_of_a_table(env, bits, cols):
    csgs, dev = env
    gen = torch.Generator().manual_seed(cols)
    cases = [dict(ids=[0]), dict(ids=[499]), dict(ids=sorted(torch.randperm(500, generator=gen)[:200].tolist())), dict(ids=[3, 9, 10, 40], n_dev=2), dict(ids=[3, 9], n_dev=0),
             dict(ids=[3, 9], n_dev=-4), dict(ids=[3, 9], n_dev=77), dict(ids=[-1, 4, 500, 2_000_000_000]), dict(ids=None, n_dev=123)]
    for k, case in enumerate(cases):
        p = Param(csgs, dev, gen, 500, cols, bits, gap=k % 2, **case)
        other = Param(csgs, dev, gen, 7, 20, bits)
        status = torch.zeros(1, dtype=torch.int32, device=dev)
        step = torch.zeros(1, dtype=torch.int32, device=dev)
        l = csgs.make_adamw_list([other.entry(), p.entry()])
        before = p.snapshot(), other.snapshot()
        csgs.csgs_adamw(l, 1e-2, step, status=status)
        p.check(before[0], 1, 1e-2, 0.9, 0.999, 1e-8)
        other.check(before[1], 1, 1e-2, 0.9, 0.999, 1e-8)
        assert int(status) == 0 and int(step) == 1


def test_ids_that_do_not_ascend_are_left_out(env):
    csgs, dev = env
    p = Param(csgs, dev, torch.Generator().manual_seed(0), 20, 40, ids=[2, 5, 5, 7, 6, 9])
    status, step = (torch.zeros(1, dtype=torch.int32, device=dev) for _ in range(2))
    before = p.snapshot()
    csgs.csgs_adamw(csgs.make_adamw_list([p.entry()]), 1e-2, step, status=status)
    assert int(status) == csgs.ST_BAD_NODE_ID
    p.check(before, 1, 1e-2, 0.9, 0.999, 1e-8)


@pytest.mark.parametrize("bits", [32, 8])
def test_an_id_named_again_behind_ids_that_are_passed_over(env, bits):
    """The first row of g with an id is taken, whatever lies between it and the next one."""
    csgs, dev = env
    g = torch.randn(8, 40, generator=torch.Generator().manual_seed(1)).to(dev)
    got = []
    for ids, rows in (([5, -1, 5, 20, 7, 7, -1, 2_000_000_000], list(range(8))), ([5, 7], [0, 4])):
        p, step, status = torch.ones(20, 40, device=dev), *(torch.zeros(1, dtype=torch.int32, device=dev) for _ in range(2))
        state = csgs.adamw_states(p, bits)
        l = csgs.make_adamw_list([csgs.adamw_entry(p, g[rows], **state, ids=torch.tensor(ids, dtype=torch.int32, device=dev))])
        csgs.csgs_adamw(l, 1e-2, step, status=status)
        got.append((p, *state.values()))
        assert int(status) == (csgs.ST_BAD_NODE_ID if len(ids) == 8 else 0) and int(step) == 1
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert int((got[0][0] != 1).any(1).sum()) == 2


@pytest.mark.parametrize("kind", ["l2", "l1", "max"])
@pytest.mark.parametrize("bits", [32, 8])
def test_clipped_by_the_norm_of_the_gradients(env, kind, bits):
    csgs, dev = env
    gen = torch.Generator().manual_seed(2)
    params = [Param(csgs, dev, gen, 30, 70, bits, gap=1), Param(csgs, dev, gen, 400, 24, bits, ids=list(range(5, 105)), n_dev=60), Param(csgs, dev, gen, 1, 9, bits)]
    kinds = {"l2": csgs.GRAD_L2, "l1": csgs.GRAD_L1, "max": csgs.GRAD_MAX}
    live = [p.g.cpu()[:p.live()].double() for p in params]
    total = {"l2": lambda: math.sqrt(math.fsum(float((g * g).sum()) for g in live)), "l1": lambda: math.fsum(float(g.abs().sum()) for g in live),
             "max": lambda: max(float(g.abs().max()) for g in live)}[kind]()
    l = csgs.make_adamw_list([p.entry() for p in params])
    clip = csgs.make_grad_list([p.g for p in params], [None] * 3, [p.n_dev_t for p in params])
    norm, step, status = torch.zeros(1, device=dev), *(torch.zeros(1, dtype=torch.int32, device=dev) for _ in range(2))
    t64 = torch.zeros(1, dtype=torch.float64, device=dev)
    t = 0
    for max_norm in (f32(0.3 * total), f32(2 * total), math.inf):
        for by_total in (False, True):
            t += 1
            before = [p.snapshot() for p in params]
            if by_total:
                csgs.csgs_grad_norm(clip, kinds[kind], t64)
                csgs.csgs_adamw(l, 1e-2, step, total=t64, kind=kinds[kind], max_norm=max_norm, norm=norm, status=status)
            else:
                csgs.csgs_adamw(l, 1e-2, step, clip=clip, kind=kinds[kind], max_norm=max_norm, norm=norm, status=status)
            assert abs(float(norm) - total) <= 2.0 ** -23 * total and int(status) == 0 and int(step) == t
            for p, b in zip(params, before):
                p.check(b, t, 1e-2, 0.9, 0.999, 1e-8, min(1.0, max_norm / (total + 1e-6)))


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_gradients_that_are_not_finite_change_nothing(env, bad):
    csgs, dev = env
    gen = torch.Generator().manual_seed(3)
    params = [Param(csgs, dev, gen, 30, 70), Param(csgs, dev, gen, 10, 300, 8)]
    l = csgs.make_adamw_list([p.entry() for p in params])
    clip = csgs.make_grad_list([p.g for p in params], [None] * 2)
    step, status = (torch.zeros(1, dtype=torch.int32, device=dev) for _ in range(2))
    norm = torch.zeros(1, device=dev)
    good = float(params[1].g[2, 3])
    params[1].g[2, 3] = bad
    before = [p.snapshot() for p in params]
    csgs.csgs_adamw(l, 1e-2, step, clip=clip, max_norm=1.0, norm=norm, status=status)
    assert int(step) == 0 and int(status) == csgs.ST_NONFINITE_GRAD and not math.isfinite(float(norm))
    for p, b in zip(params, before):
        after = p.snapshot()
        assert all(torch.equal(after[k], b[k]) for k in after if k != "g")
    params[1].g[2, 3] = good
    status.zero_()
    before = [p.snapshot() for p in params]
    csgs.csgs_adamw(l, 1e-2, step, clip=clip, max_norm=1e9, norm=norm, status=status)
    assert int(step) == 1 and int(status) == 0
    for p, b in zip(params, before):
        p.check(b, 1, 1e-2, 0.9, 0.999, 1e-8)


def test_without_clipping_what_is_not_finite_stays_in_its_entry_or_block(env):
    csgs, dev = env
    gen = torch.Generator().manual_seed(4)
    a, b = Param(csgs, dev, gen, 4, 300), Param(csgs, dev, gen, 4, 300, 8)
    l = csgs.make_adamw_list([a.entry(), b.entry()])
    step = torch.zeros(1, dtype=torch.int32, device=dev)
    for p in (a, b):
        p.g[1, 270] = math.nan
    csgs.csgs_adamw(l, 1e-2, step)
    for p in (a, b):
        bad = torch.zeros(4, 300, dtype=torch.bool)
        bad[1, 270] = True
        assert torch.equal(p.p.cpu().isnan(), bad)
    assert torch.equal(a.state["m"].cpu().isnan(), bad)
    assert b.state["m_exp"].cpu().tolist()[1][1] == 255 and b.state["v_exp"].cpu().tolist()[1][1] == 255
    out = torch.zeros(4, 300, device=dev)
    bad[1, 256:] = True
    for k, which in (("m", csgs.STATE_FIRST), ("v", csgs.STATE_SECOND)):
        csgs.csgs_state_read(b.state[k], b.state[k + "_exp"], which, out)
        assert torch.equal(out.cpu().isnan(), bad)


VALUES = {
    "ordinary": lambda r, c, g: torch.randn(r, c, generator=g),
    "wide": lambda r, c, g: torch.randn(r, c, generator=g) * torch.exp(8 * torch.randn(r, c, generator=g)),
    "zeros": lambda r, c, g: torch.randn(r, c, generator=g) * (torch.rand(r, c, generator=g) < 0.02),
    "tiny": lambda r, c, g: torch.randn(r, c, generator=g) * 1e-37,
    "huge": lambda r, c, g: torch.randn(r, c, generator=g).clamp(-3, 3) * 1e38,
    "ties": lambda r, c, g: (torch.randint(0, 65, (r, c), generator=g).float() / 32 + 1) * 2.0 ** torch.randint(-20, 5, (r, c), generator=g).float(),
}


@pytest.mark.parametrize("name", list(VALUES))
@pytest.mark.parametrize("shape", [(1, 1), (3, 5), (7, 100), (5, 256), (4, 513), (200, 64)])
def test_values_as_codes_and_back(env, name, shape):
    csgs, dev = env
    rows, cols = shape
    x = VALUES[name](rows, cols, torch.Generator().manual_seed(rows + cols))
    nb = (cols + 255) // 256
    for which, second in ((csgs.STATE_FIRST, False), (csgs.STATE_SECOND, True)):
        y = x.abs() if second else x
        gapped = torch.full((rows, cols + 3), math.nan, device=dev)
        gapped[:, :cols] = y.to(dev)
        codes, exps = torch.full((rows, cols), 77, dtype=torch.uint8, device=dev), torch.full((rows, nb), 77, dtype=torch.uint8, device=dev)
        csgs.csgs_state_write(gapped[:, :cols], which, codes, exps)
        want, want_exps = plain.encode(y, second)
        assert torch.equal(exps.cpu(), want_exps) and torch.equal(codes.cpu(), want)
        back = torch.full((rows, cols + 2), math.nan, device=dev)
        csgs.csgs_state_read(codes, exps, which, back[:, :cols])
        v = plain.decode(want, want_exps, second)
        # (a value below the smallest float number of full precision is rounded to one of those there are)
        assert bool(((back[:, :cols].cpu().double() - v).abs() <= torch.where(v.abs() < 2.0 ** -126, 2.0 ** -149, 0.0)).all())
        assert bool(back[:, cols:].isnan().all())
        # within half a step of a value's own octave; the first state's smallest steps are those of 2^-9 of its power of two, the second's zero stays zero
        top = torch.repeat_interleave(torch.ldexp(torch.ones((), dtype=torch.float64), exps.cpu().double() - 127), 256, dim=1)[:, :cols]
        # (blocks below 2^-126 are zero: all of a value is lost; values on a border of the 8-bit second state's lower end are raised to it)
        bound = 2.0 ** -4 * y.double().abs() + (top * 2.0 ** -30 if second else top * 2.0 ** -17) + 2.0 ** -126
        assert bool(((v - y.double()).abs() <= bound).all())
        if second:
            alive = (y > 0) & (top > 0) & (torch.repeat_interleave(exps.cpu(), 256, dim=1)[:, :cols] > 0)
            assert bool((v[alive] > 0).all())


def test_negative_second_states_are_zero_and_nan_spreads_over_its_block(env):
    csgs, dev = env
    x = torch.tensor([[1.0, -2.0, -0.0, 0.25] + [0.0] * 300], device=dev)
    codes, exps = torch.zeros(1, 304, dtype=torch.uint8, device=dev), torch.zeros(1, 2, dtype=torch.uint8, device=dev)
    csgs.csgs_state_write(x, csgs.STATE_SECOND, codes, exps)
    back = torch.zeros(1, 304, device=dev)
    csgs.csgs_state_read(codes, exps, csgs.STATE_SECOND, back)
    assert back[0, :4].tolist() == [1.0, 0.0, 0.0, 0.25] and float(back.sum()) == 1.25
    x[0, 300] = math.nan
    csgs.csgs_state_write(x, csgs.STATE_SECOND, codes, exps)
    csgs.csgs_state_read(codes, exps, csgs.STATE_SECOND, back)
    assert back[0, :256].sum() == 1.25 and bool(back[0, 256:].isnan().all())


def test_new_states_and_repeatability(env):
    csgs, dev = env
    gen = torch.Generator().manual_seed(7)
    p0, g = torch.randn(50, 300, generator=gen), torch.randn(50, 300, generator=gen)
    for bits in (32, 8):
        runs = []
        for _ in range(2):
            p = p0.to(dev)
            state = csgs.adamw_states(p, bits)
            l = csgs.make_adamw_list([csgs.adamw_entry(p, g.to(dev), **state, weight_decay=0.1)])
            step = torch.zeros(1, dtype=torch.int32, device=dev)
            for _ in range(5):
                csgs.csgs_adamw(l, 1e-2, step)
            runs.append([p] + [state[k] for k in sorted(state)])
        assert all(torch.equal(a, b) for a, b in zip(*runs))
        # With a constant gradient a step is lr times its sign.  States in 8 bits: an entry whose m keeps its three bits of mantissa (at least 2^-13 of its
        # block's power of two: at least 2^-12 of the largest gradient) loses up to 2^-4 of m and of v at each of the t - 1 roundings before step t, which is then off by
        # up to (1 + 2^-4)^(t - 1) / (1 - 2^-4)^((t - 1) / 2) - 1 of itself: 0.10, 0.21, 0.33, 0.46 for t = 2 to 5, together 1.10 lr.  (5e-4: eps, the decay of the change itself.)
        drift = p0.double() * (1 - f32(1e-2) * f32(0.1)) ** 5 - 5 * 1e-2 * torch.sign(g.double())
        off = (p.cpu().double() - drift).abs()
        top = torch.cat([g[:, :256].abs().amax(1, keepdim=True).expand(50, 256), g[:, 256:].abs().amax(1, keepdim=True).expand(50, 44)], 1)
        assert float(off[g.abs() >= 2.0 ** -12 * top].max()) < (5e-4 if bits == 32 else 1.1e-2 + 5e-4)


def test_other_stream_and_replayed_graph(env):
    csgs, dev = env
    gen = torch.Generator().manual_seed(8)
    side = torch.cuda.Stream()
    params = [Param(csgs, dev, gen, 40, 70), Param(csgs, dev, gen, 90, 300, 8, ids=list(range(3, 60))), Param(csgs, dev, gen, 1, 33, g_type=torch.bfloat16)]
    lr = torch.full((1,), 1.0, device=dev)
    step, norm = torch.zeros(1, dtype=torch.int32, device=dev), torch.zeros(1, device=dev)
    side.wait_stream(torch.cuda.current_stream())
    l = csgs.make_adamw_list([p.entry() for p in params], stream=side)
    clip = csgs.make_grad_list([p.g for p in params], [None] * 3, stream=side)
    side.synchronize()
    before = [p.snapshot() for p in params]
    csgs.csgs_adamw(l, 1e-2, step, clip=clip, max_norm=0.5, lr_dev=lr, norm=norm, stream=side)
    side.synchronize()
    total = float(norm)
    total64 = math.sqrt(math.fsum(float((p.g.double() ** 2).sum()) for p in params))
    assert abs(total - total64) <= 2.0 ** -23 * total64
    for p, b in zip(params, before):
        p.check(b, 1, 1e-2, 0.9, 0.999, 1e-8, 0.5 / (total64 + 1e-6))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        csgs.csgs_adamw(l, 1e-2, step, clip=clip, max_norm=0.5, lr_dev=lr, norm=norm, stream=side)
    for t in range(2, 7):
        torch.cuda.synchronize()
        for p in params:
            p.g.mul_(1.25)           # eager work between the replays
        lr.fill_(1.0 / t)
        total64 = math.sqrt(math.fsum(float((p.g.double() ** 2).sum()) for p in params))
        before = [p.snapshot() for p in params]
        graph.replay()
        torch.cuda.synchronize()
        assert int(step) == t
        for p, b in zip(params, before):
            p.check(b, t, f32(f32(1e-2) * f32(1.0 / t)), 0.9, 0.999, 1e-8, 0.5 / (total64 + 1e-6))


def test_a_long_table(env):
    """Entries past 2^31 of a table with 8-bit states, touched at its ends."""
    csgs, dev = env
    rows, cols = 17_000_000, 128
    p = torch.zeros(rows, cols, dtype=torch.bfloat16, device=dev)
    state = csgs.adamw_states(p, 8)
    ids = [0, 1, 16_777_215, 16_777_216, 16_777_217, rows - 1]
    g = torch.randn(len(ids), cols, generator=torch.Generator().manual_seed(0)).to(dev)
    step = torch.zeros(1, dtype=torch.int32, device=dev)
    l = csgs.make_adamw_list([csgs.adamw_entry(p, g, **state, ids=torch.tensor(ids, dtype=torch.int32, device=dev))])
    csgs.csgs_adamw(l, 0.5, step)
    at = torch.tensor(ids, device=dev)
    want = -0.5 * torch.sign(g) * (g.abs() / (g.abs() + 1e-8))
    assert bool(((p[at].float() - want).abs() <= 2.0 ** -8 * 0.5 + 1e-5).all())
    assert int((p != 0).any(1).sum()) == len(ids) and int((state["v_exp"] != 0).sum()) == len(ids)


def test_two_lists_side_by_side(env):
    csgs, dev = env
    gen = torch.Generator().manual_seed(9)
    streams = [torch.cuda.Stream() for _ in range(2)]
    params = [[Param(csgs, dev, gen, 300, 200, bits) for _ in range(3)] for bits in (32, 8)]
    steps = [torch.zeros(1, dtype=torch.int32, device=dev) for _ in range(2)]
    before = [[p.snapshot() for p in ps] for ps in params]
    torch.cuda.synchronize()
    for ps, st, step in zip(params, streams, steps):
        l = csgs.make_adamw_list([p.entry() for p in ps], stream=st)
        csgs.csgs_adamw(l, 1e-2, step, stream=st)
        del l                                    # dropped while the call is enqueued
    torch.cuda.synchronize()
    for ps, bs in zip(params, before):
        for p, b in zip(ps, bs):
            p.check(b, 1, 1e-2, 0.9, 0.999, 1e-8)


def long_runs(gen, run, cols, dev):
    """A table whose gradient's ids are passed over in runs of `run` and more, in front of and between rows that count, some of them named again behind a run."""
    ids, keep = [-1] * run, []
    for k, (id, again, gap) in enumerate([(3, False, run), (3, True, 9), (7, False, 8), (9, False, 1), (9, True, run + 1), (9, True, 0), (40, False, 300), (41, False, 255), (41, True, 256),
                                          (60, False, run // 2), (50, True, 0), (400, False, run // 3)]):
        if not again:
            keep.append(len(ids))
        ids += [id] + [[-1, 500, 2_000_000_000][k % 3]] * gap
    p = torch.randn(500, cols, generator=gen).to(dev)
    g = torch.randn(len(ids), cols, generator=gen).to(dev)
    return p, g, torch.tensor(ids, dtype=torch.int32), keep


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("cols", [1, 4, 5, 64, 300])
@pytest.mark.parametrize("run", [7, 64, 70, 300, 3000])
def test_ids_behind_long_runs_that_are_passed_over(env, bits, cols, run):
    """As the ids that count alone: whatever lies between them, each is taken once, and one that is not above the last of them is left out."""
    csgs, dev = env
    p, g, ids, keep = long_runs(torch.Generator().manual_seed(run), run, cols, dev)
    got = []
    for rows in (torch.arange(len(ids)), torch.tensor(keep)):
        q, step, status = p.clone(), *(torch.zeros(1, dtype=torch.int32, device=dev) for _ in range(2))
        state = csgs.adamw_states(q, bits)
        csgs.csgs_adamw(csgs.make_adamw_list([csgs.adamw_entry(q, g[rows.to(dev)].contiguous(), **state, ids=ids[rows].to(dev))]), 1e-2, step, status=status)
        got.append((q, *state.values()))
        assert int(status) == (csgs.ST_BAD_NODE_ID if len(rows) == len(ids) else 0) and int(step) == 1
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert int((got[0][0] != p).any(1).sum()) == len(keep)


def test_a_long_run_of_ids_costs_a_look_at_them(env):
    """Rows behind a million ids that are passed over: the device looks at hundreds of them at a time (one by one they took 116 ms)."""
    csgs, dev = env
    run, rows, cols = 1_000_000, 300, 100
    p, g = torch.zeros(500, cols, device=dev), torch.ones(1, cols, device=dev).expand(run + rows, cols).contiguous()
    ids = torch.cat([torch.full((run,), -1, dtype=torch.int32), torch.arange(rows, dtype=torch.int32)]).to(dev)
    step = torch.zeros(1, dtype=torch.int32, device=dev)
    l = csgs.make_adamw_list([csgs.adamw_entry(p, g, **csgs.adamw_states(p), ids=ids)])
    times = []
    for _ in range(3):
        e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        e[0].record()
        csgs.csgs_adamw(l, 1e-2, step)
        e[1].record()
        torch.cuda.synchronize()
        times.append(e[0].elapsed_time(e[1]))
    assert int((p != 0).any(1).sum()) == rows
    assert min(times) < 50.0, times
