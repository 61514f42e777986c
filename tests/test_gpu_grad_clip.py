"""The global gradient norm over many tensors and clipping by it, against 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

KINDS = ["l2", "l1", "max"]


@pytest.fixture(scope="module")
def env():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2101_07706_amd import csgs
    csgs.lib()
    return csgs, torch.device("cuda:0")


def kind_of(csgs, kind):
    return {"l2": csgs.GRAD_L2, "l1": csgs.GRAD_L1, "max": csgs.GRAD_MAX}[kind]


def total_of(tensors, kind):
    if kind == "max":
        return max(float(t.double().abs().max()) if t.numel() else 0.0 for t in tensors)
    if kind == "l1":
        return math.fsum(float(t.double().abs().sum()) for t in tensors)
    return math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in tensors))


def make(shapes, dev, seed=0, std=0.1):
    g = torch.Generator().manual_seed(seed)
    out = []
    for i, s in enumerate(shapes):
        dtype = torch.bfloat16 if i % 3 == 2 else torch.float32
        if len(s) == 2 and i % 4 == 1:      # rows with a gap
            out.append(torch.full((s[0], s[1] + 3), float("nan"), dtype=dtype, device=dev)[:, :s[1]])
            out[-1].copy_(torch.randn(*s, generator=g) * std)
        else:
            out.append((torch.randn(*s, generator=g) * std).to(dtype).to(dev))
    return out


def check_clipped(grads, outs, total, max_norm):
    coef = min(1.0, max_norm / (total + 1e-6))
    for k, (g, o) in enumerate(zip(grads, outs)):
        want = g.double() * coef
        # the coefficient's and the product's rounding, and one to the type
        tol = (2.0 ** -23 + (2.0 ** -8 if g.dtype == torch.bfloat16 else 0.0)) * want.abs() * 1.01 + 1e-38
        assert bool(((o.double() - want).abs() <= tol).all()), f"tensor {k}"


LISTS = {
    "one": [(1,)],
    "few": [(7,), (100, 256), (256,), (256, 256), (256, 47), (47,)],
    "gaps": [(5, 9), (33, 100), (1000, 31), (3, 8191), (1, 5), (17, 1)],
    "many": [((i * 37) % 200 + 1,) if i % 2 else ((i * 13) % 50 + 1, (i * 7) % 90 + 1) for i in range(300)],
    "large": [(1000, 1000), (8192,), (8193,), (3, 20000), (70000, 65)],
}


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", list(LISTS))
def test_norm_and_clipping(env, name, kind):
    csgs, dev = env
    grads = make(LISTS[name], dev)
    total = total_of(grads, kind)
    outs = [torch.full_like(g, float("nan")) for g in grads]
    l = csgs.make_grad_list(grads, outs)
    norm, status = torch.zeros(1, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)
    for max_norm in (0.5 * total, 2.0 * total, float("inf")):
        norm.fill_(-1)
        csgs.csgs_grad_clip(l, kind_of(csgs, kind), max_norm, norm, status)
        assert abs(float(norm) - total) <= 2.0 ** -23 * total and int(status) == 0     # sums in double, one rounding
        check_clipped(grads, outs, total, float(torch.tensor(max_norm, dtype=torch.float32)))
        if max_norm > total:
            assert all(torch.equal(g, o) for g, o in zip(grads, outs))
    first = [o.clone() for o in outs]
    csgs.csgs_grad_clip(l, kind_of(csgs, kind), max_norm, norm, status)
    assert all(torch.equal(a, b) for a, b in zip(first, outs)), "two calls differ"
    # the halves, with totals of two lists added between them as between two GPUs
    t = torch.zeros(1, dtype=torch.float64, device=dev)
    csgs.csgs_grad_norm(l, kind_of(csgs, kind), t)
    raw = total * total if kind == "l2" else total
    assert abs(float(t) - raw) <= 1e-12 * raw
    if kind != "max":
        t.mul_(2.0)
    csgs.csgs_grad_scale(l, kind_of(csgs, kind), t, 0.1 * total, norm, status)
    both = total * {"l2": math.sqrt(2.0), "l1": 2.0, "max": 1.0}[kind]
    assert abs(float(norm) - both) <= 2.0 ** -23 * both
    check_clipped(grads, outs, both, float(torch.tensor(0.1 * total, dtype=torch.float32)))


def test_in_place_and_norm_only_tensors(env):
    csgs, dev = env
    grads = make(LISTS["few"], dev, seed=3)
    before = [g.clone() for g in grads]
    total = total_of(grads, "l2")
    l = csgs.make_grad_list(grads)                       # in place
    norm = torch.zeros(1, device=dev)
    csgs.csgs_grad_clip(l, csgs.GRAD_L2, 10 * total, norm)
    assert all(torch.equal(a, b) for a, b in zip(before, grads))
    csgs.csgs_grad_clip(l, csgs.GRAD_L2, 0.25 * total, norm)
    check_clipped(before, grads, total, float(torch.tensor(0.25 * total, dtype=torch.float32)))
    # in the norm alone
    grads = make(LISTS["few"], dev, seed=4)
    before = [g.clone() for g in grads]
    total = total_of(grads, "l2")
    outs = [None if i % 2 else g for i, g in enumerate(grads)]
    csgs.csgs_grad_clip(csgs.make_grad_list(grads, outs), csgs.GRAD_L2, 0.5 * total, norm)
    assert abs(float(norm) - total) <= 2.0 ** -23 * total
    for i, (b, g) in enumerate(zip(before, grads)):
        assert torch.equal(b, g) == bool(i % 2)


@pytest.mark.parametrize("count", [0, 1, 60, 100, 1000, -4])
@pytest.mark.parametrize("gap", [0, 5])
def test_rows_up_to_a_device_count(env, count, gap):
    csgs, dev = env
    raw = torch.randn(100, 300 + gap, device=dev)
    g = raw[:, :300]
    n = min(max(count, 0), 100)
    g[n:] = float("nan")
    other = torch.randn(40, device=dev)
    out = torch.full((100, 300 + gap), -5.0, device=dev)[:, :300]
    n_dev = torch.tensor([count], dtype=torch.int32, device=dev)
    l = csgs.make_grad_list([other, g], [torch.empty_like(other), out], [None, n_dev])
    norm = torch.zeros(1, device=dev)
    csgs.csgs_grad_clip(l, csgs.GRAD_L2, 1.0, norm)
    total = total_of([other, g[:n]], "l2")
    assert abs(float(norm) - total) <= 2.0 ** -23 * total
    check_clipped([g[:n]], [out[:n]], total, 1.0)
    assert bool((out[n:] == -5.0).all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_values_that_are_not_finite(env, kind, bad):
    csgs, dev = env
    for where in (0, 4999, 2500):
        grads = [torch.ones(50, device=dev), torch.ones(5000, device=dev, dtype=torch.bfloat16)]
        grads[1][where] = bad
        norm, status = torch.zeros(1, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)
        csgs.csgs_grad_clip(csgs.make_grad_list(grads, [torch.empty_like(g) for g in grads]), kind_of(csgs, kind), 1.0, norm, status)
        assert int(status) == csgs.ST_NONFINITE_GRAD
        assert math.isnan(float(norm)) if bad != bad else float(norm) == math.inf


def test_large_values_do_not_overflow(env):
    csgs, dev = env
    g = torch.full((4000,), 3e38, device=dev)
    norm, t, status = torch.zeros(1, device=dev), torch.zeros(1, dtype=torch.float64, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)
    l = csgs.make_grad_list([g])
    csgs.csgs_grad_norm(l, csgs.GRAD_L2, t)
    assert abs(float(t) / (4000 * float(g[0]) ** 2) - 1) < 1e-12
    csgs.csgs_grad_clip(l, csgs.GRAD_L2, 1.0, norm, status)
    assert int(status) == 0 and abs(float(g.double().norm()) - 1.0) < 1e-6      # the norm itself is past a float's range, its double is not


def test_entries_past_32_bits(env):
    csgs, dev = env
    n = (1 << 32) + 4097
    g = torch.zeros(n, dtype=torch.bfloat16, device=dev)
    g[-1], g[0], g[1 << 31] = 2.0, 1.0, 2.0
    rows = torch.zeros((1 << 16) + 3, 1 << 16, dtype=torch.bfloat16, device=dev)[:, :5]
    rows[-1, 4] = 4.0
    norm = torch.zeros(1, device=dev)
    csgs.csgs_grad_clip(csgs.make_grad_list([g, rows]), csgs.GRAD_L2, 2.5, norm)
    assert float(norm) == 5.0
    assert float(g[-1]) == 1.0 and float(g[0]) == 0.5 and float(g[1 << 31]) == 1.0 and float(rows[-1, 4]) == 2.0


def test_on_another_stream_and_replayed(env):
    csgs, dev = env
    grads = make(LISTS["gaps"], dev)
    outs = [torch.empty_like(g) for g in grads]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    norm = torch.zeros(1, device=dev)
    l = csgs.make_grad_list(grads, outs, stream=side)
    csgs.csgs_grad_clip(l, csgs.GRAD_L2, 1.0, norm, stream=side)
    side.synchronize()
    total = total_of(grads, "l2")
    assert abs(float(norm) - total) <= 2.0 ** -23 * total
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        csgs.csgs_grad_clip(l, csgs.GRAD_L2, 1.0, norm)
    for k in range(3):
        for g in grads:
            g.normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        total = total_of(grads, "l2")
        assert abs(float(norm) - total) <= 2.0 ** -23 * total
        csgs.csgs_grad_clip(l, csgs.GRAD_L2, 1.0, norm)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs)), f"replay {k}"


def test_calls_on_a_recorded_plan(env):
    csgs, dev = env
    grads = make(LISTS["few"], dev)
    l = csgs.make_grad_list(grads)
    norm = torch.zeros(1, device=dev)
    with csgs.record() as plan:
        csgs.csgs_grad_clip(l, csgs.GRAD_MAX, 1e-3, norm)
    total = total_of(grads, "max")
    plan.run()
    assert float(norm) == total
    plan.run()
    assert abs(float(norm) - total * 1e-3 / (total + 1e-6)) <= 1e-7


@pytest.mark.parametrize("used_on", ["its own stream", "another"])
def test_a_list_dropped_while_its_calls_are_enqueued(env, used_on):
    """Made, used and dropped on side streams that are busy, while the current stream clears memory of the same size that was freed before and takes more of it
    after.  (Descriptions that such work clears describe nothing: outputs then keep their NaN.)"""
    csgs, dev = env
    grads = make(LISTS["gaps"], dev, seed=6)
    outs = [torch.full_like(g, float("nan")) for g in grads]
    norm, total = torch.full((1,), -1.0, device=dev), total_of(grads, "l2")
    long = [torch.empty(1 << 28, dtype=torch.float32, device=dev) for _ in range(3)]
    words = csgs.make_grad_list(grads, outs)._keep[0].numel()
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()

    def keep_busy(t):
        for _ in range(20):      # 1 GB each
            t.fill_(1.0)

    freed = [torch.empty(words, dtype=torch.int64, device=dev) for _ in range(32)]
    keep_busy(long[0])
    for t in freed:
        t.zero_()
    del freed, t
    with torch.cuda.stream(side):
        keep_busy(long[1])
    l = csgs.make_grad_list(grads, outs, stream=side)
    last = side
    if used_on == "another":
        last = other
        other.wait_stream(side)
        with torch.cuda.stream(other):
            keep_busy(long[2])
    csgs.csgs_grad_clip(l, csgs.GRAD_L2, 0.5 * total, norm, stream=last)
    del l
    taken = [torch.zeros(words, dtype=torch.int64, device=dev) for _ in range(32)]
    with torch.cuda.stream(side):
        taken += [torch.zeros(words, dtype=torch.int64, device=dev) for _ in range(32)]
    torch.cuda.synchronize()
    assert abs(float(norm) - total) <= 2.0 ** -23 * total
    check_clipped(grads, outs, total, float(torch.tensor(0.5 * total, dtype=torch.float32)))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_with_gaps_longer_than_a_tile(env, dtype, kind):
    """A tile of a tensor with gaps between its rows that lies in two of them, or in the middle of one."""
    csgs, dev = env
    grads, outs = [], []
    for rows, cols, gap in ((5, 20_000, 3), (3, 8193, 1), (2, 30_001, 8), (40, 8192, 5), (9, 4097, 7)):
        g = torch.full((rows, cols + gap), float("nan"), dtype=dtype, device=dev)[:, :cols]
        g.copy_(torch.randn(rows, cols, generator=torch.Generator().manual_seed(cols)) * 0.1)
        grads.append(g)
        outs.append(torch.full((rows, cols + gap + 1), -5.0, dtype=dtype, device=dev)[:, :cols])
    total = total_of(grads, kind)
    norm = torch.zeros(1, device=dev)
    csgs.csgs_grad_clip(csgs.make_grad_list(grads, outs), kind_of(csgs, kind), 0.5 * total, norm)
    assert abs(float(norm) - total) <= 2.0 ** -23 * total
    check_clipped(grads, outs, total, float(torch.tensor(0.5 * total, dtype=torch.float32)))
    for o in outs:                      # nothing between the rows
        whole = o.as_strided((o.shape[0] - 1, o.stride(0)), (o.stride(0), 1))
        assert bool((whole[:, o.shape[1]:] == -5.0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("in_place", [False, True])
def test_lists_longer_than_the_caches(env, dtype, in_place):
    """More than 2^26 entries, whose outputs go past the caches: whole pieces, what is left of one, tensors off any alignment, rows with gaps."""
    csgs, dev = env
    g = torch.Generator(device=dev).manual_seed(3)
    mk = lambda *s: torch.randn(*s, generator=g, device=dev).mul_(0.01).to(dtype)
    grads = [mk((1 << 26) + 5), mk(8195)[1:], mk(3, 701)[:, :700], mk(1)]
    grads.append(grads[0].new_empty(50_003)[3:].copy_(mk(50_000)))
    before = [t.clone() for t in grads]
    outs = grads if in_place else [torch.full_like(t, float("nan")) for t in grads]
    total, norm = total_of(before, "l2"), torch.zeros(1, device=dev)
    l = csgs.make_grad_list(grads, outs)
    csgs.csgs_grad_clip(l, csgs.GRAD_L2, 0.3 * total, norm)
    assert abs(float(norm) - total) <= 2.0 ** -23 * total
    check_clipped(before, outs, total, float(torch.tensor(0.3 * total, dtype=torch.float32)))
    if not in_place:
        assert all(torch.equal(a, b) for a, b in zip(before, grads))
