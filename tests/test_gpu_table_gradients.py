"""Rows of a learned table by id, and the table's gradient by sorted ids, against 64-bit sums."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import plain_operators as plain

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def env():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2101_07706_amd import csgs
    csgs.lib()
    return csgs, torch.device("cuda:0")


def make_ids(n, rows, dist, seed, pad=0.05):
    rng = np.random.default_rng(seed)
    if dist == "one":
        ids = np.full(n, rows // 2)
    elif dist == "steep":
        ids = np.minimum((np.exp(rng.random(n) * np.log(rows + 1.0)) - 1).astype(np.int64), rows - 1)
    elif dist == "half":        # half of the positions hold one id, spread over all of them
        ids = np.where(rng.random(n) < 0.5, rows - 1, rng.integers(0, rows, n))
    elif dist == "ascending":
        ids = np.sort(rng.integers(0, rows, n))
    elif dist == "none":
        ids = np.full(n, -1)
    else:
        ids = rng.integers(0, rows, n)
    if pad and dist != "none":
        bad = rng.random(n)
        ids = np.where(bad < pad / 2, -1 - rng.integers(0, 5, n), np.where(bad < pad, rows + rng.integers(0, 5, n), ids))
    return torch.from_numpy(ids.astype(np.int32))


def strided(M, F, extra, dtype, dev, fill=float("nan"), shift=0):
    """A matrix with `extra` elements between rows, `shift` elements off its allocation's start; everything holds `fill`."""
    raw = torch.full((M * (F + extra) + shift + 8,), fill, dtype=dtype, device=dev)
    return raw[shift:shift + M * (F + extra)].view(M, F + extra)[:, :F]


@pytest.mark.parametrize("dtype,out_dtype", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("n,rows,F,extra,shift", [(1, 1, 1, 0, 0), (1, 1000, 64, 0, 0), (255, 37, 100, 0, 0), (1000, 513, 7, 3, 1), (777, 5000, 602, 1, 3),
                                                  (4097, 300, 256, 8, 8), (70000, 11, 3, 0, 0), (300, 40, 2500, 0, 0)])
def test_lookup(env, n, rows, F, extra, shift, dtype, out_dtype):
    csgs, dev = env
    g = torch.Generator().manual_seed(n + F)
    T = strided(rows, F, extra, DTYPES[dtype], dev, shift=shift)
    T.copy_(torch.randn(rows, F, generator=g))
    ids = make_ids(n, rows, "uniform", n)
    out = strided(n, F, extra, DTYPES[out_dtype], dev, fill=-7.0, shift=shift)
    scale = 1.7
    csgs.csgs_embed(T, ids.to(dev), out, scale=scale)
    ok = ((ids >= 0) & (ids < rows)).to(dev)
    want = torch.where(ok.unsqueeze(1), T[ids.clamp(0, rows - 1).long().to(dev)].float() * torch.tensor(scale, device=dev), torch.zeros(1, device=dev))
    assert torch.equal(out, want.to(DTYPES[out_dtype]))        # one product, one rounding: the same bits
    if extra:
        assert bool((out.as_strided((n - 1, extra), (F + extra, 1), out.storage_offset() + F) == -7.0).all()), "wrote between the rows"
    # rows up to a device count
    m = n // 3
    out.fill_(-7.0)
    csgs.csgs_embed(T, ids.to(dev), out, scale=scale, n_dev=torch.tensor([m], dtype=torch.int32, device=dev))
    assert torch.equal(out[:m], want[:m].to(DTYPES[out_dtype])) and bool((out[m:] == -7.0).all())


def run_grad(csgs, dev, ids, G, rows, scale, d_dtype, n_dev=None, extra=0):
    """Dense, accumulated and compact form on the same input: (dT, dT on top of ones, uniq, n_uniq, dR)."""
    n, F = G.shape
    scratch = torch.full((csgs.csgs_embed_grad_scratch_bytes(n, rows, F),), 0xA5, dtype=torch.uint8, device=dev)
    dT = strided(rows, F, extra, d_dtype, dev)
    acc = strided(rows, F, extra, d_dtype, dev, fill=1.0)
    uniq = torch.full((n,), -9, dtype=torch.int32, device=dev)
    n_uniq = torch.full((1,), -9, dtype=torch.int32, device=dev)
    dR = strided(n, F, extra, d_dtype, dev)
    ids = ids.to(dev)
    csgs.csgs_embed_grad(ids, G, dT, scratch, scale=scale, n_dev=n_dev)
    csgs.csgs_embed_grad(ids, G, acc, scratch, scale=scale, accumulate=True, n_dev=n_dev)
    csgs.csgs_embed_grad_rows(ids, G, rows, uniq, n_uniq, dR, scratch, scale=scale, n_dev=n_dev)
    torch.cuda.synchronize()
    return dT, acc, uniq, n_uniq, dR


def check_grad(out, ids, G, rows, scale, m=None):
    dT, acc, uniq, n_uniq, dR = out
    m = len(ids) if m is None else m
    scale = float(np.float32(scale))
    keys, want, mag = plain.embed_grad(ids[:m], G[:m].cpu(), rows, scale)
    k = len(keys)
    want, mag = torch.from_numpy(want), torch.from_numpy(mag)
    assert int(n_uniq) == k and uniq[:k].cpu().numpy().tolist() == keys.tolist()
    assert bool((uniq[k:] == -9).all()) and bool(torch.isnan(dR[k:].float()).all()), "wrote past the count"
    # sums in double (2^-53 a step: less than 2^-24 of the magnitudes), one rounding
    plain.check(dR[:k], want, mag, 1e-2, "compact")
    at = torch.from_numpy(keys)
    plain.check(dT.cpu()[at], want, mag, 1e-2, "dense")
    plain.check(acc.cpu()[at], want + 1.0, mag + 1.0, 1e-2, "accumulated")
    rest = torch.ones(rows, dtype=torch.bool)
    rest[at] = False
    assert bool((dT.cpu()[rest] == 0).all()) and bool((acc.cpu()[rest] == 1).all())


@pytest.mark.parametrize("g_dtype,d_dtype", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("n,rows,F,dist", [(1, 1, 1, "uniform"), (1, 5000, 3, "uniform"), (2, 2, 70, "one"), (63, 9, 64, "steep"), (768, 4096, 64, "steep"),
                                           (2049, 100, 33, "half"), (4096, 70000, 100, "uniform"), (5000, 3, 31, "uniform"), (3000, 65536, 16, "ascending"),
                                           (20000, 20000, 12, "half"), (40000, 1 << 24, 8, "steep"), (33000, 50, 600, "steep"), (500, 500, 5, "none")])
def test_gradient_by_sorted_ids(env, n, rows, F, dist, g_dtype, d_dtype):
    csgs, dev = env
    if rows * F > 1 << 25:
        F = 2
    ids = make_ids(n, rows, dist, n + rows)
    g = torch.Generator().manual_seed(n)
    G = strided(n, F, 1 if n % 2 else 0, DTYPES[g_dtype], dev)
    G.copy_(torch.randn(n, F, generator=g))
    G[((ids < 0) | (ids >= rows)).to(dev)] = float("nan")      # rows that no id points from do not count, whatever they hold
    out = run_grad(csgs, dev, ids, G, rows, 0.37, DTYPES[d_dtype], extra=n % 3)
    check_grad(out, ids, G, rows, 0.37)
    again = run_grad(csgs, dev, ids, G, rows, 0.37, DTYPES[d_dtype])
    for a, b in zip(out, again):
        assert torch.equal(torch.nan_to_num(a.float(), 5.0), torch.nan_to_num(b.float(), 5.0)), "two calls differ"


@pytest.mark.parametrize("n,rows,F,dist", [(1_000_000, 3000, 4, "steep"), (300_000, 1 << 20, 8, "uniform"), (200_000, 10, 17, "one"), (131_072, 50_021, 40, "half")])
def test_gradient_of_many_positions(env, n, rows, F, dist):
    csgs, dev = env
    ids = make_ids(n, rows, dist, 5)
    G = torch.randn(n, F, generator=torch.Generator().manual_seed(1)).to(dev)
    check_grad(run_grad(csgs, dev, ids, G, rows, 1.0, torch.float32), ids, G, rows, 1.0)


@pytest.mark.parametrize("n,rows", [(1 << 15, 1 << 24), (1 << 15, 1 << 17), (1 << 18, 1 << 24), (1 << 18, 1 << 17), (50_000, 1 << 20), (98_000, 1 << 18)])
@pytest.mark.parametrize("sample", [1024, 4096])
def test_ids_that_a_sample_misses(env, n, rows, sample):
    """Every (n / sample)-th position holds an id from all over the table, all the others one of a narrow range between two of those."""
    csgs, dev = env
    rng = np.random.default_rng(n)
    step = rows // sample
    ids = 5 * step + 1 + rng.integers(0, step - 1, n)
    at = np.arange(sample) * n // sample
    ids[at] = np.arange(sample) * step
    ids = torch.from_numpy(ids.astype(np.int32))
    G = torch.randn(n, 2, generator=torch.Generator().manual_seed(7)).to(dev)
    check_grad(run_grad(csgs, dev, ids, G, rows, 1.0, torch.float32), ids, G, rows, 1.0)


@pytest.mark.parametrize("n", [2048, 2049, 32768, 32769, 98_304, 98_305, 262_144])
@pytest.mark.parametrize("dist", ["steep", "half", "one", "none", "ascending"])
def test_gradient_around_the_forms_of_the_sort(env, n, dist):
    csgs, dev = env
    rows = 1000 if dist != "half" else 70_000
    ids = make_ids(n, rows, dist, n)
    G = torch.randn(n, 5, generator=torch.Generator().manual_seed(8)).to(dev)
    check_grad(run_grad(csgs, dev, ids, G, rows, 1.0, torch.float32), ids, G, rows, 1.0)


@pytest.mark.parametrize("n", [300, 9000, 70000])
@pytest.mark.parametrize("share", [0.0, 0.004, 0.5, 2.0])
def test_gradient_up_to_a_device_count(env, n, share):
    csgs, dev = env
    rows, F = 700, 20
    ids = make_ids(n, rows, "steep", n)
    m = min(n, int(n * share))
    G = torch.randn(n, F, generator=torch.Generator().manual_seed(2)).to(dev)
    G[m:] = float("inf")
    n_dev = torch.tensor([int(n * share)], dtype=torch.int32, device=dev)
    check_grad(run_grad(csgs, dev, ids, G, rows, 2.0, torch.float32, n_dev=n_dev), ids, G, rows, 2.0, m)
    n_dev.fill_(-3)
    check_grad(run_grad(csgs, dev, ids, G, rows, 2.0, torch.float32, n_dev=n_dev), ids, G, rows, 2.0, 0)


def test_gradient_against_differences(env):
    """L = sum over t of c[t] . embed(T)[t]^2 / 2: dL/dT by the library from G = c embed, and by differences of L in 64 bits."""
    csgs, dev = env
    n, rows, F, scale = 200, 30, 6, 1.5
    ids = make_ids(n, rows, "steep", 3)
    g = torch.Generator().manual_seed(4)
    T, c = torch.randn(rows, F, generator=g), torch.randn(n, F, generator=g)
    out = torch.empty((n, F), device=dev)
    csgs.csgs_embed(T.to(dev), ids.to(dev), out, scale=scale)
    G = c.to(dev) * out
    dT = torch.empty((rows, F), device=dev)
    csgs.csgs_embed_grad(ids.to(dev), G, dT, torch.empty(csgs.csgs_embed_grad_scratch_bytes(n, rows, F), dtype=torch.uint8, device=dev), scale=scale)
    ok = (ids >= 0) & (ids < rows)

    def loss(t):
        e = torch.where(ok.unsqueeze(1), scale * t[ids.clamp(0, rows - 1).long()], torch.zeros(1, dtype=torch.float64))
        return (c.double() * e * e).sum() / 2

    step = 1e-4    # L is quadratic: a central difference is exact but for rounding, 2^-53 L / step
    for v, f in [(0, 0), (1, 5), (7, 2), (29, 3), (12, 1)]:
        e = torch.zeros(rows, F, dtype=torch.float64)
        e[v, f] = step
        want = ((loss(T.double() + e) - loss(T.double() - e)) / (2 * step)).item()
        size = float((c.double().abs() * scale * scale * T.double().abs().max()).sum())
        assert abs(dT[v, f].item() - want) <= 4 * 2.0 ** -24 * size + 1e-7


def test_rows_past_32_bits(env):
    """Tables and gradients of more than 2^32 elements: rows at their very end."""
    csgs, dev = env
    rows, F, ld = (1 << 22) + 5, 3, 1 << 10
    big = torch.empty(rows * ld, dtype=torch.bfloat16, device=dev).view(rows, ld)[:, :F]
    assert (rows - 1) * ld > 1 << 32
    picks = torch.tensor([rows - 1, 0, rows - 2, rows - 1, 1 << 21], dtype=torch.int32)
    g = torch.Generator().manual_seed(6)
    vals = torch.randn(5, F, generator=g).bfloat16()
    vals[3] = vals[0]
    big[picks.long().to(dev)] = vals.to(dev)
    out = torch.empty((5, F), device=dev)
    csgs.csgs_embed(big, picks.to(dev), out)
    assert torch.equal(out.cpu(), vals.float())
    G = torch.randn(5, F, generator=g)
    csgs.csgs_embed_grad(picks.to(dev), G.to(dev), big, torch.empty(csgs.csgs_embed_grad_scratch_bytes(5, rows, F), dtype=torch.uint8, device=dev), accumulate=True)
    want = vals.double() + torch.stack([G[0].double() + G[3].double(), G[1].double(), G[2].double(), G[0].double() + G[3].double(), G[4].double()])
    plain.check(big[picks.long().to(dev)], want, want.abs(), 1e-2, "rows past 32 bits")
    # G and out past 32 bits
    n = 5 + (1 << 22)
    ids = torch.zeros(n, dtype=torch.int32)
    ids[-1] = 1
    wide = torch.zeros(1, dtype=torch.bfloat16, device=dev).expand(1)
    del big
    wide = torch.zeros(n * ld, dtype=torch.bfloat16, device=dev).view(n, ld)[:, :F]
    wide[-1] = 3.0
    wide[5] = 2.0
    dT = torch.empty((2, F), device=dev)
    csgs.csgs_embed_grad(ids.to(dev), wide, dT, torch.empty(csgs.csgs_embed_grad_scratch_bytes(n, 2, F), dtype=torch.uint8, device=dev))
    assert dT.cpu().tolist() == [[2.0] * F, [3.0] * F]
    csgs.csgs_embed(dT, ids.to(dev), wide)
    assert wide[-1].tolist() == [3.0] * F and wide[-2].tolist() == [2.0] * F


def test_on_another_stream_and_replayed(env):
    """The whole sequence on a side stream, then captured into a graph and replayed over changing inputs."""
    csgs, dev = env
    n, rows, F = 5000, 900, 24
    ids = make_ids(n, rows, "steep", 8).to(dev)
    G = torch.randn(n, F, device=dev)
    scratch = torch.empty(csgs.csgs_embed_grad_scratch_bytes(n, rows, F), dtype=torch.uint8, device=dev)
    dT, T, out = torch.empty((rows, F), device=dev), torch.randn(rows, F, device=dev), torch.empty((n, F), device=dev)
    uniq, n_uniq, dR = torch.full((n,), -1, dtype=torch.int32, device=dev), torch.zeros(1, dtype=torch.int32, device=dev), torch.zeros((n, F), device=dev)
    side = torch.cuda.Stream()

    def step(stream):
        csgs.csgs_embed(T, ids, out, scale=2.0, stream=stream)
        csgs.csgs_embed_grad(ids, G, dT, scratch, stream=stream)
        csgs.csgs_embed_grad_rows(ids, G, rows, uniq, n_uniq, dR, scratch, stream=stream)

    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    keys, want, mag = plain.embed_grad(ids.cpu(), G.cpu(), rows, 1.0)
    plain.check(dT.cpu()[torch.from_numpy(keys)], torch.from_numpy(want), torch.from_numpy(mag), 1e-2, "side stream")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(None)
    for k in range(3):
        ids.copy_(make_ids(n, rows, ["half", "uniform", "steep"][k], 20 + k))
        G.normal_()
        dT.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, dT, n_uniq)] + [dR[:int(n_uniq)].clone()]
        step(None)
        torch.cuda.synchronize()
        for a, b in zip(got, [out, dT, n_uniq, dR[:int(n_uniq)]]):
            assert torch.equal(a, b), f"replay {k}"


@pytest.mark.parametrize("rows,F,d_dtype", [(100_001, 1, "f32"), (100_001, 3, "bf16"), (300_000, 10, "f32"), (70_000, 255, "f32"), (70_000, 300, "bf16"), (33, 5, "f32")])
def test_few_positions_of_a_long_table(env, rows, F, d_dtype):
    """Rows that no position points to are cleared around those that are written, however narrow they are."""
    csgs, dev = env
    for n, dist in ((1, "one"), (500, "uniform"), (2000, "steep")):
        ids = make_ids(n, rows, dist, n + rows)
        if n > 1:
            ids[0], ids[1] = 0, rows - 1
        G = torch.randn(n, F, generator=torch.Generator().manual_seed(9)).to(dev)
        for extra in (0, 3):
            check_grad(run_grad(csgs, dev, ids, G, rows, 1.0, DTYPES[d_dtype], extra=extra), ids, G, rows, 1.0)


@pytest.mark.parametrize("F,sized_for,n", [(1024, 32768, 32767), (1024, 16384, 16383), (512, 65536, 65535), (100, 200_000, 167_000), (256, 4096, 3000)])
def test_scratch_sized_for_a_larger_call(env, F, sized_for, n):
    """Exactly the bytes that the larger call asks for serve the smaller one, which stays within them."""
    csgs, dev = env
    rows = 300
    nbytes = csgs.csgs_embed_grad_scratch_bytes(sized_for, rows, F)
    raw = torch.full((nbytes + 4096,), 0xA5, dtype=torch.uint8, device=dev)
    ids = make_ids(n, rows, "half", n)
    G = torch.randn(n, F, generator=torch.Generator().manual_seed(3)).to(dev)
    dT = torch.full((rows, F), float("nan"), device=dev)
    csgs.csgs_embed_grad(ids.to(dev), G, dT, raw[:nbytes])
    keys, want, mag = plain.embed_grad(ids, G.cpu(), rows, 1.0)
    plain.check(dT.cpu()[torch.from_numpy(keys)], torch.from_numpy(want), torch.from_numpy(mag), 1e-2, "dense")
    assert bool((raw[nbytes:] == 0xA5).all()), "wrote past the scratch"


@pytest.mark.parametrize("g_dtype,d_dtype,extra", [("f32", "f32", 0), ("bf16", "bf16", 3), ("f32", "bf16", 1), ("bf16", "f32", 5)])
@pytest.mark.parametrize("count", [0, 1, 65_536, 98_304, 131_071, 200_000, -7])
def test_many_positions_up_to_a_device_count(env, count, g_dtype, d_dtype, extra):
    """The sort by digits with a count of its own, ids outside the table among those that count, and rows that start anywhere."""
    csgs, dev = env
    n, rows, F = 131_072, 3000, 9
    ids = make_ids(n, rows, "steep", 11)
    m = max(0, min(count, n))
    G = strided(n, F, extra, DTYPES[g_dtype], dev)
    G.copy_(torch.randn(n, F, generator=torch.Generator().manual_seed(12)))
    G[m:] = float("inf")
    G[((ids < 0) | (ids >= rows)).to(dev)] = float("nan")
    out = run_grad(csgs, dev, ids, G, rows, 1.3, DTYPES[d_dtype], n_dev=torch.tensor([count], dtype=torch.int32, device=dev), extra=extra)
    check_grad(out, ids, G, rows, 1.3, m)


@pytest.mark.parametrize("g_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,F,rows,dist", [(131_072, 300, 900, "steep"), (262_144, 160, 40, "half"), (131_072, 600, 700, "steep"), (98_304, 1000, 300, "half"), (131_072, 520, 131_072, "uniform")])
def test_long_shares(env, n, F, rows, dist, g_dtype):
    """Groups whose share of a chunk is 32 positions (the first two) and 64, of many positions of wide rows."""
    csgs, dev = env
    ids = make_ids(n, rows, dist, n + F)
    G = torch.randn(n, F, generator=torch.Generator().manual_seed(13)).to(DTYPES[g_dtype]).to(dev)
    check_grad(run_grad(csgs, dev, ids, G, rows, 1.0, torch.float32), ids, G, rows, 1.0)
