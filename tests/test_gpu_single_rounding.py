"""Results that are formed in double reach bfloat16 by one rounding: sums of a table's gradient, and clipped gradients."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def env():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2101_07706_amd import csgs
    csgs.lib()
    return csgs, torch.device("cuda:0")


def nearest_bf16(x):
    """The bfloat16 nearest to each double, ties to even, by whole multiples of its spacing (normal numbers)."""
    x = np.asarray(x, np.float64)
    _, e = np.frexp(x)                          # |x| in [2^(e - 1), 2^e): 8 bits of it
    step = np.ldexp(1.0, e - 8)
    return np.where(x == 0, 0.0, np.rint(x / step) * step)


# sums whose float lies halfway between two bfloat16 numbers, and the double on one side of it
TRIPLES = [(1.0, 2.0 ** -8, 2.0 ** -30), (1.0, 3 * 2.0 ** -8, -(2.0 ** -30)), (-1.0, -(2.0 ** -8), -(2.0 ** -40)), (1.0, 2.0 ** -8, 0.0), (1.0, 2.0 ** -8, -(2.0 ** -30)),
           (-64.0, -0.75, 2.0 ** -26)]


@pytest.mark.parametrize("g_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,rows,F", [(6, 2, 1), (700, 9, 100), (1500, 300, 7), (5000, 700, 33), (30_000, 3, 6), (120_000, 500, 16)])
def test_sums(env, n, rows, F, g_dtype):
    """Every id's positions hold one of the triples somewhere and zeros otherwise."""
    csgs, dev = env
    rng = np.random.default_rng(n)
    ids = rng.integers(0, rows, n)
    ids[:3 * min(rows, n // 3)] = np.repeat(np.arange(min(rows, n // 3)), 3)
    rng.shuffle(ids)
    G = np.zeros((n, F))
    for v in range(rows):
        at = np.flatnonzero(ids == v)
        if len(at) >= 3:
            at = rng.choice(at, 3, replace=False)
            for f in range(F):
                G[at, f] = rng.permutation(TRIPLES[(v + f) % len(TRIPLES)])
    sums = np.zeros((rows, F))
    np.add.at(sums, ids, G)                     # exact: the triples need 34 to 47 bits
    G, ids = torch.from_numpy(G).to(g_dtype).to(dev), torch.from_numpy(ids.astype(np.int32)).to(dev)
    bf16 = torch.bfloat16
    scratch = torch.empty(csgs.csgs_embed_grad_scratch_bytes(n, rows, F), dtype=torch.uint8, device=dev)
    dT, acc = torch.empty(rows, F, dtype=bf16, device=dev), torch.full((rows, F), 2.0, dtype=bf16, device=dev)
    uniq, n_uniq, dR = torch.empty(n, dtype=torch.int32, device=dev), torch.zeros(1, dtype=torch.int32, device=dev), torch.empty(n, F, dtype=bf16, device=dev)
    csgs.csgs_embed_grad(ids, G, dT, scratch)
    csgs.csgs_embed_grad(ids, G, acc, scratch, accumulate=True, scale=-2.0)
    csgs.csgs_embed_grad_rows(ids, G, rows, uniq, n_uniq, dR, scratch, scale=0.5)
    k = int(n_uniq)
    at = uniq[:k].long().cpu().numpy()
    assert np.array_equal(dT.double().cpu().numpy(), nearest_bf16(sums))
    assert np.array_equal(acc.double().cpu().numpy(), nearest_bf16(2.0 - 2.0 * sums))
    assert np.array_equal(dR[:k].double().cpu().numpy(), nearest_bf16(0.5 * sums[at]))


def test_clipped_gradients(env):
    """Coefficients for which some number's product, as a float, lies halfway between two bfloat16 numbers."""
    csgs, dev = env
    values = np.concatenate([np.arange(128, 256), -np.arange(128, 256)]) / 128.0
    total = np.abs(values).max()
    limits = (np.float32(0.5) + np.arange(40_000, dtype=np.float32) * np.float32(2.0 ** -17)).astype(np.float64)
    products = (limits / (total + 1e-6))[:, None] * values
    once = nearest_bf16(products)
    twice = nearest_bf16(products.astype(np.float32).astype(np.float64))
    picks = np.flatnonzero((once != twice).any(1))[:12]
    assert len(picks) >= 4                      # (about one product in 2^17)
    g = torch.from_numpy(values).bfloat16().to(dev)
    gapped = torch.zeros(3, 300, dtype=torch.bfloat16, device=dev)[:, :256]
    gapped.copy_(g)
    outs = [torch.empty_like(g), torch.empty_like(gapped)]
    l = csgs.make_grad_list([g, gapped], outs)
    for k in picks:
        csgs.csgs_grad_clip(l, csgs.GRAD_MAX, float(limits[k]))
        assert np.array_equal(outs[0].double().cpu().numpy(), once[k])
        assert all(np.array_equal(row, once[k]) for row in outs[1].double().cpu().numpy())


def test_values_at_the_ends_of_the_range(env):
    """Zeros, the smallest numbers, and sums past the largest one."""
    csgs, dev = env
    pairs = [(0.0, 0.0), (2.0 ** -133, 0.0), (2.0 ** -133, 2.0 ** -133), (3.3e38, 3.3e38), (-3.3e38, -3.3e38), (3.0e38, -3.0e38), (float("inf"), 1.0),
             (float("nan"), 1.0), (float("inf"), float("-inf"))]
    ids = torch.arange(len(pairs), dtype=torch.int32).repeat_interleave(2).to(dev)
    G = torch.tensor(pairs).view(-1, 1).to(dev)
    dT = torch.empty(len(pairs), 1, dtype=torch.bfloat16, device=dev)
    scratch = torch.empty(csgs.csgs_embed_grad_scratch_bytes(len(ids), len(pairs), 1), dtype=torch.uint8, device=dev)
    csgs.csgs_embed_grad(ids, G, dT, scratch)
    inf, nan = float("inf"), float("nan")
    want = torch.tensor([0.0, 2.0 ** -133, 2.0 ** -132, inf, -inf, 0.0, inf, nan, nan])
    got = dT.float().cpu().view(-1)
    assert torch.equal(torch.nan_to_num(got, 7.0, 8e37, -8e37), torch.nan_to_num(want, 7.0, 8e37, -8e37)) and torch.equal(torch.isnan(got), torch.isnan(want))
