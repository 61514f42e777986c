"""Products of floats that are formed from three bfloat16 parts of each operand: operands whose parts are as large as they get, all of one sign, and the ends of the range."""
import itertools
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ULP = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2101_07706_amd import csgs
    csgs.lib()
    return csgs, torch.device("cuda:0")


# Bits of a float in [1, 2): parts cut off where they are largest, rounded where they are, ties, one part alone, all bits set.
WORST = [0x3F80FFFF, 0x3F80FF7F, 0x3F807F7F, 0x3F807F80, 0x3F808080, 0x3F808081, 0x3F818180, 0x3FFF7F7F, 0x3FFFFFFF, 0x3F800001, 0x3F80007F]


def floats(bits):
    return torch.tensor(bits, dtype=torch.int32).view(torch.float32)


def bound(K, mag):
    """Of a sum of K products whose absolute values add up to mag, in 2^-24 of that: what is left out of the products, 1.001; the sums of the smaller products, 5 K roundings of at most
    2^-7 of it, 0.04 K; a rounding of the large ones' sum for 16 of them and one of both sums' sum, K / 16 + 1; what the matrix cores cut off of K - 1 terms below the largest, K - 1:
    together below 2.25 K."""
    return 2.25 * K * ULP * mag + 2.0 ** -149


# tiles of 64 and of 128, groups of wavefronts over long sums; sums of one to three products, whose bounds are close
@pytest.mark.parametrize("size", [(3, 1, 2), (2, 2, 70), (70, 3, 80), (40, 64, 130), (20, 300, 30), (5, 1024, 64), (2100, 2, 2060)], ids=str)
def test_the_largest_parts_with_one_sign(env, size):
    csgs, dev = env
    M, K, N = size
    pairs = list(itertools.product(WORST, WORST))
    if M * N > 10_000:
        pairs = pairs[:3] + [(b, b) for b in WORST]
    out, da, dw = torch.zeros(M, N, device=dev), torch.zeros(M, K, device=dev), torch.zeros(K, N, device=dev)
    scratch = torch.empty(csgs.csgs_linear_grad_scratch_bytes(M, K, N, csgs.F32), dtype=torch.uint8, device=dev)
    ones = torch.ones(M, 1, dtype=torch.float64) @ torch.ones(1, N, dtype=torch.float64)
    for a, b in pairs:
        x, y = float(floats([a])), float(floats([b]))
        A, W = torch.full((M, K), x, device=dev), torch.full((K, N), y, device=dev)
        csgs.csgs_linear(A, W, out)
        assert bool(((out.cpu().double() - K * x * y * ones).abs() <= bound(K, K * x * y)).all()), (hex(a), hex(b), "y")
        d = torch.full((M, N), y, device=dev)
        csgs.csgs_linear_grad(A, W, d, da, dw, None, None, scratch)
        # (parts of the sum, joined: one more rounding)
        assert bool(((da.cpu().double() - N * y * y).abs() <= bound(N + 1, N * y * y)).all()), (hex(a), hex(b), "da")
        assert bool(((dw.cpu().double() - M * x * y).abs() <= bound(M + 1, M * x * y)).all()), (hex(a), hex(b), "dw")


def test_gated_with_the_largest_parts(env):
    csgs, dev = env
    M, K, N = 70, 2, 80
    h = torch.zeros(M, N, device=dev)
    for bits in WORST:
        x = float(floats([bits]))
        X, W = torch.full((M, K), x, device=dev), torch.full((K, N), x, device=dev)
        csgs.csgs_gated(X, W, W, h, act=csgs.ACT_NONE)
        want = (K * x * x) ** 2
        assert bool(((h.cpu().double() - want).abs() <= 2.01 * bound(K, K * x * x) * K * x * x + ULP * want).all()), hex(bits)


# Operands near both ends of the range, whose products lie in it: every bit of every float counts, in numbers below 2^-126 as well.
@pytest.mark.parametrize("size", [(3, 1, 5), (70, 40, 80), (5, 1024, 64), (2100, 40, 2060)], ids=str)
@pytest.mark.parametrize("ends", [(1e-36, 1e3), (1e-38, 1e20), (3e-40, 1e30), (3e38, 1e-3), (1e34, 1e-34), (3.4e38, 0.0009), (2e-44, 3e38)], ids=str)
def test_the_ends_of_the_range(env, size, ends):
    csgs, dev = env
    M, K, N = size
    gen = torch.Generator().manual_seed(K)
    near = lambda r, c, v: (v * (1 - 0.4 * torch.rand(r, c, generator=gen, dtype=torch.float64))).float()
    for lo, hi in (ends, ends[::-1]):
        A, W = near(M, K, lo), near(K, N, hi)
        out = torch.zeros(M, N, device=dev)
        csgs.csgs_linear(A.to(dev), W.to(dev), out)
        want = A.double() @ W.double()
        if float(want.max()) > 3.4e38:
            continue
        # (one more rounding for each product where they are formed by the float cores)
        assert bool(((out.cpu().double() - want).abs() <= bound(K, want) + K * ULP * want).all())


def test_the_largest_float_among_others(env):
    csgs, dev = env
    M, K, N = 70, 90, 40
    gen = torch.Generator().manual_seed(1)
    A, W = torch.randn(M, K, generator=gen), torch.randn(K, N, generator=gen).abs()
    clean, out = torch.zeros(M, N, device=dev), torch.zeros(M, N, device=dev)
    csgs.csgs_linear(A.to(dev), W.to(dev), clean)
    for big in (0x7F7FFFFF, 0x7F7F8000, 0x7F7F7FFF, 0x7800_0000):
        A2, W2 = A.clone(), W.clone()
        A2[33, 7] = floats([big])[0]
        W2[7] *= 0.25 / W2[7].max()
        csgs.csgs_linear(A.to(dev), W2.to(dev), clean)
        csgs.csgs_linear(A2.to(dev), W2.to(dev), out)
        want, mag = A2.double() @ W2.double(), A2.abs().double() @ W2.abs().double()
        assert bool(((out.cpu().double() - want).abs() <= bound(2 * K, mag)).all()), hex(big)
        keep = torch.arange(M, device=dev) != 33
        assert torch.equal(out[keep], clean[keep])
        # times nothing it is nothing
        W2[7] = 0.0
        csgs.csgs_linear(A2.to(dev), W2.to(dev), out)
        want, mag = A.double() @ W2.double(), A.abs().double() @ W2.abs().double()
        assert bool(((out.cpu().double() - want).abs() <= bound(2 * K, mag)).all()), hex(big)
    assert math.isfinite(float(out.sum()))
