"""Products of e4m3 rows with e2m1 weights: what the matrix instruction keeps of its products, pinned from both sides.

The instruction adds the products of eight neighbouring columns aligned to the group's largest exponent and cuts each 13 bits
below it; the groups' sums and the steps are added in fp32.  With E(x) the exponent of a code (e4m3 at least -6, e2m1 at least 0), a
group's products are cut to multiples of 2^(max(E(a) + E(w)) - 13) times the block's scales.  Where the elements of A span at most eight
binades (exponents e .. e + 7) nothing is cut: their last bit is 2^(e - 3), that of W's 2^-1, and e - 4 = (e + 7) + 2 - 13."""
import numpy as np
import pytest

import ops_reference as R

U = 2.0 ** -24


def rows(rng, kind, M, K):
    """Values on e4m3's grid and scale bytes."""
    sign = rng.choice([-1.0, 1.0], (M, K))
    if kind == "eight_binades":
        return sign * R.FP8[rng.integers(64, 127, (M, K))], np.full((M, K // 32), 120)  # exponents 1 to 8
    if kind == "normal":
        c, s = R.quantize(rng.standard_normal((M, K)), "fp8")
        return np.where(c > 127, -1.0, 1.0) * R.FP8[c & 127], s
    return sign * R.FP8[rng.integers(0, 127, (M, K))], np.full((M, K // 32), 120) if kind == "all_codes" else rng.integers(97, 157, (M, K // 32))


def weights(rng, kind, N, K):
    return (rng.choice([-1.0, 1.0], (N, K)) * R.FP4[rng.integers(0, 8, (N, K))],
            rng.integers(97, 157, (N, K // 32)) if kind == "all_scales" else np.full((N, K // 32), 125))


def exponent(x, least):
    return np.maximum(np.frexp(np.abs(x))[1] - 1, least) * (x != 0) + least * (x == 0)


def steps(a, sa, w, sw, bits=13):
    """The multiple that the products of every row, column and group of eight are cut to: [M, N, K / 8]."""
    ea, ew = (exponent(x, least).reshape(len(x), -1, 8) for x, least in ((a, -6), (w, 0)))
    e = (ea[:, None] + ew[None]).max(-1)
    s = (sa[:, None] + sw[None] - 254).repeat(4, -1)
    return np.exp2((e + s - bits).astype(np.float64))


def bound(a, sa, w, sw, A, W):
    """Of |sum - exact|.  At most seven products of a group lose less than a step each, toward zero; their signs are
    independent, so a sum of errors of at most q_i passes 7 sqrt(sum q_i^2) with a probability of 2 exp(-49 / 2) = 5e-11
    (Hoeffding, 1963).  Sums in fp32, one a group: 4 sqrt(K / 8) U of the sum of magnitudes, and its rounding."""
    q = steps(a, sa, w, sw)
    mag = np.abs(A) @ np.abs(W).T
    return np.minimum(7 * q.sum(-1), 7 * np.sqrt(7 * (q * q).sum(-1))) + (4 * np.sqrt(a.shape[1] / 8) + 1) * U * mag, q


def case(kind, M, N, K, seed=0):
    rng = np.random.default_rng(K + M + seed)
    a, sa = rows(rng, kind, M, K)
    w, sw = weights(rng, kind, N, K)
    return a, sa, w, sw, a * np.exp2(sa - 127.0).repeat(32, 1), w * np.exp2(sw - 127.0).repeat(32, 1)


def emulate(a, sa, w, sw, A, W, bits=13, group=8):
    """The instruction's sums with the cut at `bits` under the largest exponent of `group` columns (which has nonzero products only)."""
    p = A[:, None] * W[None]
    e = np.frexp(np.abs(p))[1] - 2  # a product of two significands below 2 lies up to a binade above its exponents' sum
    e = np.where(p == 0, -1000, e).reshape(*p.shape[:2], -1, group).max(-1)
    q = np.exp2((np.maximum(e, -900) - bits).astype(np.float64)).repeat(group, -1)
    return (np.trunc(p / q) * q).sum(-1)


@pytest.mark.parametrize("kind", ["normal", "all_codes", "all_scales"])
@pytest.mark.parametrize("K", [64, 512])
def test_coarser_sums_break_the_bound(kind, K):
    """The described cut keeps the bound; a cut four bits earlier and sums held in bf16 do not."""
    c = case(kind, 16, 24, K)
    z = c[4] @ c[5].T
    tol, _ = bound(*c)
    assert (np.abs(emulate(*c, bits=13) - z) <= tol).all()
    assert (np.abs(emulate(*c, bits=9, group=64) - z) > tol).any()
    b = z.astype(np.float32).view(np.uint32)
    half = (((b + 0x7FFF + ((b >> 16) & 1)) & np.uint32(0xFFFF0000)).view(np.float32)).astype(np.float64)
    assert (np.abs(half - z) > tol).any()


def product(P, a, sa, w, sw, tile):
    import torch
    ca = R.nearest(np.abs(a), "fp8") + 128 * np.signbit(a)
    cw = R.nearest(np.abs(w), "fp4") + 8 * np.signbit(w)
    A, W = (P.MxTensor(f, torch.from_numpy(R.pack_codes(c, f)).cuda(), torch.from_numpy(R.pack_scales(s)).cuda())
            for f, c, s in (("fp8", ca, sa), ("fp4", cw, sw)))
    out = torch.empty(a.shape[0], w.shape[0], device="cuda")
    P.op_linear_mx(A, W, out, tile=tile)
    return out.cpu().numpy().astype(np.float64)


@pytest.fixture(scope="module")
def P():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_29505_amd as P
    P.lib()
    return P


@pytest.mark.gpu
@pytest.mark.parametrize("tile", range(1, 9))
@pytest.mark.parametrize("K", [64, 512])
def test_rows_of_eight_binades_are_exact(P, tile, K):
    c = case("eight_binades", 16, 68, K)
    unit = 2.0 ** (1 - 3 - 1) * 2.0 ** (120 + 125 - 254)
    assert (np.abs(c[4]) @ np.abs(c[5]).T).max() < unit * 2.0 ** 24  # every partial sum is a whole number of units that fp32 holds
    assert np.array_equal(product(P, *c[:4], tile), c[4] @ c[5].T)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["normal", "all_codes", "all_scales"])
@pytest.mark.parametrize("M,K,tile", [(16, 64, 8), (16, 4096, 8), (70, 64, 7), (70, 512, 1), (70, 512, 2), (70, 512, 3), (70, 512, 4), (70, 512, 5),
                                      (70, 512, 6), (70, 2048, 7)])
def test_sums_keep_thirteen_bits_of_a_group(P, kind, M, K, tile):
    c = case(kind, M, 64, K)
    z = c[4] @ c[5].T
    tol, q = bound(*c)
    off = np.abs(product(P, *c[:4], tile) - z)
    size = np.sqrt((c[4] ** 2) @ (c[5] ** 2).T)
    print(kind, M, K, tile, "of the bound", (off / tol).max(), "rms", np.sqrt((off ** 2).mean() / (size ** 2).mean()), "largest", (off / size).max())
    assert (off <= tol).all()
    # on average: the squares of at most seven errors below a step each, and of the sums' roundings
    assert (off ** 2).mean() <= (7 * (q * q).sum(-1) + (K / 8) * (U * (np.abs(c[4]) @ np.abs(c[5]).T)) ** 2).mean()
