"""Microscaled rows on the GPU: quantisation, the pre-norm that writes them, their products, against float64."""
import numpy as np
import pytest

import ops_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_29505_amd as P
    P.lib()
    return P


def dev(x, dtype="f32"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to("cuda", torch.bfloat16 if dtype == "bf16" else torch.float32)


def host(t):
    import torch
    return t.to(torch.float32).cpu().numpy().astype(np.float64) if t.is_floating_point() else t.cpu().numpy()


def mx_of(P, fmt, x):
    """Device tensor of the float64 rows x, quantised by the reference, and the values it holds."""
    import torch
    c, s = R.quantize(x, fmt)
    codes, scales = R.pack_codes(c, fmt), R.pack_scales(s)
    return P.MxTensor(fmt, torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()), R.decode(codes, scales, fmt)


def spread(rng, rows, K):
    """Rows whose blocks differ widely in size."""
    return rng.standard_normal((rows, K)) * np.exp2(rng.integers(-12, 12, (rows, K // 32))).repeat(32, 1)


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K", [(1, 32), (3, 64), (7, 288), (200, 4096), (65, 8224)])
def test_quantize(P, fmt, dtype, rows, K):
    import torch
    rng = np.random.default_rng(rows + K)
    x = spread(rng, rows, K)
    x[0, :32] = 0.0
    x[-1, 5] = np.exp2(-140.0)  # a subnormal among ordinary values
    # ties and the values around them: halves of the grid's steps, exact in bf16
    x[-1, :32] = (np.arange(32) - 16) * 0.25
    t = dev(x, dtype)
    x = host(t)
    mx = P.MxTensor.empty(fmt, rows, K)
    mx.codes.fill_(0xEE)
    mx.scales.fill_(0xEE)
    P.op_mx_quantize(t, mx)
    c, s = R.quantize(x, fmt)
    assert np.array_equal(host(mx.scales), R.pack_scales(s))
    assert np.array_equal(host(mx.codes), R.pack_codes(c, fmt))
    for dt in (torch.bfloat16, torch.float32):
        out = torch.full((rows, K), 7.0, dtype=dt, device="cuda")
        P.op_mx_dequantize(mx, out)
        assert np.array_equal(host(out), R.decode(host(mx.codes), host(mx.scales), fmt))


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_quantize_special_values(P, fmt):
    """Zeros of either sign, the smallest and largest blocks, infinities and NaN; strided rows."""
    import torch
    x = np.zeros((6, 64))
    x[0, :4] = [-0.0, 0.0, -1e-45, 1e-45]
    x[1, :3] = [2.0 ** 127, -3e38, 1.0]
    x[2, 3] = np.inf
    x[3, 40] = np.nan
    x[4, :32] = np.exp2(-126.0) * np.linspace(-2, 2, 32)
    x[5] = np.linspace(-500, 500, 64)
    wide = torch.full((6, 96), 3.0, device="cuda")
    wide[:, 8:72] = dev(x)
    mx = P.MxTensor.empty(fmt, 6, 64)
    P.op_mx_quantize(wide[:, 8:72], mx)
    x = host(wide[:, 8:72])
    c, s = R.quantize(x, fmt)
    assert np.array_equal(host(mx.scales), R.pack_scales(s))
    assert np.array_equal(host(mx.codes), R.pack_codes(c, fmt))
    P.op_mx_dequantize(mx, wide[:, 8:72])
    got = host(wide)
    ref = R.decode(host(mx.codes), host(mx.scales), fmt)
    assert np.array_equal(got[:, 8:72], ref, equal_nan=True)
    assert np.isnan(ref[2, :32]).all() and np.isnan(ref[3, 32:]).all() and np.isfinite(ref[3, :32]).all()
    assert (got[:, :8] == 3).all() and (got[:, 72:] == 3).all()  # what lies beside the rows is left alone


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("xdt,adt", [("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", None), ("bf16", None)])
@pytest.mark.parametrize("M,d", [(1, 32), (5, 4096), (3, 8192), (1030, 288), (1027, 2080), (37, 4128)])
def test_norm_add(P, fmt, xdt, adt, M, d):
    """The stream bit for bit, and the codes of the float64 norm of the stored stream."""
    import torch
    rng = np.random.default_rng(M + d)
    x = dev(rng.standard_normal((M, d)) * np.exp2(rng.integers(-3, 4, (1, d))), xdt)
    add = None if adt is None else dev(rng.standard_normal((M, d)) * 0.3, adt)
    w = 1 + 0.1 * rng.standard_normal(d).astype(np.float32)
    mx = P.MxTensor.empty(fmt, M, d)
    mx.scales.fill_(0xEE)
    h = x.clone() if add is None else (x.float() + add.float()).to(x.dtype)
    out = None if add is None else torch.empty_like(x)
    before = x.clone()
    P.op_norm_add_mx(x, dev(w), mx, 1e-5, add=add, out=out)
    assert torch.equal(x, before)
    if add is not None:
        assert torch.equal(out, h)
        mx2 = P.MxTensor.empty(fmt, M, d)
        P.op_norm_add_mx(x, dev(w), mx2, 1e-5, add=add)  # in place
        assert torch.equal(x, h) and torch.equal(mx2.codes, mx.codes) and torch.equal(mx2.scales, mx.scales)
    c, s = R.quantize(R.norm(host(h), w.astype(np.float64), float(np.float32(1e-5))), fmt)
    assert np.array_equal(host(mx.scales), R.pack_scales(s))
    assert np.array_equal(host(mx.codes), R.pack_codes(c, fmt))


def test_norm_add_zero_and_nan_rows(P):
    import torch
    x = torch.zeros(3, 64, device="cuda")
    x[1, 7] = float("nan")
    x[2, :] = 1.0
    mx = P.MxTensor.empty("fp8", 3, 64)
    P.op_norm_add_mx(x, torch.ones(64, device="cuda"), mx, 1e-5)
    v = R.decode(host(mx.codes), host(mx.scales), "fp8")
    # 1 / sqrt(1 + 1e-5) = 0.999995 lies in [2^-1, 1): scale 2^(-1 - 8), 511.997 saturates at 448, 448 / 512 = 0.875
    assert (v[0] == 0).all() and np.isnan(v[1]).all() and (v[2] == 0.875).all()


def linear_case(P, fmt, M, N, K, seed, gated=False):
    rng = np.random.default_rng(seed)
    A, a = mx_of(P, fmt, spread(rng, M, K))
    W, w = mx_of(P, "fp4", rng.standard_normal((2 * N if gated else N, K)) / np.sqrt(K))
    return rng, A, a, W, w


def product(a, w, fmt):
    """The product and a bound on the error of its sum.  fp32 additions: each of at most K / 16 roundings of
    partial sums is off by 2^-24 of the sum of magnitudes.  e4m3 rows: a step of 64 products drops what lies
    2^-16 below its largest product, at most 64 of them: 2^-10 of it; the largest is at most the product of the
    block maxima."""
    z = a @ w.T
    err = (a.shape[1] / 16 + 4) * 2.0 ** -24 * (np.abs(a) @ np.abs(w).T)
    if fmt == "fp8":
        err = err + 2.0 ** -10 * (R.block_max(a) @ R.block_max(w).T)
    return z, err


LINEAR = [(1, 64, 64), (1, 580, 4096), (16, 260, 160), (17, 64, 96), (33, 132, 288), (64, 1024, 1024), (130, 200, 480), (200, 256, 2048),
          (257, 580, 128), (300, 768, 736), (513, 320, 256), (1000, 516, 1312)]


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("M,N,K", LINEAR)
@pytest.mark.parametrize("tile", [0, 1, 2, 3, 4, 5, 6, 7, 8])
def test_linear(P, fmt, M, N, K, tile):
    """Every tile, both outputs, with and without bias; rows and columns past the output stay as they were."""
    import torch
    if tile == 8 and M > 16:
        pytest.skip("the kernel for up to 16 rows")
    rng, A, a, W, w = linear_case(P, fmt, M, N, K, M + N + K)
    b = 0.1 * rng.standard_normal(N)
    bias = dev(b)
    z, err = product(a, w, fmt)
    z = z + host(bias)
    err = err + 2.0 ** -23 * np.abs(z)  # the bias's addition
    for dt, half in ((torch.bfloat16, 2.0 ** -8), (torch.float32, 2.0 ** -24)):
        wide = torch.full((M + 2, N + 8), 5.0, dtype=dt, device="cuda")
        P.op_linear_mx(A, W, wide[1:M + 1, 4:N + 4], bias=bias, tile=tile)
        got = host(wide)
        assert (np.abs(got[1:-1, 4:-4] - z) <= half * np.abs(z) + err * (1 + half)).all()
        assert (got[0] == 5).all() and (got[-1] == 5).all() and (got[:, :4] == 5).all() and (got[:, -4:] == 5).all()


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("M,N,K,tile", [(1, 64, 256, 0), (16, 96, 4096, 8), (5, 32, 96, 7), (130, 256, 288, 1), (130, 288, 288, 2), (130, 256, 288, 3),
                                        (260, 384, 160, 4), (200, 128, 512, 5), (70, 160, 224, 6), (70, 160, 224, 7), (300, 1152, 320, 0)])
@pytest.mark.parametrize("act", [0, 1, 2, 3])
def test_linear_act_and_gate(P, fmt, M, N, K, tile, act):
    import torch
    rng, A, a, W, w = linear_case(P, fmt, M, N, K, M + N + K + act, gated=True)
    b = dev(0.1 * rng.standard_normal(2 * N))
    z, err = product(a, w, fmt)
    z = z + host(b)
    err = err + 2.0 ** -23 * np.abs(z)
    out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    P.op_linear_mx(A, W, out, bias=b, act=act, gated=True, tile=tile)
    g, u = R.act(z[:, :N], act), z[:, N:]
    # slopes of the activations are at most 1.13; their fp32 forms are off by 1e-6 of their argument
    eg = 1.13 * err[:, :N] + 2e-6 * (1 + np.abs(z[:, :N]))
    tol = 2.0 ** -8 * np.abs(g * u) + eg * np.abs(u) + np.abs(g) * err[:, N:] + eg * err[:, N:]
    assert (np.abs(host(out) - g * u) <= tol * 1.01).all()
    half = P.MxTensor("fp4", W.codes[:N].contiguous(), W.scales[:, :N].contiguous())
    P.op_linear_mx(A, half, out, bias=b[:N].contiguous(), act=act, tile=tile)
    assert (np.abs(host(out) - g) <= 2.0 ** -8 * np.abs(g) + eg * 1.01).all()


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_linear_whole_range(P, fmt):
    """Codes of every value, scales from end to end of a range that fp32 holds, and a block without a value."""
    import torch
    rng = np.random.default_rng(3)
    M, N, K = 40, 64, 512
    ca = rng.integers(0, 256, (M, K if fmt == "fp8" else K // 2)).astype(np.uint8)
    if fmt == "fp8":
        ca[(ca & 127) == 127] = 0
    cw = rng.integers(0, 256, (N, K // 2)).astype(np.uint8)
    sa = rng.integers(97, 157, (2, M, 8)).astype(np.uint8)
    sw = rng.integers(97, 157, (2, N, 8)).astype(np.uint8)
    sa[0, 3, 2] = 255  # a NaN block spoils its row, and no other
    a, w = R.decode(ca, sa, fmt), R.decode(cw, sw, "fp4")
    A, W = (P.MxTensor(f, torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()) for f, c, s in ((fmt, ca, sa), ("fp4", cw, sw)))
    for tile in (0, 1, 2, 5, 7):
        out = torch.empty(M, N, device="cuda")
        P.op_linear_mx(A, W, out, tile=tile)
        got = host(out)
        assert np.isnan(got[3]).all()
        keep = np.arange(M) != 3
        z, err = product(a[keep], w, fmt)
        assert (np.abs(got[keep] - z) <= 2.0 ** -24 * np.abs(z) + err).all()


def test_linear_same_bits(P):
    """The same call twice, and on a stream of its own, gives the same bits (no atomics)."""
    import torch
    rng, A, a, W, w = linear_case(P, "fp8", 300, 512, 2048, 1)
    outs = [torch.empty(300, 512, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    P.op_linear_mx(A, W, outs[0])
    P.op_linear_mx(A, W, outs[1])
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    P.op_linear_mx(A, W, outs[2], stream=st)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_binding_refuses(P):
    """Tensors that do not fit together never reach the library."""
    import torch
    A, W = P.MxTensor.empty("fp8", 4, 64), P.MxTensor.empty("fp4", 8, 64)
    out = torch.empty(4, 8, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        P.op_linear_mx(A, P.MxTensor.empty("fp4", 8, 96), out)
    with pytest.raises(ValueError):
        P.op_linear_mx(A, P.MxTensor.empty("fp8", 8, 64), out)
    with pytest.raises(ValueError):
        P.op_linear_mx(A, W, out.t())
    with pytest.raises(ValueError):
        P.op_linear_mx(A, W, out, bias=torch.zeros(4, device="cuda"))
    with pytest.raises(ValueError):
        P.op_mx_quantize(torch.zeros(4, 32, device="cuda"), A)
    with pytest.raises(ValueError):
        P.op_norm_add_mx(torch.zeros(4, 64, device="cuda"), torch.ones(64, device="cuda"), A, 1e-5, out=torch.zeros(4, 64, device="cuda"))
    with pytest.raises(ValueError):
        P.MxTensor("fp8", A.codes, A.scales[:, :2].contiguous())
    with pytest.raises(P.SgdError):
        P.MxTensor.empty("fp8", 4, 40)


@pytest.mark.parametrize("d", [64, 640, 4096])
@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_norm_rounds_once_below_fp32s_normal_range(P, fmt, d):
    """Gains so small that the normalised values lie below 2^-126, a quarter of fp32's last bit above or below the middle between two
    codes: their rows are normalised by exactly 1, so the values are 1.25 w and 0.75 w."""
    import torch
    x = np.ones((2, d), np.float32)
    x[:, :7] = [1.25, 0.75, 1.25, 0.75, 0.5, 1.5, 0.5]  # squares that sum to 7: the mean square is 1
    x[1] = -x[1]
    q = 4096 if fmt == "fp8" else 1 << 20  # the first middle in units of 2^-149 (code steps of 2^-136 and 2^-128)
    assert (4 * q + 1) % 5 == 0 and (28 * q - 1) % 3 == 0
    w = np.zeros(d)
    w[0], w[1] = (4 * q + 1) // 5, (28 * q - 1) // 3  # 1.25 w = q + 1/4 goes up to code 1; 0.75 w = 7 q - 1/4 down to code 3
    w[2], w[3] = (4 * q - 4) // 5, (28 * q + 4) // 3
    w[40:] = q * np.arange(d - 40) % (1 << 22)
    w = (w * 2.0 ** -149).astype(np.float32)
    t = torch.from_numpy(x).cuda()
    mx = P.MxTensor.empty(fmt, 2, d)
    P.op_norm_add_mx(t, torch.from_numpy(w).cuda(), mx, 0.0)
    y = R.norm(x.astype(np.float64), w.astype(np.float64), 0.0)
    assert np.array_equal(y, x * w.astype(np.float64))
    c, s = R.quantize(y, fmt)
    assert not s.any() and list(c[0, :2]) == [1, 3]
    assert np.array_equal(host(mx.scales), R.pack_scales(s))
    assert np.array_equal(host(mx.codes), R.pack_codes(c, fmt))
