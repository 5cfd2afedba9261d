"""Rotary positions on the GPU against float64."""
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


def tolerance(x, ref, rot, interleaved, dtype, mag):
    """Half a step of the output's type, and 2^-20 of the pair's magnitudes: the angle's fraction in fp32 is off by
    2 pi 2^-25 = 2^-22.3, the hardware sine and cosine by at most 2^-22, two products and a sum by 2^-23."""
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    pair = np.zeros(x.shape)
    i = np.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    pair[..., a] = pair[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return half * np.abs(ref) + 2.0 ** -20 * mag * pair


CASES = [  # T, H, dh, rot
    (1, 1, 2, 2), (1, 8, 128, 128), (3, 5, 64, 64), (48, 64, 128, 128), (7, 3, 72, 72), (19, 6, 72, 40), (33, 4, 96, 24), (5, 2, 256, 256),
    (9, 3, 80, 6), (11, 7, 18, 14), (5, 3, 7, 4), (700, 12, 64, 32), (2500, 33, 64, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,dh,rot", CASES)
def test_rotary(P, dtype, interleaved, T, H, dh, rot):
    import torch
    rng = np.random.default_rng(T * 7 + dh + rot)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.from_numpy(rng.standard_normal((T, H, dh)).astype(np.float32)).to("cuda", dt)
    xs = x.float().cpu().numpy().astype(np.float64)
    pos = rng.integers(0, 1 << 20, T).astype(np.int32)
    pos[0] = (1 << 31) - 1 if T > 2 else 0
    turns, mag = P.rope_turns(rot, scaling="parts", factor=8, context=4096)
    tt, pp = torch.from_numpy(turns).cuda(), torch.from_numpy(pos).cuda()
    out = torch.full_like(x, 9.0)
    P.op_rotary(x, out, tt, pos=pp, interleaved=interleaved, magnitude=mag)
    ref = R.rotate(xs, pos, turns, rot, interleaved, mag)
    got = out.float().cpu().numpy().astype(np.float64)
    assert (np.abs(got - ref) <= tolerance(xs, ref, rot, interleaved, dtype, mag)).all()
    assert np.array_equal(got[..., rot:], xs[..., rot:])
    # in place gives the same bits, and what lies past the rotated dims stays
    y = x.clone()
    P.op_rotary(y, y, tt, pos=pp, interleaved=interleaved, magnitude=mag)
    assert torch.equal(y, out)
    # without positions: the token's index
    P.op_rotary(x, out, tt, interleaved=interleaved)
    ref = R.rotate(xs, np.arange(T), turns, rot, interleaved)
    assert (np.abs(out.float().cpu().numpy() - ref) <= tolerance(xs, ref, rot, interleaved, dtype, 1.0)).all()


@pytest.mark.parametrize("off", [0, 1, 4])
def test_rotary_strided(P, off):
    """Query and key heads inside a fused projection's rows, at any alignment; the value heads are not touched."""
    import torch
    rng = np.random.default_rng(off)
    T, H, dh = 21, 4, 64
    buf = torch.from_numpy(rng.standard_normal((T, 3 * H * dh + 8)).astype(np.float32)).to("cuda", torch.bfloat16)
    before = buf.clone()
    turns, _ = P.rope_turns(dh)
    x = buf[:, off:off + 3 * H * dh].unflatten(1, (3 * H, dh))[:, :2 * H]
    xs = x.float().cpu().numpy().astype(np.float64)
    P.op_rotary(x, x, torch.from_numpy(turns).cuda())
    ref = R.rotate(xs, np.arange(T), turns, dh, False)
    assert (np.abs(x.float().cpu().numpy() - ref) <= tolerance(xs, ref, dh, False, "bf16", 1.0)).all()
    keep = torch.ones(buf.shape[1], dtype=torch.bool)
    keep[off:off + 2 * H * dh] = False
    assert torch.equal(buf[:, keep.cuda()], before[:, keep.cuda()])


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_inverse_is_the_gradient(P, interleaved):
    """<rotate(x), g> has the gradient rotate_inverse(g): against the formula and against differences."""
    import torch
    rng = np.random.default_rng(5)
    T, H, dh, rot = 6, 2, 32, 24
    x, g = (torch.from_numpy(rng.standard_normal((T, H, dh)).astype(np.float32)).cuda() for _ in range(2))
    turns, mag = P.rope_turns(rot, scaling="parts", factor=4, context=64)
    tt = torch.from_numpy(turns).cuda()
    pos = torch.from_numpy(rng.integers(0, 9000, T).astype(np.int32)).cuda()
    gx = torch.empty_like(g)
    P.op_rotary(g, gx, tt, pos=pos, interleaved=interleaved, magnitude=mag, inverse=True)
    ref = R.rotate(g.cpu().numpy(), pos.cpu().numpy(), turns, rot, interleaved, mag, inverse=True)
    assert (np.abs(gx.cpu().numpy() - ref) <= tolerance(g.cpu().numpy().astype(np.float64), ref, rot, interleaved, "f32", mag)).all()
    f = lambda v: float((R.rotate(v, pos.cpu().numpy(), turns, rot, interleaved, mag) * g.cpu().numpy()).sum())  # noqa: E731
    xs = x.cpu().numpy().astype(np.float64)
    for t, h, d in [(0, 0, 0), (3, 1, 5), (5, 0, 23), (2, 1, 31)]:
        e = np.zeros_like(xs)
        e[t, h, d] = 0.5  # linear in x: any step gives the gradient
        assert abs((f(xs + e) - f(xs - e)) - float(gx[t, h, d])) <= 1e-4


def test_rotary_refuses(P):
    import torch
    x = torch.zeros(4, 2, 64, device="cuda")
    t = torch.zeros(32, dtype=torch.float64, device="cuda")
    with pytest.raises(ValueError):
        P.op_rotary(x, torch.zeros(4, 2, 32, device="cuda"), t)
    with pytest.raises(ValueError):
        P.op_rotary(x, x, t.float())
    with pytest.raises(ValueError):
        P.op_rotary(x, x, t, pos=torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(P.SgdError):
        P.op_rotary(x, x, torch.zeros(33, dtype=torch.float64, device="cuda"))
