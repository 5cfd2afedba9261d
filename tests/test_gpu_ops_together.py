"""The operators together, as a unit on packed prompts with 4-bit weights runs them: pre-norm that adds the last branch
and writes 8-bit rows, fused projection, rotation of the query and key heads in place, attention within documents,
quantisation, output projection, pre-norm, gated MLP.  Every stage is held to float64 on the data that it was given."""
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


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def values(mx):
    return R.decode(mx.codes.cpu().numpy(), mx.scales.cpu().numpy(), mx.fmt)


class Unit:
    """Buffers and weights of one unit of width d for n packed tokens."""

    def __init__(self, P, n, H, Hk, dh, F, seed):
        import torch
        rng = np.random.default_rng(seed)
        d = H * dh
        g = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda()  # noqa: E731
        self.P, self.n, self.H, self.Hk, self.dh, self.d, self.F = P, n, H, Hk, dh, d, F

        def weight(rows, K):
            m = P.MxTensor.empty("fp4", rows, K)
            P.op_mx_quantize(g(rows, K) / K ** 0.5, m)
            return m

        self.w_qkv, self.w_o, self.w1, self.w2 = weight((H + 2 * Hk) * dh, d), weight(d, d), weight(2 * F, d), weight(d, F)
        self.gain1, self.gain2 = 1 + 0.1 * g(d), 1 + 0.1 * g(d)
        self.bias = 0.1 * g((H + 2 * Hk) * dh)
        self.h0, self.r0 = g(n, d), (0.3 * g(n, d)).bfloat16()
        self.h = torch.empty(n, d, device="cuda")
        self.x1, self.x2 = P.MxTensor.empty("fp8", n, d), P.MxTensor.empty("fp8", n, d)
        self.qkv = torch.empty(n, H + 2 * Hk, dh, dtype=torch.bfloat16, device="cuda")
        self.att = torch.empty(1, n, H, dh, dtype=torch.bfloat16, device="cuda")
        self.xa, self.xf = P.MxTensor.empty("fp8", n, d), P.MxTensor.empty("fp4", n, F)
        self.o = torch.empty(n, d, device="cuda")
        self.mid = torch.empty(n, F, dtype=torch.bfloat16, device="cuda")
        self.out = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
        cuts = [0, n // 7, n // 7 + 1, n // 2, n - 5]
        r = np.zeros((1, n, 2), np.int32)
        pos = np.zeros(n, np.int32)
        for a, b in zip(cuts, cuts[1:]):
            r[0, a:b] = (a, b)
            pos[a:b] = np.arange(b - a)
        self.cuts, self.ranges, self.pos = r, torch.from_numpy(r).cuda(), torch.from_numpy(pos).cuda()
        self.turns_h, self.mag = P.rope_turns(dh, scaling="parts", factor=4, context=128)
        self.turns = torch.from_numpy(self.turns_h).cuda()

    def run(self, stream=None):
        P, H, Hk = self.P, self.H, self.Hk
        P.op_norm_add_mx(self.h0, self.gain1, self.x1, 1e-5, add=self.r0, out=self.h, stream=stream)
        P.op_linear_mx(self.x1, self.w_qkv, self.qkv.view(self.n, -1), bias=self.bias, stream=stream)
        qk = self.qkv[:, :H + Hk]
        P.op_rotary(qk, qk, self.turns, pos=self.pos, magnitude=self.mag, stream=stream)
        q, k, v = self.qkv[None, :, :H], self.qkv[None, :, H:H + Hk], self.qkv[None, :, H + Hk:]
        P.op_attention_ranges(q, k, v, self.att, self.ranges, stream=stream)
        P.op_mx_quantize(self.att.view(self.n, -1), self.xa, stream=stream)
        P.op_linear_mx(self.xa, self.w_o, self.o, stream=stream)
        P.op_norm_add_mx(self.h, self.gain2, self.x2, 1e-5, add=self.o, stream=stream)
        P.op_linear_mx(self.x2, self.w1, self.mid, act=3, gated=True, stream=stream)
        P.op_mx_quantize(self.mid, self.xf, stream=stream)
        P.op_linear_mx(self.xf, self.w2, self.out, stream=stream)

    def results(self):
        return [self.h, self.qkv, self.att, self.o, self.mid, self.out]


@pytest.mark.parametrize("n,H,Hk,dh,F", [(300, 4, 2, 64, 352), (37, 2, 2, 128, 96), (13, 6, 1, 32, 64)])
def test_unit(P, n, H, Hk, dh, F):
    u = Unit(P, n, H, Hk, dh, F, n)
    u.run()
    d = u.d
    # stream: two additions in fp32
    h1 = (u.h0 + u.r0.float())
    assert np.array_equal(f64(u.h), f64(h1 + u.o))
    # first pre-norm, exactly; projection on what it wrote, and the rotation of it
    c, s = R.quantize(R.norm(f64(h1), f64(u.gain1), float(np.float32(1e-5))), "fp8")
    assert np.array_equal(u.x1.codes.cpu().numpy(), R.pack_codes(c, "fp8")) and np.array_equal(u.x1.scales.cpu().numpy(), R.pack_scales(s))

    def product(a, w):
        a, w = values(a), values(w)
        return a @ w.T, 2.0 ** -10 * (R.block_max(a) @ R.block_max(w).T) + (a.shape[1] / 16 + 4) * 2.0 ** -24 * (np.abs(a) @ np.abs(w).T)

    z, e = product(u.x1, u.w_qkv)
    z = (z + f64(u.bias)).reshape(n, H + 2 * Hk, dh)
    e = e.reshape(z.shape) + 2.0 ** -8 * np.abs(z) * 1.01
    got = f64(u.qkv)
    assert (np.abs(got[:, H + Hk:] - z[:, H + Hk:]) <= e[:, H + Hk:]).all()
    rot = R.rotate(z[:, :H + Hk], u.pos.cpu().numpy(), u.turns_h, dh, False, u.mag)
    ez = e[:, :H + Hk]
    pair = np.concatenate([ez[..., :dh // 2] + ez[..., dh // 2:]] * 2, -1) * u.mag
    pz = np.abs(z[:, :H + Hk])
    pair += 2.0 ** -20 * u.mag * np.concatenate([pz[..., :dh // 2] + pz[..., dh // 2:]] * 2, -1)
    assert (np.abs(got[:, :H + Hk] - rot) <= pair + 2.0 ** -8 * (np.abs(rot) + pair)).all()
    # attention on the rotated heads: bf16 probabilities and output, half a step each
    q, k, v = got[None, :, :H], got[None, :, H:H + Hk], got[None, :, H + Hk:]
    ref, mag = R.attention(q, k, v, u.cuts.astype(np.int64), dh ** -0.5)
    big = dh ** -0.5 * np.linalg.norm(q, axis=-1).max() * np.linalg.norm(k, axis=-1).max()
    err = 4 * ((dh + 8) * 2.0 ** -24 + 2.0 ** -21) * big + (n + 64) * 2.0 ** -24
    assert (np.abs(f64(u.att) - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + err) * mag + 1e-30).all()
    assert (f64(u.att)[0, n - 5:] == 0).all()
    # output projection, second pre-norm, MLP
    c, s = R.quantize(f64(u.att).reshape(n, d), "fp8")
    assert np.array_equal(u.xa.codes.cpu().numpy(), R.pack_codes(c, "fp8"))
    z, e = product(u.xa, u.w_o)
    assert (np.abs(f64(u.o) - z) <= e + 2.0 ** -24 * np.abs(z)).all()
    c, s = R.quantize(R.norm(f64(u.h), f64(u.gain2), float(np.float32(1e-5))), "fp8")
    assert np.array_equal(u.x2.codes.cpu().numpy(), R.pack_codes(c, "fp8")) and np.array_equal(u.x2.scales.cpu().numpy(), R.pack_scales(s))
    z, e = product(u.x2, u.w1)
    g, up = R.act(z[:, :F], 3), z[:, F:]
    eg = 1.13 * e[:, :F] + 2e-6 * (1 + np.abs(z[:, :F]))
    assert (np.abs(f64(u.mid) - g * up) <= 2.0 ** -8 * np.abs(g * up) + 1.01 * (eg * np.abs(up) + np.abs(g) * e[:, F:] + eg * e[:, F:])).all()
    c, s = R.quantize(f64(u.mid), "fp4")
    assert np.array_equal(u.xf.codes.cpu().numpy(), R.pack_codes(c, "fp4"))
    a, w = values(u.xf), values(u.w2)
    z = a @ w.T
    assert (np.abs(f64(u.out) - z) <= 2.0 ** -8 * np.abs(z) + 1.01 * (F / 16 + 4) * 2.0 ** -24 * (np.abs(a) @ np.abs(w).T)).all()


def test_unit_streams_and_graph(P):
    """The same bits on another stream, side by side with a second unit, and in a captured graph replayed between
    eager runs."""
    import torch
    u, v = Unit(P, 200, 4, 2, 64, 160, 5), Unit(P, 333, 2, 1, 128, 96, 6)
    u.run()
    v.run()
    torch.cuda.synchronize()
    ru, rv = [t.clone() for t in u.results()], [t.clone() for t in v.results()]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (a, b):
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        u.run(a)
        v.run(b)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(u.results(), ru)) and all(torch.equal(x, y) for x, y in zip(v.results(), rv))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=a):
        u.run()
    for k in range(3):
        u.h0.mul_(0.5 + k)
        u.run()
        torch.cuda.synchronize()
        ru = [t.clone() for t in u.results()]
        for t in u.results():
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(u.results(), ru))


def test_two_graphs_with_workspaces_of_their_own(P):
    """Two captured attention calls whose splits meet in different workspaces, replayed side by side."""
    import torch
    rng = np.random.default_rng(0)
    mk = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda().bfloat16()  # noqa: E731
    calls = []
    for i in range(2):
        q, k, v = mk(1, 1, 8, 128), mk(1, 6000, 2, 128), mk(1, 6000, 2, 128)
        r = torch.tensor([[[i * 7, 6000 - i]]], dtype=torch.int32, device="cuda")
        o, ref = torch.empty_like(q), torch.empty_like(q)
        ws = torch.empty(8 << 20, dtype=torch.uint8, device="cuda")
        P.op_attention_ranges(q, k, v, ref, r)
        calls.append((q, k, v, o, r, ws, ref))
    torch.cuda.synchronize()
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for (q, k, v, o, r, ws, ref), st in zip(calls, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            P.op_attention_ranges(q, k, v, o, r, workspace=ws)
        graphs.append(g)
    for _ in range(4):
        for c in calls:
            c[3].zero_()
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for c in calls:
            assert torch.equal(c[3], c[6])
