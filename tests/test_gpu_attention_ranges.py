"""Attention over key intervals on the GPU against float64."""
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


def make(seed, dtype, B, H, Hk, dh, nq, nk, size=1.0):
    """q, k, v on the device, key and value rows beside each other, and as float64."""
    import torch
    rng = np.random.default_rng(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = torch.from_numpy((size * rng.standard_normal((B, nq, H, dh))).astype(np.float32)).to("cuda", dt)
    kv = torch.from_numpy(rng.standard_normal((B, nk, 2, Hk, dh)).astype(np.float32)).to("cuda", dt)
    return rng, q, kv[:, :, 0], kv[:, :, 1]


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def check(P, q, k, v, ranges, dtype, cap=0.0, slopes=None, pos=None, scale=None, o=None):
    """Runs and compares.  Bound: half a step of the output; in bf16 the probabilities are rounded to bf16 for
    their product (half a step of sum p |v|); a score is off by (dh + 8) 2^-24 of scale sum |q| |k| and by 2^-21 of its
    own size and its bias's (log2 domain, tanh), and a probability by twice that, in the sum over the keys and in the
    divisor; fp32 sums over the keys: nk 2^-24 of sum p |v| in order."""
    import torch
    B, nq, H, dh = q.shape
    nk = k.shape[1]
    o = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda") if o is None else o
    r = torch.from_numpy(ranges.astype(np.int32)).cuda()
    P.op_attention_ranges(q, k, v, o, r, scale=scale, cap=cap, slopes=None if slopes is None else torch.from_numpy(slopes.astype(np.float32)).cuda(),
                          pos=None if pos is None else torch.from_numpy(pos.astype(np.int32)).cuda())
    sc = dh ** -0.5 if scale is None else scale
    sl = None if slopes is None else slopes.astype(np.float32).astype(np.float64)
    qs, ks, vs = f64(q), f64(k), f64(v)
    ref, mag = R.attention(qs, ks, vs, np.clip(ranges, 0, nk), sc, cap, sl, pos)
    with np.errstate(invalid="ignore"):
        big = sc * np.nanmax(np.linalg.norm(qs, axis=-1)) * np.nanmax(np.where(np.isfinite(ks), np.abs(ks), 0).max(-1)) * dh ** 0.5
    err = 2 * ((dh + 8) * 2.0 ** -24 * big + 2.0 ** -21 * (min(big, cap) if cap else big)
               + (0 if sl is None else 2.0 ** -21 * np.abs(sl).max() * (np.abs(pos).max() + nk if pos is not None else nk + nq)))
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    p_err = (2.0 ** -8 if dtype == "bf16" else 0) + 2 * err + (nk + 64) * 2.0 ** -24
    got = f64(o)
    fine = np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)])
    off = np.abs(np.where(fine, got, 0) - np.where(fine, ref, 0))
    tol = half * np.abs(np.where(fine, ref, 0)) + p_err * np.where(fine, mag, 1) + 1e-30
    assert (off <= tol).all(), float((off / tol).max())
    return o, ref


def documents(B, n, cuts):
    """Bidirectional within documents; sample b's cuts."""
    r = np.zeros((B, n, 2), np.int64)
    for b in range(B):
        c = cuts[b]
        for x, y in zip(c, c[1:]):
            r[b, x:y] = (x, y)
    return r


def causal(B, nq, nk, lens, prefix=0):
    r = np.zeros((B, nq, 2), np.int64)
    for b in range(B):
        for i in range(nq):
            p = i + lens[b] - nq
            r[b, i] = (0, min(max(p + 1, prefix), lens[b])) if p >= 0 else (0, 0)
    return r


SHAPES = [  # B, H, Hk, dh, n
    (1, 1, 1, 8, 1), (2, 3, 3, 64, 17), (1, 4, 2, 72, 64), (2, 2, 2, 128, 65), (1, 8, 1, 128, 130), (1, 2, 1, 96, 257), (3, 2, 2, 80, 100),
    (1, 6, 2, 40, 333), (1, 1, 1, 128, 700)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mode", ["plain", "cap", "bias", "both"])
@pytest.mark.parametrize("B,H,Hk,dh,n", SHAPES)
def test_documents_and_prefixes(P, dtype, mode, B, H, Hk, dh, n):
    rng, q, k, v = make(n + dh, dtype, B, H, Hk, dh, n, n, size=3.0 if mode in ("cap", "both") else 1.0)
    kw = {}
    if mode in ("cap", "both"):
        kw["cap"] = 5.0
    if mode in ("bias", "both"):
        kw["slopes"] = np.exp2(-rng.uniform(0, 8, H))
    cuts = [[0] + sorted(rng.integers(0, n + 1, 3).tolist()) + [n - b if n > b else n] for b in range(B)]
    cuts = [sorted(min(x, c[-1]) for x in c) for c in cuts]
    check(P, q, k, v, documents(B, n, cuts), dtype, **kw)
    lens = [max(1, n - 5 * b) for b in range(B)]
    r = causal(B, n, n, [n] * B, prefix=n // 3)
    for b in range(B):
        r[b, :, 1] = np.minimum(r[b, :, 1], lens[b])
        r[b, lens[b]:] = 0  # padding: its queries see nothing
    o, ref = check(P, q, k, v, r, dtype, **kw)
    for b in range(B):
        assert (f64(o)[b, lens[b]:] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hk,dh,nq,nk", [(1, 1, 1, 64, 1, 1), (2, 8, 2, 128, 1, 900), (1, 32, 1, 128, 1, 4100), (3, 4, 4, 72, 4, 2000),
                                             (1, 2, 1, 128, 16, 5000), (1, 8, 1, 64, 5, 3000), (2, 4, 1, 96, 9, 1500)])
@pytest.mark.parametrize("mode", ["plain", "both"])
def test_single_tokens(P, dtype, mode, B, H, Hk, dh, nq, nk):
    """Few query rows over long caches of different lengths: keys split between waves and workgroups."""
    rng, q, k, v = make(nk + nq, dtype, B, H, Hk, dh, nq, nk)
    lens = [max(nq, nk - 301 * b) for b in range(B)]
    kw = {} if mode == "plain" else dict(cap=20.0, slopes=np.exp2(-8.0 * np.arange(1, H + 1) / H),
                                         pos=np.array([[l - nq + i for i in range(nq)] for l in lens]))
    r = causal(B, nq, nk, lens)
    if B > 2:
        r[2] = 0  # a sample without a cache
    check(P, q, k, v, r, dtype, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq", [3, 150])
def test_any_intervals(P, dtype, nq):
    """Windows, empty, reversed and out-of-range intervals in one block of rows."""
    rng, q, k, v = make(nq, dtype, 1, 2, 1, 64, nq, 400)
    lo = rng.integers(-50, 420, (1, nq, 1))
    r = np.concatenate([lo, lo + rng.integers(-20, 200, (1, nq, 1))], -1)
    r[0, 0] = (-(1 << 31), (1 << 31) - 1)
    r[0, 1] = (399, 400)
    r[0, 2] = (10, 10)
    check(P, q, k, v, r, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nk", [(2, 200), (2, 1500), (140, 200)])
def test_bad_values_stay_with_those_who_see_them(P, dtype, nq, nk):
    """Infinities and NaN among keys and values of one document do not reach another's queries, nor do those past
    every interval; who sees them gets them."""
    import torch
    rng, q, k, v = make(nq * nk, dtype, 1, 2, 2, 64, nq, nk)
    cut = 75
    r = np.zeros((1, nq, 2), np.int64)
    r[0, :nq // 2] = (0, cut)
    r[0, nq // 2:] = (cut, nk - 10)
    v[0, nk - 10:] = float("nan")
    k[0, nk - 5:] = float("inf")
    o, ref = check(P, q, k, v, r, dtype)
    assert np.isfinite(ref).all()
    v[0, cut - 3, 0, 5] = float("inf")
    v[0, cut - 2, 0, 6] = float("-inf")
    v[0, cut - 3, 1, 7] = float("nan")
    v[0, cut - 4, 1, 8] = float("inf")
    v[0, cut - 5, 1, 8] = float("-inf")
    o, ref = check(P, q, k, v, r, dtype)
    assert np.isinf(ref[0, 0, 0, 5]) and np.isnan(ref[0, 0, 1, 7]) and np.isfinite(ref[0, nq // 2:]).all()
    k[0, cut - 1, 1] = float("nan")
    o, ref = check(P, q, k, v, r, dtype)
    assert np.isnan(ref[0, :nq // 2, 1]).all() and np.isfinite(ref[0, nq // 2:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layouts(P, dtype):
    """Head-major tensors, slices of a fused projection, an output inside a larger tensor; scale given."""
    import torch
    B, H, dh, n = 2, 3, 64, 90
    rng, q, k, v = make(9, dtype, B, H, H, dh, n, n)
    r = documents(B, n, [[0, 20, n], [0, 50, n]])
    base, _ = check(P, q, k, v, r, dtype, scale=0.3)
    heads = [t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for t in (q, k, v)]
    big = torch.full((B, n, H, dh + 16), 7.0, dtype=q.dtype, device="cuda")
    o, _ = check(P, *heads, r, dtype, scale=0.3, o=big[..., 8:8 + dh])
    assert torch.equal(o, base) and (big[..., :8] == 7).all() and (big[..., 8 + dh:] == 7).all()
    fused = torch.cat([q, k, v], 2)  # [B, n, 3 H, dh]
    o, _ = check(P, fused[:, :, :H], fused[:, :, H:2 * H], fused[:, :, 2 * H:], r, dtype, scale=0.3)
    assert torch.equal(o, base)


def test_far_keys(P):
    """A cache whose last keys lie past 2^32 bytes from its first."""
    import torch
    if torch.cuda.get_device_properties(0).total_memory < 40e9:
        pytest.skip("needs 20 GB")
    nk, Hk, dh = 600, 1, 64
    stride = 4 << 20  # elements a token: 8 MiB
    buf = torch.empty(nk * stride, dtype=torch.bfloat16, device="cuda")
    view = buf.view(1, nk, stride)
    rng, q, k, v = make(1, "bf16", 1, 2, Hk, dh, 1, nk)
    far_k, far_v = view[:, :, :dh].unsqueeze(2), view[:, :, 1024:1024 + dh].unsqueeze(2)
    far_k.copy_(k)
    far_v.copy_(v)
    r = np.array([[[300, nk]]])
    o, _ = check(P, q, far_k, far_v, r, "bf16")
    q2 = q.expand(1, 1, 2, dh).repeat(1, 40, 1, 1)  # many rows: the other kernel
    check(P, q2, far_k, far_v, np.repeat(r, 40, 1), "bf16")
    del buf, view, far_k, far_v


def test_streams_workspace_and_graph(P):
    """A stream of its own, a caller's workspace, and a captured call replayed between eager ones."""
    import torch
    rng, q, k, v = make(3, "bf16", 2, 8, 2, 128, 1, 4096)
    r = torch.tensor([[[0, 4096]], [[100, 3000]]], dtype=torch.int32, device="cuda")
    base = torch.empty_like(q)
    P.op_attention_ranges(q, k, v, base, r)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    o = torch.empty_like(q)
    P.op_attention_ranges(q, k, v, o, r, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(o, base)
    ws = torch.full((64 << 20,), 0xFF, dtype=torch.uint8, device="cuda")
    P.op_attention_ranges(q, k, v, o, r, workspace=ws)
    assert torch.equal(o, base)
    with pytest.raises(P.SgdError):
        P.op_attention_ranges(q, k, v, o, r, workspace=ws[:64])
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=st):
        P.op_attention_ranges(q, k, v, o, r, workspace=ws)
    for s in range(3):
        q.copy_(torch.from_numpy(rng.standard_normal(q.shape).astype(np.float32)))
        o.zero_()
        g.replay()
        P.op_attention_ranges(q, k, v, base, r)
        torch.cuda.synchronize()
        assert torch.equal(o, base)


def test_binding_refuses(P):
    import torch
    rng, q, k, v = make(0, "bf16", 1, 2, 2, 64, 4, 8)
    r = torch.zeros(1, 4, 2, dtype=torch.int32, device="cuda")
    o = torch.empty_like(q)
    for bad in (dict(k=k.float()), dict(v=v[:, :4]), dict(o=o.float()), dict(r=r.long()), dict(r=r[:, :2]), dict(q=q[..., ::2].repeat(1, 1, 1, 2)[..., ::2])):
        a = dict(q=q, k=k, v=v, o=o, r=r)
        a.update(bad)
        with pytest.raises(ValueError):
            P.op_attention_ranges(a["q"], a["k"], a["v"], a["o"], a["r"])
    with pytest.raises(ValueError):
        P.op_attention_ranges(q, k, v, o, r, slopes=torch.zeros(3, device="cuda"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,H,Hk", [(1, 4, 2), (160, 2, 2)])
def test_positions_far_from_their_keys(P, dtype, nq, H, Hk):
    """A query past (or before) every key that it sees: the bias differs between keys only by their own distances, so the
    error bound has those and not the position.  Positions up to the ends of int32."""
    import torch
    nk, dh = 300, 64
    rng, q, k, v = make(nq, dtype, 1, H, Hk, dh, nq, nk)
    slopes = np.exp2(-np.arange(1, H + 1, dtype=np.float64))
    lo = rng.integers(0, 200, (1, nq, 1))
    r = np.concatenate([lo, lo + rng.integers(1, 100, (1, nq, 1))], -1)
    far = np.array([(1 << 31) - 1, -(1 << 31), 10 ** 6, 1 << 24, -12345, 310])
    pos = far[np.arange(nq) % len(far)][None]
    for first in range(len(far) if nq == 1 else 1):
        p = far[first:first + 1][None] if nq == 1 else pos
        o = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
        P.op_attention_ranges(q, k, v, o, torch.from_numpy(r.astype(np.int32)).cuda(), slopes=torch.from_numpy(slopes.astype(np.float32)).cuda(),
                              pos=torch.from_numpy(p.astype(np.int32)).cuda())
        near = np.clip(p, r[..., 0], r[..., 1] - 1)
        ref, mag = R.attention(f64(q), f64(k), f64(v), r, dh ** -0.5, 0.0, slopes, p)
        same, _ = R.attention(f64(q), f64(k), f64(v), r, dh ** -0.5, 0.0, slopes, near)
        assert np.abs(ref - same).max() < 1e-5  # float64 at a distance of 2^31: scores off by 2^-23
        big = dh ** -0.5 * np.linalg.norm(f64(q), axis=-1).max() * np.linalg.norm(f64(k), axis=-1).max()
        err = 2 * ((dh + 8) * 2.0 ** -24 * big + 2.0 ** -21 * (big + slopes.max() * 100))
        half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
        tol = half * np.abs(same) + ((half if dtype == "bf16" else 0) + 2 * err + (nk + 64) * 2.0 ** -24) * mag
        assert (np.abs(f64(o) - same) <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_and_small_caps(P, dtype):
    """A cap far above the scores changes nothing; bf16's form of it is off by some 2^-22 of the cap."""
    rng, q, k, v = make(5, dtype, 1, 2, 1, 128, 70, 200)
    r = documents(1, 70, [[0, 70]])
    r[0, :, 1] = 200
    for cap in (1024.0, 1e-3) + ((1e7,) if dtype == "f32" else ()):
        import torch
        o = torch.empty_like(q)
        P.op_attention_ranges(q, k, v, o, torch.from_numpy(r.astype(np.int32)).cuda(), cap=cap)
        ref, mag = R.attention(f64(q), f64(k), f64(v), r, 128 ** -0.5, cap, None, None)
        big = 128 ** -0.5 * np.linalg.norm(f64(q), axis=-1).max() * np.linalg.norm(f64(k), axis=-1).max()
        err = 2 * (136 * 2.0 ** -24 * big + 2.0 ** -21 * min(big, cap) + (2.0 ** -22 * cap if dtype == "bf16" else 0))
        half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
        tol = half * np.abs(ref) + ((half if dtype == "bf16" else 0) + 2 * err + 264 * 2.0 ** -24) * mag
        assert (np.abs(f64(o) - ref) <= tol).all(), (cap, float((np.abs(f64(o) - ref) / tol).max()))


def test_binding_refuses_zero_scale_and_foreign_streams(P):
    import types
    rng, q, k, v = make(0, "bf16", 1, 2, 2, 64, 4, 8)
    import torch
    r, o = torch.zeros(1, 4, 2, dtype=torch.int32, device="cuda"), torch.empty_like(q)
    with pytest.raises(ValueError):
        P.op_attention_ranges(q, k, v, o, r, scale=0.0)
    with pytest.raises(ValueError):
        P.op_attention_ranges(q, k, v, o, r, stream=types.SimpleNamespace(cuda_stream=0, device_index=1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mode", ["plain", "cap", "bias", "both"])
@pytest.mark.parametrize("B,H,Hk,dh,n", [(5, 52, 52, 64, 45), (4, 52, 26, 56, 75), (2, 26, 26, 128, 150), (1, 104, 104, 40, 131), (3, 44, 44, 96, 33)])
def test_many_heads(P, dtype, mode, B, H, Hk, dh, n):
    """Enough rows and heads for row blocks of 128 in either type; prefixes and packed documents in which rows end."""
    rng, q, k, v = make(n * dh, dtype, B, H, Hk, dh, n, n, size=3.0 if mode in ("cap", "both") else 1.0)
    kw = {}
    if mode in ("cap", "both"):
        kw["cap"] = 5.0
    if mode in ("bias", "both"):
        kw["slopes"] = np.exp2(-rng.uniform(0, 8, H))
    r = causal(B, n, n, [n] * B, prefix=n // 3)
    for b in range(B):
        r[b, n - b:] = 0
    r[0, :, :] = documents(1, n, [[0, n // 4, n // 2, n - 3]])[0]
    o, _ = check(P, q, k, v, r, dtype, **kw)
    for b in range(1, B):
        assert (f64(o)[b, n - b:] == 0).all()
    assert (f64(o)[0, n - 3:] == 0).all()


@pytest.mark.parametrize("dtype,H,dh", [("bf16", 104, 64), ("bf16", 64, 128), ("f32", 104, 64), ("f32", 52, 128)])
def test_bad_values_under_many_heads(P, dtype, H, dh):
    """As above in row blocks of 128: infinities and NaN reach the rows that see them, in their head."""
    nq, nk, cut = 140, 200, 75
    rng, q, k, v = make(H, dtype, 1, H, H, dh, nq, nk)
    r = np.zeros((1, nq, 2), np.int64)
    r[0, :nq // 2] = (0, cut)
    r[0, nq // 2:] = (cut, nk - 10)
    v[0, nk - 10:] = float("nan")
    k[0, nk - 5:] = float("inf")
    v[0, cut - 3, 0, 5] = float("inf")
    v[0, cut - 2, 0, 6] = float("-inf")
    v[0, cut - 3, 1, 7] = float("nan")
    v[0, cut - 4, 1, 8] = float("inf")
    v[0, cut - 5, 1, 8] = float("-inf")
    k[0, cut - 1, H - 1] = float("nan")
    o, ref = check(P, q, k, v, r, dtype)
    assert np.isinf(ref[0, 0, 0, 5]) and np.isnan(ref[0, 0, 1, 7]) and np.isnan(ref[0, :nq // 2, H - 1]).all()
    assert np.isfinite(ref[0, nq // 2:]).all() and np.isfinite(ref[0, :, 2:H - 1]).all()


def test_far_keys_in_row_blocks_of_128(P):
    """A cache whose last keys lie past 2^32 bytes from its first, many rows of many heads."""
    import torch
    if torch.cuda.get_device_properties(0).total_memory < 40e9:
        pytest.skip("needs 20 GB")
    nk, H, dh, nq = 600, 130, 64, 100
    stride = 4 << 20
    buf = torch.empty(nk * stride, dtype=torch.bfloat16, device="cuda")
    view = buf.view(1, nk, stride)
    rng, q, k, v = make(2, "bf16", 1, H, H, dh, nq, nk)
    far_k, far_v = view[:, :, :H * dh].view(1, nk, H, dh), view[:, :, 16384:16384 + H * dh].view(1, nk, H, dh)
    far_k.copy_(k)
    far_v.copy_(v)
    r = np.zeros((1, nq, 2), np.int64)
    r[0, :, 0] = 560 - np.arange(nq)
    r[0, :, 1] = nk
    base, _ = check(P, q, k, v, r, "bf16")
    o = torch.empty_like(q)
    P.op_attention_ranges(q, far_k, far_v, o, torch.from_numpy(r.astype(np.int32)).cuda())
    assert torch.equal(o, base)
    del buf, view, far_k, far_v


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk,dh,nq,nk", [(16, 16, 128, 257, 1024), (8, 2, 128, 515, 2048), (8, 8, 72, 520, 1100)])
def test_splits_of_many_rows(P, dtype, H, Hk, dh, nq, nk):
    """Thousands of query rows whose keys are split between workgroups, some rows seeing nothing or one split's keys only."""
    rng, q, k, v = make(nq + dh, dtype, 1, H, Hk, dh, nq, nk)
    r = causal(1, nq, nk, [nk])
    r[0, ::7, 0] = np.maximum(r[0, ::7, 1] - 40, 0)
    r[0, ::11] = 0
    o, _ = check(P, q, k, v, r, dtype)
    assert (f64(o)[0, ::11] == 0).all()


def test_calls_on_two_streams_with_their_own_workspaces(P, monkeypatch):
    """Calls that split their keys, on the current stream and on another one with no wait between them: the workspaces that
    they make are different blocks, and every result has the bits of the call alone."""
    import torch
    from paper_2609_29505_amd import binding
    made = []
    make_one = binding._workspace

    def noted(*args):
        made.append(make_one(*args))
        return made[-1]

    st = torch.cuda.Stream()
    sets = []
    for i in range(2):
        rng, q, k, v = make(20 + i, "bf16", 1, 8, 2, 128, 1, 6000)
        r = torch.tensor([[[i, 6000 - 7 * i]]], dtype=torch.int32, device="cuda")
        alone = torch.empty_like(q)
        P.op_attention_ranges(q, k, v, alone, r)
        sets.append((q, k, v, r, alone))
    outs = [(torch.empty_like(s[0]), s[4]) for s in sets * 4]  # before the loop: none of them is a workspace's block
    torch.cuda.synchronize()
    monkeypatch.setattr(binding, "_workspace", noted)
    for n, (o, _) in enumerate(outs):
        q, k, v, r, _ = sets[n % 2]
        P.op_attention_ranges(q, k, v, o, r, stream=st if n % 2 else None)
        made[n] = made[n].data_ptr()  # the block goes back to its pool, as without this test
    torch.cuda.synchronize()
    assert not set(made[0::2]) & set(made[1::2])
    assert all(torch.equal(o, alone) for o, alone in outs)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("power", [-100, 100])
def test_far_scales_and_caps(P, dtype, power):
    """Scores of ordinary size out of a scale far from one, and fp32's largest cap, which changes nothing."""
    B, H, dh, n = 1, 2, 64, 80
    rng, q, k, v = make(7, dtype, B, H, H, dh, n, n)
    q, k = q * 2.0 ** (-power // 2), k * 2.0 ** (-power // 2)
    r = causal(B, n, n, [n])
    check(P, q, k, v, r, dtype, scale=2.0 ** power / 8)
    check(P, q, k, v, r, dtype, scale=2.0 ** power / 8, cap=20.0)
    if dtype == "f32" and power > 0:
        check(P, q, k, v, r, dtype, scale=2.0 ** power / 8, cap=2.0 ** 126)
