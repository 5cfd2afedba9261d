"""fp32 attention over key intervals held to fp32's precision: a bound per query, key and dim that bf16 probabilities, bf16 values or a
cap of fewer bits break.  That they break it is shown on the CPU, with the mistake planted in the float64 reference."""
import numpy as np
import pytest

U = 2.0 ** -24  # half a step of fp32, relative
LAMBDA = 4.0    # n rounding errors of independent signs add up to at most this many times sqrt(n)

# name: B, H, Hk, dh, nq, nk, cap, bias.  The comments name the form of the kernel that a case reaches.
CASES = {
    "rows_of_32": (1, 4, 2, 64, 130, 130, 0.0, False),        # 32 rows a workgroup
    "rows_of_32_cap": (1, 4, 4, 96, 257, 257, 20000.0, False),
    "rows_of_32_both": (2, 2, 2, 128, 300, 300, 30.0, True),
    "rows_of_128": (1, 16, 16, 128, 520, 520, 0.0, False),    # a wave's 32 of 128 rows
    "rows_of_128_cap": (1, 104, 104, 40, 131, 131, 20000.0, False),
    "rows_of_128_both": (1, 16, 16, 128, 520, 520, 300.0, True),
    "token": (2, 8, 2, 128, 1, 4100, 0.0, False),             # keys split between workgroups
    "token_cap": (1, 8, 8, 72, 2, 2000, 20000.0, True),
}


def make(name):
    """q, k, v (fp32), ranges, slopes: scores of ordinary size, causal with a prefix, some rows with a window, one empty."""
    B, H, Hk, dh, nq, nk, cap, bias = CASES[name]
    rng = np.random.default_rng(len(name) + dh + nk)
    q = (0.5 * rng.standard_normal((B, nq, H, dh))).astype(np.float32)
    k, v = (rng.standard_normal((B, nk, Hk, dh)).astype(np.float32) for _ in range(2))
    r = np.zeros((B, nq, 2), np.int32)
    r[..., 1] = np.minimum(np.maximum(np.arange(nq) + nk - nq + 1, nk // 2), nk)
    if nq > 100:
        r[:, ::9, 0] = r[:, ::9, 1] - 40
        r[:, 50] = 0
    slopes = np.exp2(-4.0 - 4.0 * rng.random(H)).astype(np.float32) if bias else None
    return q, k, v, r, slopes, cap


def to_bf16(x):
    """Rounded to bf16, ties to even."""
    b = np.asarray(x, np.float32).view(np.uint32)
    b = (b + 0x7FFF + ((b >> 16) & 1)) & np.uint32(0xFFFF0000)
    return b.view(np.float32).astype(np.float64)


def reference(q, k, v, r, slopes, cap, plant=None):
    """(o, bound) in float64.  plant: "p" and "v" round probabilities and values to bf16, "cap" takes cap tanh(x / cap) as
    cap - 2 cap / (1 + exp(2 x / cap)) with the quotient in fp32.

    The bound, per query i, key j, dim d.  A score is off by e: the chain of dh products and additions rounds 2 dh partial sums,
    LAMBDA sqrt(2 dh) U scale sum |q| |k|; its factors, the cap's argument and tanhf, the bias and the exponent's argument (with the
    maximum) are some ten roundings of the score's own parts, 16 U (|z| + |bias| + 1), the exponential's 2 U among them.
    A probability is then off by p e, in the output and in the divisor: sum p e (|v| + |o|).  The sums over nk
    keys round 2 nk partial sums (one more each for the joins): LAMBDA sqrt(2 nk + 64) U (sum p |v| + |o|).  And the output's own U."""
    B, nq, H, dh = q.shape
    nk, G = k.shape[1], H // k.shape[2]
    q, k, v = (t.astype(np.float64) for t in (q, k, v))
    scale = float(np.float32(1.0) / np.sqrt(np.float32(dh)))
    o, tol = np.zeros(q.shape), np.zeros(q.shape)
    j = np.arange(nk)
    for b in range(B):
        see = (j >= r[b, :, :1]) & (j < r[b, :, 1:])
        for h in range(H):
            kk, vv = k[b, :, h // G], v[b, :, h // G]
            if plant == "v":
                vv = to_bf16(vv)
            z = q[b, :, h] @ kk.T * scale
            e = LAMBDA * np.sqrt(2 * dh) * U * scale * (np.abs(q[b, :, h]) @ np.abs(kk).T)
            if cap and plant == "cap":
                z = cap - 2 * cap * (1 / (1 + np.exp(2 * z / cap))).astype(np.float32).astype(np.float64)
            elif cap:
                z = cap * np.tanh(z / cap)
            bias = 0.0 if slopes is None else float(slopes[h]) * np.abs(np.arange(nq)[:, None] + nk - nq - j)
            e = e + 16 * U * (np.abs(z) + bias + 1)
            z = np.where(see, z - bias, -np.inf)
            some = see.any(-1)
            p = np.exp(z - np.where(some, z.max(-1), 0.0)[:, None])
            div = np.where(some, p.sum(-1), 1.0)[:, None]
            if plant == "p":
                p = to_bf16(p)
            p = p / div
            o[b, :, h] = p @ vv
            mag, av = p @ np.abs(vv), np.abs(o[b, :, h])
            tol[b, :, h] = (p * e) @ np.abs(vv) + (p * e).sum(-1, keepdims=True) * av + LAMBDA * np.sqrt(2 * nk + 64) * U * (mag + av) + U * av
    return o, tol


@pytest.mark.parametrize("name", list(CASES))
def test_planted_losses_break_the_bound(name):
    """bf16 probabilities, bf16 values and the short cap each leave the bound, by a factor of two at least."""
    a = make(name)
    o, tol = reference(*a)
    for plant in ("p", "v") + (("cap",) if a[-1] >= 20000 else ()):
        bad, _ = reference(*a, plant=plant)
        with np.errstate(invalid="ignore"):
            assert np.nanmax(np.abs(bad - o) / tol) > 2, plant


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(CASES))
def test_fp32_attention_keeps_fp32(name):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_29505_amd as P
    q, k, v, r, slopes, cap = make(name)
    dev = lambda t: None if t is None else torch.from_numpy(t).cuda()  # noqa: E731
    out = torch.full(q.shape, 7.0, device="cuda")
    P.op_attention_ranges(dev(q), dev(k), dev(v), out, dev(r), cap=cap, slopes=dev(slopes))
    o, tol = reference(q, k, v, r, slopes, cap)
    off = np.abs(out.cpu().numpy() - o)
    print(name, "largest error", off.max(), "of its bound", float((off / np.where(tol > 0, tol, 1)).max()))
    assert (off <= tol).all()
