"""Plain float64 definitions of the operators on microscaled rows, rotary positions and key intervals
(numpy), written apart from the kernels."""
import numpy as np

FP4 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
FP8 = np.array([m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)][:-1])
GRID = {"fp4": FP4, "fp8": FP8}
EMAX = {"fp4": 2, "fp8": 8}


def blocks(x):
    return np.asarray(x, np.float64).reshape(x.shape[0], -1, 32)


def scale_bytes(x, fmt):
    """Scale byte of every 32-column block: [rows, K / 32]."""
    big = np.abs(blocks(x)).max(-1)
    bad = ~np.isfinite(big)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.frexp(np.where(bad, 1.0, big))[1] - 1  # floor(log2)
    e = np.where(big == 0, -200, e)
    return np.where(bad, 255, np.maximum(e - EMAX[fmt], -127) + 127).astype(np.int64)


def nearest(y, fmt):
    """Index of the nearest value of the format (ties to the even code, saturating) for y >= 0."""
    g = GRID[fmt]
    up = np.minimum(np.searchsorted(g, y), len(g) - 1)
    dn = np.maximum(up - 1, 0)
    mid = (g[up] + g[dn]) / 2
    return np.where((y > mid) | ((y == mid) & (up % 2 == 0)) | (y >= g[up]), up, dn)


def quantize(x, fmt):
    """(codes per value incl. sign [rows, K], scale bytes [rows, K / 32])."""
    s = scale_bytes(x, fmt)
    with np.errstate(invalid="ignore"):
        y = np.where(s[..., None] == 255, 0.0, blocks(x) * np.exp2(127.0 - s)[..., None])
    sign = np.where(np.signbit(y), 8 if fmt == "fp4" else 128, 0)
    return (nearest(np.abs(y), fmt) + sign).reshape(x.shape), s


def pack_codes(c, fmt):
    return c.astype(np.uint8) if fmt == "fp8" else (c[:, 0::2] | (c[:, 1::2] << 4)).astype(np.uint8)


def pack_scales(s):
    """[rows, K / 32] -> [ceil(K / 256), rows, 8], zeros past the last block."""
    rows, nb = s.shape
    full = np.zeros((rows, -(-nb // 8) * 8), np.uint8)
    full[:, :nb] = s
    return np.ascontiguousarray(full.reshape(rows, -1, 8).transpose(1, 0, 2))


def decode(codes, scales, fmt):
    """Values of packed codes and scales, float64."""
    if fmt == "fp8":
        c = codes.astype(np.int64)
        v = np.where(c > 127, -1.0, 1.0) * np.append(FP8, np.nan)[c & 127]
    else:
        c = np.empty((codes.shape[0], codes.shape[1] * 2), np.int64)
        c[:, 0::2], c[:, 1::2] = codes & 15, codes >> 4
        v = np.where(c > 7, -1.0, 1.0) * FP4[c & 7]
    rows, K = v.shape
    s = scales.transpose(1, 0, 2).reshape(rows, -1)[:, :K // 32].astype(np.float64)
    f = np.where(s == 255, np.nan, np.exp2(s - 127))
    return (v.reshape(rows, -1, 32) * f[..., None]).reshape(rows, K)


def block_max(v):
    return np.abs(v).reshape(v.shape[0], -1, 32).max(-1)


def act(z, kind):
    from oracle import model as om
    return {0: lambda t: t, 1: om.gelu_erf, 2: om.gelu_tanh, 3: om.silu}[kind](z)


def norm(h, w, eps):
    return h / np.sqrt((h * h).mean(-1, keepdims=True) + eps) * w


def rotate(x, pos, turns, rot, interleaved, magnitude=1.0, inverse=False):
    x = np.array(x, np.float64)
    a = 2 * np.pi * np.mod(np.asarray(pos, np.float64)[:, None] * turns[None], 1.0) * (-1 if inverse else 1)
    f = (magnitude * np.exp(1j * a))[:, None]
    i = np.arange(rot // 2)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    z = (x[..., first] + 1j * x[..., second]) * f
    x[..., first], x[..., second] = z.real, z.imag
    return x


def attention(q, k, v, ranges, scale, cap=0.0, slopes=None, pos=None):
    """(o, sum p |v| / sum p, largest score error factor) for q [B, nq, H, dh], k, v [B, nk, Hk, dh]."""
    B, nq, H, dh = q.shape
    nk, G = k.shape[1], H // k.shape[2]
    o = np.zeros(q.shape)
    mag = np.zeros(q.shape)
    j = np.arange(nk)
    for b in range(B):
        lo, hi = ranges[b, :, 0:1], ranges[b, :, 1:2]
        see = (j >= lo) & (j < hi)
        for h in range(H):
            z = q[b, :, h] @ k[b, :, h // G].T * scale
            if cap:
                z = cap * np.tanh(z / cap)
            if slopes is not None:
                p = pos[b] if pos is not None else np.arange(nq) + nk - nq
                z = z - slopes[h] * np.abs(p[:, None] - j)
            for i in range(nq):
                s = see[i]
                if not s.any():
                    continue
                with np.errstate(invalid="ignore", over="ignore"):
                    e = np.exp(z[i, s] - z[i, s].max())
                    o[b, i, h] = e @ v[b, s, h // G] / e.sum()
                    mag[b, i, h] = e @ np.abs(v[b, s, h // G]) / e.sum()
    return o, mag
