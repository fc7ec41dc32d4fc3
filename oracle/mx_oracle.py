"""Plain fp64 definition of the microscaled 4-bit format, its grouped product and FFN, and of the whole layer for a few tokens, with bounds of what
fp32 arithmetic may make of them (test infrastructure: NumPy only, nothing shared with the HIP path)."""
from __future__ import annotations

import numpy as np

CODES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
U32 = 2.0 ** -24          # unit roundoff of fp32
UBF16 = 2.0 ** -8         # ... and of bf16, with its 8 significant bits, doubled: a rounding may start from either side of a tie
EXP = 2.0 ** -20          # relative error of the sigmoid's exponential and quotient for g > -5, with room


def silu_error(g):
    """Relative error of silu(g) in fp32: far below zero that of the exponential, 2^t of a rounded t = -g log2 e (|g| 2^-24, and a quarter of that for log2 e)."""
    return np.maximum(EXP, (8 - 1.5 * np.minimum(g, 0)) * U32)


def scale_codes(blocks):
    """[..., 32] -> scale codes: clamp(floor(log2 max) - 2, -127, 127) + 127; 0 of zeros; 255 where something is not finite."""
    top = np.abs(blocks).max(-1)
    bad = ~np.isfinite(top)
    safe = np.where(bad | (top == 0), 1.0, top)
    e = np.frexp(safe)[1] - 1
    s = np.clip(e - 2, -127, 127) + 127
    return np.where(bad, 255, np.where(top == 0, 0, s)).astype(np.int64)


def encode(blocks, s):
    """Codes (0 .. 15) of [..., 32] at scale codes s [...]: the nearest, ties to the even code, the sign bit on top."""
    scale = np.exp2(np.where(s == 255, 0, s - 127.0))[..., None]
    with np.errstate(invalid="ignore"):
        a = np.abs(blocks) / scale
    a = np.where(np.isfinite(a), a, 0.0)
    dist = np.abs(a[..., None] - CODES)
    near = dist.min(-1, keepdims=True) == dist
    lo = near.argmax(-1)
    hi = 7 - near[..., ::-1].argmax(-1)
    code = np.where(lo % 2 == 0, lo, hi)
    code = np.where(s[..., None] == 255, 0, code + 8 * np.signbit(blocks))
    return code.astype(np.uint8)


def decode(codes, s):
    v = np.where(codes & 8, -1.0, 1.0) * CODES[codes & 7]
    scale = np.where(s == 255, np.nan, np.exp2(np.where(s == 255, 0, s - 127.0)))
    return v * scale[..., None]


def quantize(x):
    """x [..., K] -> (q [..., K/2] uint8, scales [..., K/32] uint8)."""
    b = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 32)
    s = scale_codes(b)
    c = encode(b, s).reshape(x.shape)
    return (c[..., 0::2] | (c[..., 1::2] << 4)).astype(np.uint8), s.astype(np.uint8)


def dequantize(q, scales):
    c = np.stack([q & 15, q >> 4], -1).reshape(*scales.shape, 32)
    return decode(c, scales.astype(np.int64)).reshape(*q.shape[:-1], 2 * q.shape[-1])


def _segments(offsets):
    return [(e, int(a), int(b)) for e, (a, b) in enumerate(zip(offsets[:-1], offsets[1:])) if b > a]


def grouped_gemm(x, w, offsets):
    """x [N, K], w [E, C, K] (values) -> (y, how far fp32 sums and one bf16 rounding may be off)."""
    y, q = np.zeros((x.shape[0], w.shape[1])), np.zeros((x.shape[0], w.shape[1]))
    for e, a, b in _segments(offsets):
        y[a:b] = x[a:b] @ w[e].T
        q[a:b] = np.abs(x[a:b]) @ np.abs(w[e]).T
    return y, UBF16 * np.abs(y) + (x.shape[1] + 8) * U32 * q + 1e-38


def swiglu(x, wg, wu):
    """x [n, K], wg, wu [K, C] -> (H, bound of what fp32 sums make of it)."""
    g, u = x @ wg, x @ wu
    n = (x.shape[1] + 8) * U32
    dg, du = n * (np.abs(x) @ np.abs(wg)), n * (np.abs(x) @ np.abs(wu))
    s = g / (1 + np.exp(-np.clip(g, -700, None)))
    h = s * u
    return h, 1.1 * dg * np.abs(u) + np.abs(s) * du + 1.1 * dg * du + silu_error(g) * np.abs(h)


def quantized_spread(h, dh):
    """Values of Q(h), and how far Q of anything within dh of h may be from them (a value or a block's largest may lie on a rounding boundary)."""
    hb, db = h.reshape(h.shape[0], -1, 32), dh.reshape(h.shape[0], -1, 32)
    top = np.abs(hb).max(-1)
    room = db.max(-1)
    every = []
    for t in (top, np.maximum(top - room, 0), top + room):
        s = scale_codes(t[..., None])
        for v in (hb, hb - db, hb + db):
            every.append(decode(encode(v, s), s))
    every = np.stack(every)
    far = np.maximum(every.max(0) - every[0], every[0] - every.min(0))
    return every[0].reshape(h.shape), far.reshape(h.shape)


def grouped_ffn(x, wg, wu, wd, offsets):
    """x [N, d] (before quantisation), wg, wu [E, f, d], wd [E, d, f] (values) -> (y, bound)."""
    xq = dequantize(*quantize(x))
    y, far = np.zeros_like(xq), np.zeros_like(xq)
    for e, a, b in _segments(offsets):
        h, dh = swiglu(xq[a:b], wg[e].T, wu[e].T)
        hq, spread = quantized_spread(h, dh)
        y[a:b] = hq @ wd[e].T
        far[a:b] = spread @ np.abs(wd[e]).T + (wd.shape[2] + 8) * U32 * (np.abs(hq) @ np.abs(wd[e]).T)
    return y, far + UBF16 * (np.abs(y) + far) + 1e-38


def layer_few(x, idx, w, wg, wu, wd):
    """x [T, d], idx, w [T, K'], wg, wu [E', d, f], wd [E', f, d] -> (out, bound): per token the plain definition.  The hidden activation is
    kept with 16 significant bits (2^-16 of it at most is lost), gate weights are within 1e-5."""
    out, far = np.zeros_like(x), np.zeros_like(x)
    for e in np.unique(idx):
        t, j = np.nonzero(idx == e)
        h, dh = swiglu(x[t], wg[e], wu[e])
        y = h @ wd[e]
        dy = (dh + 2.0 ** -16 * np.abs(h) + (wd.shape[1] + 64) * U32 * np.abs(h)) @ np.abs(wd[e])
        np.add.at(out, t, w[t, j][:, None] * y)
        np.add.at(far, t, w[t, j][:, None] * (dy + 1e-5 * np.abs(y)))
    return out, far + UBF16 * (np.abs(out) + far) + 1e-38
