"""64-bit references of the 8-bit products, the expert layer over them and the norms around a block, with
bounds on what the kernels may be off by.  numpy on the CPU; shares no code with the library.

Bounds, element by element.  A sum of code products is exact; turned into fp32 (half a step, 2^-24 relative) and
multiplied with two scales (2^-24 each) it is off by PRODUCT = 3 * 2^-24 (plus second order, covered by 3.1), and a
result in bf16 by another half step, 2^-8.  h = silu(a)*b of such a and b: e^-a is off by |a| times the relative
errors of a and of a*log2(e) (4 * 2^-24) and two steps of the exponential (2^-22), silu by as much and a sum and a division,
and two products follow: RH(a) = (4.1 |a| + 4 + 2 + 3.1 * 2.1 + 4) * 2^-24, rounded up to (5 |a| + 20) * 2^-24.  A row's
scale is off by what its largest magnitude is (and half a step for the division), and a quotient h / scale by both: where that
reaches a border between two codes (an integer and a half), the code may be either, one step apart."""
import numpy as np

PRODUCT = 3.1 * 2.0 ** -24
BF16 = 2.0 ** -8


def bf16(a):
    """fp32 values rounded to bf16 (nearest, ties to even), as fp32."""
    u = np.asarray(a, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32)


def quantize(v):
    """v [..., K] -> codes int8 [..., K], scales fp32 [...]."""
    v = np.asarray(v)
    top = np.abs(v).max(axis=-1)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        s = (top / np.float32(127)).astype(np.float32) if v.dtype == np.float32 else (top / 127).astype(np.float32)
        s = np.where(np.isfinite(v).all(axis=-1), s, np.float32(np.nan)).astype(np.float32)
        z = v.astype(np.float64) / s.astype(np.float64)[..., None]
    q = np.where((s > 0)[..., None], np.clip(np.rint(z), -127, 127), 0.0)
    return q.astype(np.int8), s


def matrix(w):
    """W [E,K,C] -> codes [E,C,K], scales [E,C]."""
    return quantize(np.ascontiguousarray(np.asarray(w, dtype=np.float32).transpose(0, 2, 1)))


def product(q, s, codes, scales):
    """q [M,K], s [M], codes [C,K], scales [C] -> fp64 [M,C]: the sum of codes exactly (fp64 holds it)."""
    return (q.astype(np.float64) @ codes.astype(np.float64).T) * s.astype(np.float64)[:, None] * scales.astype(np.float64)


def expert(q, s, w1, w3, w2):
    """One expert's rows in 8 bits -> (y, bound) fp64 [M,d]."""
    a, b = product(q, s, *w1), product(q, s, *w3)
    h = a / (1 + np.exp(-a)) * b
    dh = (5 * np.abs(a) + 20) * 2.0 ** -24 * np.abs(h)
    top = np.abs(h).max(axis=-1)
    sh = (top / 127).astype(np.float32).astype(np.float64)
    off = (dh + 2.0 ** -24 * np.abs(h)).max(axis=-1) / np.where(top > 0, top, 1) + 2.0 ** -23   # of the scale, relative
    z = h / np.where(sh > 0, sh, 1)[:, None]
    near = np.abs(z) * off[:, None] + dh / np.where(sh > 0, sh, 1)[:, None]
    either = np.abs(np.abs(z) - np.floor(np.abs(z)) - 0.5) <= near
    hq = np.clip(np.rint(z), -127, 127)
    w = w2[0].astype(np.float64).T * w2[1].astype(np.float64)
    y = (hq * sh[:, None]) @ w
    bound = (either * sh[:, None]) @ np.abs(w) + (off[:, None] + PRODUCT) * (np.abs(hq * sh[:, None]) @ np.abs(w))
    return y, bound


def route(logits, k):
    lg = np.asarray(logits, dtype=np.float64)
    idx = np.argsort(-lg, axis=1, kind="stable")[:, :k]
    u = np.exp(np.take_along_axis(lg, idx, 1) - np.take_along_axis(lg, idx[:, :1], 1))
    return idx.astype(np.int32), u / u.sum(axis=1, keepdims=True)


def layer(q, s, logits, k, mats, out_bf16):
    """-> (idx, gate weights, y, bound)."""
    idx, w = route(logits, k)
    y, bound = np.zeros(q.shape), np.zeros(q.shape)
    for e in range(mats[0][0].shape[0]):
        tok, slot = np.nonzero(idx == e)
        if tok.size:
            ye, be = expert(q[tok], s[tok], *((c[e], t[e]) for c, t in mats))
            wt = w[tok, slot][:, None]
            np.add.at(y, tok, wt * ye)
            # the gate weight (1e-6 absolute, the layer's own contract), its product and the sum over the slots
            np.add.at(bound, tok, wt * be + (1e-6 + (k + 1) * 2.0 ** -24) * np.abs(ye))
    return idx, w, y, bound + (BF16 if out_bf16 else 2.0 ** -24) * (np.abs(y) + bound)


def block_norm(x, y, norm_after, gain_after, gate, row_gate, scale, gain_before, eps):
    """fp64 (x', h); None for a gain or gate of ones."""
    f = lambda v, n: np.ones(n) if v is None else np.asarray(v, dtype=np.float64)  # noqa: E731
    x = np.asarray(x, dtype=np.float64)
    T, d = x.shape
    if y is not None:
        u = np.asarray(y, dtype=np.float64)
        if norm_after:
            u = u / np.sqrt((u * u).mean(axis=1, keepdims=True) + float(np.float32(eps))) * f(gain_after, d)
        x = x + float(np.float32(scale)) * f(row_gate, T)[:, None] * f(gate, d) * u
    h = x / np.sqrt((x * x).mean(axis=1, keepdims=True) + float(np.float32(eps))) * f(gain_before, d)
    return x, h
