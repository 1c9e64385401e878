"""64-bit references of the 4-bit expert matrices and the layer over them, with bounds on what the
kernels may be off by.  numpy on the CPU; shares no code with the library.

Bounds, element by element.  A product a = x.W formed from exact 4-bit values is off by at most
`u` |x|.|W| for rows that are represented to a relative u, plus the roundings of its fp32 sum:
a matrix instruction adds 32 products to its accumulator, so a sum over K passes K/32 of them, each
off by at most one step (2^-23) of a partial sum, and 32 more sums join waves and parts.  With
g = silu(a) and |silu'| <= 1.1, h = g*b is off by 1.1 |da| |b| + |g| |db| + 2^-20 |h| (exp, a
division, two products in fp32); and the second product carries that on."""
import numpy as np

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=np.float64)


def bf16(a):
    """fp32 values rounded to bf16 (nearest, ties to even), as fp32."""
    u = np.asarray(a, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32)


def quantize(w):
    """w [E,K,C] -> codes [E,C,K/2], scales [E,C,K/32], by the distances to the eight magnitudes."""
    w = np.asarray(w, dtype=np.float64)
    E, K, C = w.shape
    b = np.ascontiguousarray(w.transpose(0, 2, 1)).reshape(E, C, K // 32, 32)
    top = np.abs(b).max(axis=3)
    ex = np.clip(np.frexp(np.where(top > 0, top, 1.0))[1] - 1 - 2, -126, 127)
    ex = np.where(top > 0, ex, -126)
    m = np.abs(b) / np.exp2(ex.astype(np.float64))[..., None]
    near = np.abs(m - VALUES[0])
    for c in range(1, 8):
        near = np.minimum(near, np.abs(m - VALUES[c]))
    code = np.zeros(m.shape, dtype=np.int64)
    for c in (7, 5, 3, 1, 6, 4, 2, 0):  # in a tie the even code is written last
        code = np.where(np.abs(m - VALUES[c]) <= near, c, code)
    code = (code + 8 * np.signbit(b)).reshape(E, C, K // 2, 2).astype(np.uint8)
    return code[..., 0] | (code[..., 1] << 4), (ex + 127).astype(np.uint8)


def dequantize(codes, scales):
    """-> fp64 [E,K,C]."""
    E, C, half = codes.shape
    v = np.stack([VALUES[codes & 15], VALUES[codes >> 4]], axis=-1).reshape(E, C, 2 * half // 32, 32)
    v = v * np.exp2(scales.astype(np.float64) - 127)[..., None]
    return v.reshape(E, C, 2 * half).transpose(0, 2, 1)


def silu(a):
    return a / (1 + np.exp(-a))


def expert(x, w1, w3, w2, u, uh):
    """One expert's rows and their bound: rows represented to u, h to uh."""
    def product(a, da, w, rel):
        K = w.shape[0]
        mag = np.abs(a) @ np.abs(w)
        return a @ w, (rel + (K / 32 + 32) * 2.0 ** -23) * mag + da @ np.abs(w)
    zero = np.zeros_like(x)
    a, da = product(x, zero, w1, u)
    b, db = product(x, zero, w3, u)
    g = silu(a)
    h = g * b
    dh = 1.1 * da * (np.abs(b) + db) + np.abs(g) * db + 2.0 ** -20 * np.abs(h)
    return product(h, dh * (1 + uh), w2, uh)


# what rows and h are held to: three bf16 parts (all 24 bits), two (half a step of half a step), one
SPLIT, PAIR, ROUND = 2.0 ** -24, 2.0 ** -16, 2.0 ** -8


def ffn(x, offsets, mats, u, uh):
    """Rows in expert order -> (yg, bound); rows of no expert stay zero."""
    yg = np.zeros((x.shape[0], mats[2].shape[2]))
    bound = np.zeros_like(yg)
    for e in range(len(offsets) - 1):
        lo, hi = offsets[e], offsets[e + 1]
        if hi > lo:
            yg[lo:hi], bound[lo:hi] = expert(x[lo:hi].astype(np.float64), mats[0][e], mats[1][e], mats[2][e], u, uh)
    return yg, bound


def route(logits, k):
    idx = np.argsort(-logits.astype(np.float64), axis=1, kind="stable")[:, :k]
    v = np.take_along_axis(logits.astype(np.float64), idx, axis=1)
    w = np.exp(v - v[:, :1])
    return idx.astype(np.int32), w / w.sum(axis=1, keepdims=True)


def batch(idx, E):
    flat = idx.reshape(-1)
    perm = np.argsort(flat, kind="stable").astype(np.int32)
    inv = np.empty_like(perm)
    inv[perm] = np.arange(len(perm), dtype=np.int32)
    counts = np.bincount(flat, minlength=E).astype(np.int32)
    return counts, np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), perm, inv


def layer(x, logits, mats, k, u, uh):
    """-> dict with the index outputs, w, y and y's bound (before y's own rounding).  The gate
    weights, off by at most 2^-20 relative (two exp, a sum, a division in fp32), count in it, and
    so do the k fp32 sums of the combine."""
    idx, w = route(logits, k)
    counts, offsets, perm, inv = batch(idx, logits.shape[1])
    yg, bg = ffn(x[perm // k], offsets, mats, u, uh)
    T, d = x.shape
    rows, brows = yg[inv].reshape(T, k, d), bg[inv].reshape(T, k, d)
    y = (rows * w[..., None]).sum(axis=1)
    bound = (brows * w[..., None]).sum(axis=1) + (2.0 ** -20 + k * 2.0 ** -23) * (np.abs(rows) * w[..., None]).sum(axis=1)
    return dict(idx=idx, w=w, counts=counts, offsets=offsets, perm=perm, inv_perm=inv, yg=yg, yg_bound=bg, y=y,
                bound=bound)


def matrices(seed, E, d, f):
    """Converted expert matrices ((codes, scales) of w1, w3, w2) and their 64-bit values."""
    rng = np.random.default_rng(seed)
    conv, vals = [], []
    for K, C in ((d, f), (d, f), (f, d)):
        codes = rng.integers(0, 256, size=(E, C, K // 2), dtype=np.uint8)
        # elements of variance 8.5 over the codes: unit-variance products, scales that differ
        top = 127 + int(np.round(-0.5 * np.log2(8.5 * K)))
        scales = rng.integers(top - 1, top + 2, size=(E, C, K // 32)).astype(np.uint8)
        conv.append((codes, scales))
        vals.append(dequantize(codes, scales))
    return conv, vals
