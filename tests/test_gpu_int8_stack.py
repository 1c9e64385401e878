"""A stack's block over 8-bit experts, held to a 64-bit reference through each of the stack's front ends.

Rows are integers in [-127, 127] with a 127 among them, times a constant, so that their norms' codes are these integers: a
quotient is off by 127 * DELTA < 0.01, half a code away from any border.  An expert whose matrices' scales are zero adds
nothing, so a block of such experts hands its rows on as they are and the seam's front end sees them too.

DELTA, of a normed row in fp32, relative: the sum of d squares (2^-24 each and d - 1 additions), the mean and eps, half of
it by the square root, then root, quotient and product (6 * 2^-24 with two steps for the root).  A logit is off by DELTA and
d + 2 roundings of sum |h||w|, a gate weight by twice that and 1e-6.  h = silu(a)*b of a and b that are off by DELTA each:
(2 + |a|) * DELTA on top of int8_ref's bound."""
import numpy as np
import pytest
import torch

import int8_ref as ref
from test_gpu_int8 import F32, _dev, _host, _mats, _pack, _rng, moe  # noqa: F401

pytestmark = pytest.mark.gpu

E, K, D, F, EPS = 8, 2, 256, 192, 1e-5
DELTA = ((D + 3) / 2 + 6) * 2.0 ** -24


def rows(rng, T):
    n = rng.integers(-127, 128, (T, D))
    n[np.arange(T), rng.integers(0, D, T)] = 127
    c = 2.0 ** rng.integers(-8, -4, T) * (1 + rng.integers(0, 8, T) / 8)
    return n, (n * c[:, None]).astype(np.float32)


def expert(n, s, w1, w3, w2):
    """int8_ref.expert for rows of codes n whose scales s (64 bits) are off by DELTA."""
    a, b = ref.product(n, s, *w1), ref.product(n, s, *w3)
    h = a / (1 + np.exp(-a)) * b
    dh = ((5 * np.abs(a) + 20) * 2.0 ** -24 + 1.01 * (2 + np.abs(a)) * (DELTA + 2.0 ** -24)) * np.abs(h)
    top = np.abs(h).max(axis=-1)
    sh = top / 127
    off = (dh + 2.0 ** -24 * np.abs(h)).max(axis=-1) / top + 2.0 ** -23
    z = h / sh[:, None]
    near = np.abs(z) * off[:, None] + dh / sh[:, None]
    either = np.abs(np.abs(z) - np.floor(np.abs(z)) - 0.5) <= near
    hq = np.clip(np.rint(z), -127, 127)
    w = w2[0].astype(np.float64).T * w2[1].astype(np.float64)
    return (hq * sh[:, None]) @ w, (either * sh[:, None]) @ np.abs(w) + (off[:, None] + ref.PRODUCT) * (np.abs(hq * sh[:, None]) @ np.abs(w))


def block(n, x, w_gate, mats):
    """x + the block's output, and its bound."""
    x = x.astype(np.float64)
    r = 1 / np.sqrt((x * x).mean(axis=1) + float(np.float32(EPS)))
    s = np.abs(x).max(axis=1) * r / 127
    h, wg = x * r[:, None], w_gate.astype(np.float64)
    logits = h @ wg
    dl = (DELTA + (D + 2) * 2.0 ** -24) * (np.abs(h) @ np.abs(wg)).max(axis=1)
    last = -np.sort(-logits, axis=1)
    assert ((last[:, K - 1] - last[:, K]) > 2 * dl).all() and ((last[:, 0] - last[:, 1]) > 2 * dl).all()  # the choice is clear
    idx, w = ref.route(logits, K)
    y, bound = np.zeros(x.shape), np.zeros(x.shape)
    for e in range(E):
        tok, slot = np.nonzero(idx == e)
        if tok.size:
            ye, be = expert(n[tok], s[tok], *((c[e], t[e]) for c, t in mats))
            wt = w[tok, slot][:, None]
            np.add.at(y, tok, wt * ye)
            np.add.at(bound, tok, wt * be + (wt * 2.02 * dl[tok][:, None] + 1e-6 + (K + 1) * 2.0 ** -24) * np.abs(ye))
    return idx, x + y, bound * 1.01 + 2.0 ** -24 * (np.abs(x) + np.abs(y))


def _case(T):
    rng = _rng(31, T)
    mats = _mats(rng, E, D, F)
    n, x = rows(rng, T)
    w_gate = (rng.standard_normal((D, E)) * D ** -0.5 * 3).astype(np.float32)
    return mats, n, x, w_gate


@pytest.mark.parametrize("T", [1, 3, 4, 5, 40])
@pytest.mark.parametrize("before", [0, 1, 2])
@pytest.mark.parametrize("seam", [True, False])
@pytest.mark.parametrize("fused", [True, False])
def test_block_of_a_stack(moe, T, before, seam, fused):  # noqa: F811
    """Behind `before` blocks that add nothing."""
    mats, n, x, w_gate = _case(T)
    idx, want, bound = block(n, x, w_gate, mats)
    none = _pack(moe, [(c, np.zeros_like(t)) for c, t in mats])
    layers = [(none, _dev(w_gate))] * before + [(_pack(moe, mats), _dev(w_gate))]
    chosen = []
    got = _host(moe.moe_stack_forward(layers, _dev(x), K, eps=EPS, fused=fused, seam=seam, idx_out=chosen)).astype(np.float64)
    assert len(chosen) == before + 1 and all(np.array_equal(_host(c).reshape(T, K), idx) for c in chosen)
    err = np.abs(got - want) - bound
    assert (err <= 0).all(), err.max()
