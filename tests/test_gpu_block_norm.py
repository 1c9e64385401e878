"""The norms around a block against a 64-bit reference, and the chain norm -> router -> 8-bit experts."""
import numpy as np
import pytest
import torch

import int8_ref as ref
from test_gpu_int8 import BF16, F32, _dev, _host, _mats, _pack, _rng, _same, _values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    import paper_2402_07033_amd as m
    m.lib()
    return m


def _inputs(rng, T, d, xd, yd):
    return dict(x=_values(rng, (T, d), xd), y=_values(rng, (T, d), yd, 0.5),
                gain_after=(1 + 0.1 * rng.standard_normal(d)).astype(np.float32),
                gain_before=(1 + 0.1 * rng.standard_normal(d)).astype(np.float32),
                gate=rng.standard_normal(d).astype(np.float32), row_gate=rng.random(T).astype(np.float32))


def _close(t, want):
    # one rounding from 64 bits: half a step (to bf16 by way of fp32: 2^-24 more); 2^-140: subnormal steps
    rel = 2.0 ** -24 + (ref.BF16 if t.dtype == BF16 else 0)
    assert (np.abs(_host(t).astype(np.float64) - want) <= rel * 1.0001 * np.abs(want) + 2.0 ** -140).all()


def _check_codes(codes, scales, h):
    q, s = ref.quantize(h)
    # the scale is top / 127 rounded once; the sums' order moves top by parts in 2^50
    assert (np.abs(_host(scales).astype(np.float64) - s) <= 2.0 ** -23 * np.abs(s)).all()
    z = h / np.where(_host(scales) > 0, _host(scales), 1).astype(np.float64)[:, None]
    clear = np.abs(np.abs(z) - np.floor(np.abs(z)) - 0.5) > 1e-9
    want = np.clip(np.rint(z), -127, 127)
    assert (_host(codes).astype(np.float64) == want)[clear].all() and clear.mean() > 0.999


@pytest.mark.parametrize("T,d", [(1, 64), (3, 128), (1, 4096), (7, 1408), (2, 8192), (5, 8256), (2, 16384), (1, 40000 // 64 * 64),
                                 (301, 2048)])
@pytest.mark.parametrize("xd,yd", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("after,gated", [(True, "feature"), (False, "token"), (True, "both"), (False, "none")])
def test_block_norm(moe, T, d, xd, yd, after, gated):
    i = _inputs(_rng(21, T, d), T, d, xd, yd)
    gate = i["gate"] if gated in ("feature", "both") else None
    row_gate = i["row_gate"] if gated in ("token", "both") else None
    gain_after = i["gain_after"] if after and gated != "both" else None
    gain_before = i["gain_before"] if gated != "none" else None
    x, h = ref.block_norm(i["x"], i["y"], after, gain_after, gate, row_gate, 0.7, gain_before, 1e-5)
    t = lambda v: None if v is None else _dev(v)  # noqa: E731
    for h_dtype, int8 in ((F32, True), (BF16, False), (None, True)):
        xx = _dev(i["x"], xd)
        out = moe.moe_block_norm(xx, _dev(i["y"], yd), norm_after=after, gain_after=t(gain_after), gate=t(gate),
                                 row_gate=t(row_gate), residual_scale=0.7, gain_before=t(gain_before), h_dtype=h_dtype,
                                 int8=int8, x_out=xx if int8 else None)  # (in place, and not)
        _close(out["x"], x)
        if h_dtype is not None:
            _close(out["h"], h)
        if int8:
            _check_codes(out["codes"], out["scales"], h)
        assert int8 or torch.equal(xx, _dev(i["x"], xd))


@pytest.mark.parametrize("xd", [F32, BF16])
def test_norm_alone(moe, xd):
    """Without a block's output: the first norm of a stack; only the codes; only the sum."""
    T, d = 5, 320
    i = _inputs(_rng(22), T, d, xd, xd)
    xx = _dev(i["x"], xd)
    out = moe.moe_block_norm(xx, gain_before=_dev(i["gain_before"]), int8=True)
    _, h = ref.block_norm(i["x"], None, False, None, None, None, 1.0, i["gain_before"], 1e-5)
    _close(out["h"], h)
    _check_codes(out["codes"], out["scales"], h)
    assert out["x"] is xx
    out = moe.moe_block_norm(xx, _dev(i["y"], xd), h_dtype=None)
    _close(out["x"], ref.block_norm(i["x"], i["y"], False, None, None, None, 1.0, None, 1e-5)[0])
    assert out["h"] is None and out["codes"] is None


def test_special_rows(moe):
    """All zeros, huge and tiny rows, NaN and infinity in one row only."""
    T, d = 8, 128
    i = _inputs(_rng(23), T, d, F32, F32)
    i["x"][0], i["y"][0] = 0, 0
    i["x"][1] *= 1e30
    i["y"][1] *= 1e30
    i["x"][2] *= 1e-36
    i["y"][2] *= 1e-36
    i["x"][3] *= 1e37
    ref_x, ref_h = ref.block_norm(i["x"], i["y"], False, None, None, None, 1.0, None, 1e-5)
    bad = {k: v.copy() for k, v in i.items()}
    bad["x"][5, 7], bad["y"][6, 9], bad["x"][7, 1] = np.nan, np.inf, -np.inf
    out = moe.moe_block_norm(_dev(bad["x"]), _dev(bad["y"]), int8=True)
    good = np.arange(T) < 5
    g = torch.from_numpy(good).cuda()
    _close(out["x"][g], ref_x[good])
    _close(out["h"][g], ref_h[good])
    _check_codes(out["codes"][g], out["scales"][g], ref_h[good])
    assert _host(out["scales"])[0] == 0 and (_host(out["codes"])[0] == 0).all()
    assert np.isnan(_host(out["scales"])[~good]).all() and (_host(out["codes"])[~good] == 0).all()


def test_no_tokens(moe):
    out = moe.moe_block_norm(torch.empty((0, 64), device="cuda"), torch.empty((0, 64), device="cuda"), int8=True)
    assert out["x"].shape == (0, 64) and out["codes"].shape == (0, 64)


@pytest.mark.parametrize("T,E,k,d,f", [(1, 8, 2, 256, 448), (7, 16, 4, 320, 128), (65, 4, 1, 128, 192)])
def test_chain(moe, T, E, k, d, f):
    """norm -> router -> 8-bit experts, then the next norm, captured and replayed; and the experts in a stack."""
    rng = _rng(24, T, d)
    mats = _mats(rng, E, d, f)
    W = _pack(moe, mats)
    i = _inputs(rng, T, d, F32, BF16)
    w_gate = (rng.standard_normal((d, E)) * d ** -0.5).astype(np.float32)
    dev = {n: _dev(v, BF16 if n == "y" else None) for n, v in i.items()}
    wg = _dev(w_gate)

    def chain():
        n = moe.moe_block_norm(dev["x"], dev["y"], norm_after=True, gain_after=dev["gain_after"], gate=dev["gate"],
                               gain_before=dev["gain_before"], int8=True)
        logits = moe.moe_router_logits(n["h"], wg)
        lay = moe.moe_layer_int8(W, (n["codes"], n["scales"]), logits, k)
        last = moe.moe_block_norm(n["x"], lay["y"], row_gate=dev["row_gate"])
        return n["codes"], n["scales"], logits, lay["y"], last["x"], last["h"]

    eager = [t.clone() for t in chain()]
    # the layer's result from the chain's own rows and logits
    q, s, lg = (_host(t) for t in eager[:3])
    _, _, y, bound = ref.layer(q, s, lg, k, mats, True)
    assert (np.abs(_host(eager[3]).astype(np.float64) - y) <= bound).all()
    x1, h1 = ref.block_norm(i["x"], i["y"], True, i["gain_after"], i["gate"], None, 1.0, i["gain_before"], 1e-5)
    _check_codes(eager[0], eager[1], h1)
    x2, h2 = ref.block_norm(x1.astype(np.float32), _host(eager[3]), False, None, None, i["row_gate"], 1.0, None, 1e-5)
    _close(eager[4], x2)
    _close(eager[5], h2)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = chain()
    for _ in range(4):
        g.replay()
        again = chain()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.equal(c, b) for a, b, c in zip(held, eager, again))


@pytest.mark.parametrize("T", [1, 3, 40])
def test_stack(moe, T):
    """moe_stack_forward over 8-bit handles is its separate calls."""
    E, k, d, f = 8, 2, 256, 192
    rng = _rng(25, T)
    layers = [(_pack(moe, _mats(rng, E, d, f)), _dev((rng.standard_normal((d, E)) * d ** -0.5).astype(np.float32)))
              for _ in range(3)]
    x0 = _dev(_values(rng, (T, d), F32))
    got = moe.moe_stack_forward(layers, x0.clone(), k, fused=False)
    x = x0.clone()
    for W, wg in layers:
        h = moe.moe_rmsnorm(x)
        x = x + moe.moe_layer_int8(W, h, moe.moe_router_logits(h, wg), k)["y"]
    assert torch.equal(got, x)
    # the fused front ends sum in another order: rounding of the rows, one code apart at most here and there
    fused = moe.moe_stack_forward(layers, x0.clone(), k)
    assert (fused - x).abs().max() <= 0.02 * x.abs().max()
