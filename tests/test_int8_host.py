"""Host-only checks of the 8-bit calls and of moe_block_norm: what they refuse before anything is launched, their
queries, and the reference's own arithmetic."""
import ctypes as C

import numpy as np
import pytest

import int8_ref as ref
from test_abi_host import L, _Weights  # noqa: F401
from test_mxfp4_host import _MxWeights

F32, BF16, INT8 = 0, 1, 3
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3


@pytest.fixture(scope="module")
def at():
    """Aligned fake addresses, 1 MiB apart."""
    return [C.c_void_p((1 << 40) + (i << 20)) for i in range(20)]


def _off(p, n):
    return C.c_void_p(p.value + n)


def test_conversions_refuse(L, at):  # noqa: F811
    w, q, s = at[:3]
    ok = dict(w=w, t=F32, E=2, K=64, C=48, q=q, s=s)

    def both(code, **change):
        a = dict(ok, **change)
        assert L.moe_int8_quantize(a["w"], a["t"], a["E"], a["K"], a["C"], a["q"], a["s"], None) == code
        assert L.moe_int8_dequantize(a["q"], a["s"], a["E"], a["K"], a["C"], a["w"], a["t"], None) == code

    for change in (dict(w=None), dict(q=None), dict(s=None), dict(t=2), dict(t=INT8), dict(E=0), dict(E=65), dict(K=0), dict(K=24),
                   dict(K=(1 << 17) + 16), dict(C=0), dict(C=(1 << 20) + 1), dict(w=_off(w, 8)), dict(q=_off(q, 4)), dict(s=_off(s, 4)),
                   dict(q=_off(w, 2 * 64 * 48 * 4 - 16)), dict(s=_off(q, 2 * 64 * 48 - 16)), dict(s=_off(w, 16))):
        both(INVALID, **change)

    def rows(code, **change):
        a = dict(dict(w=w, t=BF16, T=3, K=64, q=q, s=s), **change)
        assert L.moe_int8_quantize_rows(a["w"], a["t"], a["T"], a["K"], a["q"], a["s"], None) == code
        assert L.moe_int8_dequantize_rows(a["q"], a["s"], a["T"], a["K"], a["w"], a["t"], None) == code

    for change in (dict(w=None), dict(q=None), dict(s=None), dict(t=INT8), dict(T=-1), dict(K=40), dict(K=0), dict(K=1 << 18),
                   dict(w=_off(w, 2)), dict(q=_off(w, 3 * 64 * 2 - 16)), dict(s=_off(q, 3 * 64 - 16))):
        rows(INVALID, **change)
    rows(0, T=0, w=None, q=None, s=None)


def test_matmul_refuses(L, at):  # noqa: F811
    xq, xs, wq, ws, off, y = at[:6]
    ok = dict(xq=xq, xs=xs, M=5, wq=wq, ws=ws, E=2, K=64, C=48, off=off, y=y, t=BF16)

    def call(**change):
        a = dict(ok, **change)
        return L.moe_int8_matmul(a["xq"], a["xs"], a["M"], a["wq"], a["ws"], a["E"], a["K"], a["C"], a["off"], a["y"], a["t"], None)

    for change in (dict(xq=None), dict(xs=None), dict(wq=None), dict(ws=None), dict(y=None), dict(off=None), dict(M=-1), dict(M=1 << 24),
                   dict(E=0), dict(E=65), dict(K=8), dict(K=72), dict(K=1 << 18), dict(C=0), dict(C=(1 << 20) + 1), dict(t=INT8), dict(t=2),
                   dict(xq=_off(xq, 4)), dict(wq=_off(wq, 8)), dict(y=_off(y, 2)), dict(off=_off(off, 4)),
                   dict(y=_off(xq, 5 * 64 - 16)), dict(y=_off(xs, 16)), dict(y=_off(wq, 2 * 48 * 64 - 16)), dict(y=ws), dict(y=off)):
        assert call(**change) == INVALID, change
    assert call(M=0) == 0
    assert call(M=0, xq=None, y=None) == 0


def test_pack_refuses(L, at):  # noqa: F811
    h = C.c_void_p(1)
    ptrs = at[:6]
    assert L.moe_weights_pack_int8(*ptrs, 8, 4096, 14336, None, None) == INVALID
    for E, d, f in ((0, 64, 64), (65, 64, 64), (8, 96, 64), (8, 64, 100), (8, (1 << 17) + 64, 64), (8, 64, 1 << 18)):
        assert L.moe_weights_pack_int8(*ptrs, E, d, f, C.byref(h), None) == INVALID and h.value is None
    for i in range(6):
        for bad in (None, _off(ptrs[i], 4)):
            p = list(ptrs)
            p[i] = bad
            assert L.moe_weights_pack_int8(*p, 8, 64, 64, C.byref(h), None) == INVALID and h.value is None


def _handle(E=8, d=256, f=512, dtype=INT8):
    w = _MxWeights()
    w.E, w.d, w.f, w.dtype = E, d, f, dtype
    return w


def test_layer_refuses(L, at):  # noqa: F811
    W = _handle()
    need = L.moe_layer_int8_workspace(4, 8, 2, 256, 512)
    assert need > 4 * 2 * (256 * 4 + 512 * 5)
    for bad in ((-1, 8, 2, 256, 512), (4, 8, 9, 256, 512), (4, 65, 2, 256, 512), (4, 8, 2, 100, 512), (4, 8, 2, 256, 0)):
        assert L.moe_layer_int8_workspace(*bad) == 0
    x, xs, lg, idx, w, cnt, off, perm, inv, ws, y = at[:11]
    ok = dict(W=C.byref(W), x=x, t=F32, xs=None, lg=lg, T=4, k=2, idx=idx, w=w, cnt=cnt, off=off, perm=perm, inv=inv, ws=ws,
              n=need, y=y, yt=F32)

    def call(**change):
        a = dict(ok, **change)
        return L.moe_layer_int8(*(a[n] for n in ("W", "x", "t", "xs", "lg", "T", "k", "idx", "w", "cnt", "off", "perm", "inv", "ws",
                                                 "n", "y", "yt")), None)

    for change in (dict(W=None), dict(W=C.byref(_handle(dtype=BF16))), dict(W=C.byref(_handle(dtype=2))), dict(x=None), dict(lg=None),
                   dict(idx=None), dict(w=None), dict(cnt=None), dict(off=None), dict(perm=None), dict(inv=None), dict(y=None),
                   dict(t=2), dict(yt=INT8), dict(T=-1), dict(k=0), dict(k=9), dict(xs=xs), dict(t=INT8), dict(x=_off(x, 8)),
                   dict(y=_off(y, 4)), dict(lg=_off(lg, 4)), dict(t=INT8, xs=_off(xs, 4)), dict(y=x), dict(y=lg), dict(idx=lg), dict(w=x),
                   dict(t=INT8, xs=xs, y=xs), dict(t=INT8, xs=xs, w=xs), dict(ws=C.c_void_p(x.value - 4096)), dict(T=1 << 23)):
        assert call(**change) == INVALID, change
    for change in (dict(ws=None), dict(n=need - 1), dict(ws=_off(ws, 16))):
        assert call(**change) == WORKSPACE, change


def test_other_calls_on_a_handle(L, at):  # noqa: F811
    W = _handle()
    p = at[:14]
    assert L.moe_expert_ffn(C.byref(W), p[0], INT8, p[1], 4, p[2], 1 << 30, p[3], None) == INVALID
    assert L.moe_expert_ffn(C.byref(W), p[0], F32, p[1], 4, p[2], 64, p[3], None) == WORKSPACE
    assert L.moe_expert_ffn_path(C.byref(W), p[0], F32, p[1], 4, p[2], 1 << 30, p[3], 3, None) == UNSUPPORTED   # MID
    assert L.moe_decode_layer(C.byref(W), p[0], p[1], 1, 2, *p[2:8], None, p[8], 1 << 30, None, p[9], None) == UNSUPPORTED
    assert L.moe_decode_block(C.byref(W), p[0], None, 0, C.c_float(1e-5), p[1], 1, 2, *p[2:8], p[8], 1 << 30, p[9], None, None,
                              None) == UNSUPPORTED
    assert L.moe_decode_block_supported(1, 8, 2, 256, 512, INT8) == 0
    assert L.moe_layer_mxfp4(C.byref(W), p[0], F32, p[1], 1, 2, *p[2:8], p[8], 1 << 30, p[9], F32, None) == INVALID
    from paper_2402_07033_amd import binding
    plan = binding.FfnPlan()
    assert L.moe_expert_ffn_plan(4096, 8, 4096, 14336, INT8, 0, C.byref(plan)) == 0 and plan.path == 2 and plan.n_parts == 1
    assert L.moe_expert_ffn_plan(4096, 8, 4096, 14336, INT8, 3, C.byref(plan)) == UNSUPPORTED
    assert L.moe_expert_ffn_plan(4096, 8, 1 << 18, 14336, INT8, 0, C.byref(plan)) == UNSUPPORTED
    # more threads than a launch may have
    assert L.moe_expert_ffn_plan((1 << 24) - 1, 8, 4096, 14336, INT8, 1, C.byref(plan)) == UNSUPPORTED
    assert L.moe_expert_ffn_plan((1 << 24) - 1, 8, 1 << 17, 1 << 17, INT8, 0, C.byref(plan)) == UNSUPPORTED
    assert L.moe_expert_ffn_plan(1 << 20, 8, 4096, 14336, INT8, 0, C.byref(plan)) == 0 and plan.up_tile_rows == 256
    assert L.moe_expert_ffn_workspace(1, 1, 1 << 18, 64, F32) > 0   # (no 8-bit handle has such rows)


def test_outputs_over_one_another(L, at):  # noqa: F811
    """(On a handle of a device that is not the current one: nothing is launched whatever the checks let through.)"""
    W = _handle()
    W.device = 1 << 20
    need = L.moe_layer_int8_workspace(4, 8, 2, 256, 512)
    outs = dict(idx=32, w=32, cnt=32, off=36, perm=32, inv=32, ws=need, y=4096)

    def call(**change):
        a = dict(zip(outs, at[2:]), **change)
        return L.moe_layer_int8(C.byref(W), at[0], F32, None, at[1], 4, 2, a["idx"], a["w"], a["cnt"], a["off"], a["perm"], a["inv"],
                                a["ws"], need, a["y"], F32, None)

    for n, p in zip(outs, at[2:]):
        for o, q in zip(outs, at[2:]):
            if n != o and n != "ws":
                assert call(**{n: _off(q, outs[o] // 16 * 16 - 16 if o != "cnt" else 0)}) == INVALID, (n, o)
    assert call() == INVALID  # the device


def test_handle_of_another_device(L, at):  # noqa: F811
    W = _handle()
    W.device = 1 << 20
    p = at[:14]
    big = C.c_size_t(1 << 30)
    assert L.moe_expert_ffn(C.byref(W), p[0], F32, p[1], 4, p[2], big, p[3], None) == INVALID
    assert L.moe_expert_ffn_path(C.byref(W), p[0], BF16, p[1], 4, p[2], big, p[3], 1, None) == INVALID
    assert L.moe_expert_ffn_tokens(C.byref(W), p[0], F32, 2, 2, p[4], p[1], p[2], big, p[3], None) == INVALID
    assert L.moe_expert_ffn_noalloc(C.byref(W), p[0], F32, p[1], 4, p[3], None) == INVALID
    stage = C.c_int(-1)
    assert L.moe_layer(C.byref(W), p[0], F32, 256, p[1], 2, 8, 2, 0, *p[2:8], p[8], p[9], big, p[10], p[11], C.byref(stage), None) == INVALID
    assert stage.value == 2


def test_block_norm_refuses(L, at):  # noqa: F811
    x, y, ga, g, rg, gb, xo, h, q, s = at[:10]
    ok = dict(x=x, xt=F32, y=y, yt=BF16, T=4, d=128, after=1, ga=ga, g=g, rg=rg, r=0.5, gb=gb, eps=1e-5, xo=xo, h=h, ht=BF16, q=q, s=s)

    def call(**change):
        a = dict(ok, **change)
        return L.moe_block_norm(a["x"], a["xt"], a["y"], a["yt"], a["T"], a["d"], a["after"], a["ga"], a["g"], a["rg"],
                                C.c_float(a["r"]), a["gb"], C.c_float(a["eps"]), a["xo"], a["h"], a["ht"], a["q"], a["s"], None)

    inf = float("inf")
    for change in (dict(x=None), dict(xt=2), dict(yt=INT8), dict(ht=INT8), dict(T=-1), dict(d=0), dict(d=100), dict(d=1 << 18),
                   dict(eps=0.0), dict(eps=-1.0), dict(eps=inf), dict(eps=float("nan")), dict(after=0), dict(y=None),
                   dict(y=None, after=0, ga=None), dict(y=None, after=0, ga=None, g=None), dict(q=None), dict(s=None),
                   dict(xo=None, h=None, q=None, s=None), dict(x=_off(x, 8)), dict(y=_off(y, 8)), dict(ga=_off(ga, 4)), dict(rg=_off(rg, 4)),
                   dict(xo=_off(xo, 4)), dict(q=_off(q, 4)), dict(s=_off(s, 4)), dict(xo=_off(x, 16)), dict(xo=y), dict(h=x), dict(h=y),
                   dict(h=xo), dict(q=h), dict(s=q), dict(s=rg), dict(h=gb), dict(q=x), dict(s=_off(x, 4 * 128 * 4 - 16))):
        assert call(**change) == INVALID, change
    assert call(T=0) == 0


def test_reference_codes():
    """Ties to even, the largest value's code, exactness of the quotient next to a border."""
    q, s = ref.quantize(np.array([[127.0, 0.5, 1.5, -2.5, -0.5, 126.5, 3.5]], dtype=np.float32))
    assert s[0] == 1.0 and q[0].tolist() == [127, 0, 2, -2, 0, 126, 4]
    v = np.array([[254.0, np.nextafter(np.float32(1), np.float32(2)), np.nextafter(np.float32(1), np.float32(0))]], dtype=np.float32)
    q, s = ref.quantize(v)
    assert s[0] == 2.0 and q[0].tolist() == [127, 1, 0]
    q, s = ref.quantize(np.array([[0.0, 0.0], [np.inf, 1.0], [np.nan, 1.0]], dtype=np.float32))
    assert s[0] == 0 and np.isnan(s[1:]).all() and not q.any()
