"""Arguments that lie over one another, told apart from a call that is refused for another reason: where there is no GPU
a clean call passes every check and fails at its launch."""
import ctypes as C

import pytest
import torch

from test_abi_host import L  # noqa: F401
from test_int8_host import BF16, F32, INT8, INVALID, _handle, _off, at  # noqa: F401

HIP = -4
no_gpu = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="a clean call would run on made-up addresses")


def _block_norm(L, a):  # noqa: F811
    return L.moe_block_norm(a["x"], a["xt"], a["y"], a["yt"], a["T"], a["d"], a["after"], a["ga"], a["g"], a["rg"], C.c_float(0.5),
                            a["gb"], C.c_float(1e-5), a["xo"], a["h"], a["ht"], a["q"], a["s"], None)


@pytest.fixture(scope="module")
def norm_args(at):  # noqa: F811
    x, y, ga, g, rg, gb, xo, h, q, s = at[:10]
    return dict(x=x, xt=F32, y=y, yt=F32, T=4, d=128, after=1, ga=ga, g=g, rg=rg, gb=gb, xo=xo, h=h, ht=BF16, q=q, s=s)


@no_gpu
def test_norm_in_place_is_accepted(L, norm_args):  # noqa: F811
    assert _block_norm(L, norm_args) == HIP
    assert _block_norm(L, dict(norm_args, xo=norm_args["x"])) == HIP


@pytest.mark.parametrize("T", [1, 4])
@pytest.mark.parametrize("name", ["y", "ga", "g", "rg", "gb"])
def test_norm_in_place_over_another_input(L, norm_args, name, T):  # noqa: F811
    """x_out may be x, and x alone: every row's workgroup reads gains and gates, and y has a place and a type of its own."""
    x = norm_args["x"]
    a = dict(norm_args, T=T, xo=x)
    for type_ in (F32, BF16):
        assert _block_norm(L, dict(a, **{name: x}, yt=type_)) == INVALID
        assert _block_norm(L, dict(a, **{name: _off(x, 128)}, yt=type_)) == INVALID


LAYER = ("x", "xs", "lg", "idx", "w", "cnt", "off", "perm", "inv", "ws", "y")
T, E, K, D, F = 4, 8, 2, 256, 512


@pytest.fixture(scope="module")
def layer(L, at):  # noqa: F811
    """The layer call with some addresses changed, the arguments' own ones, and their bytes.  The handle's device is what
    the library takes for the current one where there is none."""
    W = _handle(E=E, d=D, f=F)
    W.device = -1
    need = L.moe_layer_int8_workspace(T, E, K, D, F)
    at = {n: C.c_void_p((1 << 42) + (i << 24)) for i, n in enumerate(LAYER)}
    assert need < 1 << 24
    n = 4 * T * K
    size = dict(x=T * D, xs=4 * T, lg=4 * T * E, idx=n, w=n, cnt=4 * E, off=4 * E + 4, perm=n, inv=n, ws=need, y=4 * T * D)

    def call(x_type=INT8, **change):
        a = dict(at, **change)
        return L.moe_layer_int8(C.byref(W), a["x"], x_type, a["xs"] if x_type == INT8 else None, a["lg"], T, K,
                                *(a[m] for m in LAYER[3:9]), a["ws"], need, a["y"], F32, None)
    return call, at, size


@no_gpu
def test_layer_over_nothing_is_accepted(layer):
    call, at, size = layer  # noqa: F811
    assert call() == HIP and call(x_type=F32) == HIP and call(x_type=BF16) == HIP
    # neighbours that touch: 16-byte aligned ones behind their bytes
    for n in LAYER[3:9] + ("y",):
        for o in LAYER:
            if n != o:
                assert call(**{n: _off(at[o], (size[o] + 15) // 16 * 16)}) == HIP, (n, o)


@no_gpu
@pytest.mark.parametrize("out", LAYER[3:])
def test_layer_outputs_over_others(layer, out):
    """An output on the first and on the last bytes of every other argument, and the other way round."""
    call, at, size = layer  # noqa: F811
    for o in LAYER:
        if o == out:
            continue
        assert call(**{out: at[o]}) == INVALID, o
        if out != "ws":  # (a workspace that is not aligned to 256 is refused for that)
            assert call(**{out: _off(at[o], (size[o] - 1) // 16 * 16)}) == INVALID, o
            assert call(**{out: _off(at[o], 16 - 16 * ((size[out] + 15) // 16))}) == INVALID, o
