"""Arguments that lie over one another, told apart from a call that is refused for another reason: where there is no GPU
a clean call passes every check and fails at its launch."""
import ctypes as C

import pytest
import torch

from test_abi_host import L  # noqa: F401
from test_int8_host import BF16, F32, INVALID, _off, at  # noqa: F401

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
