"""Host side of the 4-bit (MXFP4) expert matrices: what the calls refuse, what they would run and need.
No GPU: a call that is not refused ends in MOE_ERR_HIP, so any other status came before a launch."""
import ctypes as C

import pytest

from paper_2402_07033_amd import binding
from test_abi_host import _Weights

INVALID, UNSUPPORTED, WORKSPACE, HIP = -1, -2, -3, -4
F32, BF16, MXFP4 = 0, 1, 2


@pytest.fixture(scope="module")
def L():
    return binding.lib()


class _MxWeights(_Weights):
    _fields_ = [("s13", C.c_void_p), ("s2", C.c_void_p)]


@pytest.fixture
def mem():
    """Aligned host memory for arguments that are never read."""
    buf = (C.c_char * (1 << 21))()
    return (C.addressof(buf) + 255) & ~255, buf


def convert(L, name, p, **change):
    a = dict(w=p, dtype=F32, E=2, K=64, C=48, codes=p + (1 << 17), scales=p + (1 << 18))
    a.update(change)
    if name == "moe_mxfp4_quantize":
        return L.moe_mxfp4_quantize(a["w"], a["dtype"], a["E"], a["K"], a["C"], a["codes"], a["scales"], None)
    return L.moe_mxfp4_dequantize(a["codes"], a["scales"], a["E"], a["K"], a["C"], a["w"], a["dtype"], None)


@pytest.mark.parametrize("name", ["moe_mxfp4_quantize", "moe_mxfp4_dequantize"])
def test_conversion_refuses(L, mem, name):
    p = mem[0]
    assert convert(L, name, p) == HIP
    for bad in (dict(w=None), dict(codes=None), dict(scales=None), dict(w=p + 8), dict(codes=p + (1 << 17) + 4),
                dict(scales=p + (1 << 18) + 1), dict(dtype=MXFP4), dict(dtype=7), dict(E=0), dict(E=65), dict(K=0), dict(K=48),
                dict(K=-32), dict(K=(1 << 20) + 32), dict(C=0), dict(C=(1 << 20) + 1), dict(codes=p + 1024),
                dict(scales=p + 1024)):
        assert convert(L, name, p, **bad) == INVALID, bad
    # two matrices of 64 x 48 are 24576 bytes: codes right behind them are fine
    assert convert(L, name, p, codes=p + 24576) == HIP


def test_quantize_refuses_overlapping_outputs(L, mem):
    p = mem[0]
    assert convert(L, "moe_mxfp4_quantize", p, scales=p + (1 << 17) + 1024) == INVALID


def test_pack_refuses(L, mem):
    p = mem[0]
    out = C.c_void_p(123)
    good = [p] * 6 + [8, 256, 512]

    def call(args):
        out.value = 123
        rc = L.moe_weights_pack_mxfp4(*args, C.byref(out), None)
        assert out.value is None  # no handle from a call that fails
        return rc
    assert call(good) == HIP
    for i in range(6):
        assert call(good[:i] + [None] + good[i + 1:]) == INVALID
        assert call(good[:i] + [p + 8] + good[i + 1:]) == INVALID
    for E, d, f in ((0, 256, 512), (65, 256, 512), (8, 0, 512), (8, 96, 512), (8, 256, 100), (8, 256, (1 << 20) + 64)):
        assert call([p] * 6 + [E, d, f]) == INVALID
    assert L.moe_weights_pack_mxfp4(*good, None, None) == INVALID


def layer(L, p, **change):
    W = _MxWeights(E=8, d=256, f=512, dtype=change.pop("w_dtype", MXFP4), device=change.pop("device", 0))
    step = 1 << 15
    a = dict(W=C.addressof(W), x=p, x_dtype=F32, logits=p + step, T=4, k=2, idx=p + 2 * step, weights=p + 3 * step,
             counts=p + 4 * step, offsets=p + 5 * step, perm=p + 6 * step, inv_perm=p + 7 * step, ws=p + 8 * step,
             ws_bytes=L.moe_layer_mxfp4_workspace(4, 8, 2, 256, 512), y=p + 48 * step, y_dtype=F32)
    assert set(change) <= set(a) and a["ws_bytes"] <= 32 * step
    a.update(change)
    return L.moe_layer_mxfp4(*a.values(), None)


def test_layer_refuses(L, mem):
    p = mem[0]
    step = 1 << 15
    assert layer(L, p) == HIP and layer(L, p, x_dtype=BF16, y_dtype=BF16) == HIP
    for bad in (dict(W=None), dict(w_dtype=BF16), dict(w_dtype=F32), dict(x=None), dict(x=p + 4), dict(x_dtype=MXFP4),
                dict(y_dtype=MXFP4), dict(y_dtype=5), dict(logits=None), dict(logits=p + step + 4), dict(T=-1), dict(k=0), dict(k=9),
                dict(T=1 << 23), dict(idx=None), dict(idx=p + 2 * step + 4), dict(weights=None), dict(counts=None),
                dict(offsets=None), dict(perm=None), dict(perm=p + 6 * step + 8), dict(inv_perm=None), dict(y=None),
                dict(y=p + 48 * step + 8),
                # outputs over x or logits
                dict(y=p), dict(y=p + 2048), dict(idx=p + step), dict(weights=p + step), dict(perm=p + step),
                dict(inv_perm=p), dict(counts=p + 64), dict(offsets=p + step + 96), dict(ws=p)):
        assert layer(L, p, **bad) == INVALID, bad
    for bad in (dict(ws=None), dict(ws=p + 8 * step + 16), dict(ws_bytes=L.moe_layer_mxfp4_workspace(4, 8, 2, 256, 512) - 1)):
        assert layer(L, p, **bad) == WORKSPACE, bad


def test_workspace_query(L):
    assert L.moe_layer_mxfp4_workspace(4, 8, 2, 256, 512) > 0
    for bad in ((-1, 8, 2, 256, 512), (4, 0, 1, 256, 512), (4, 65, 2, 256, 512), (4, 8, 9, 256, 512), (4, 2, 3, 256, 512),
                (4, 8, 2, 100, 512), (4, 8, 2, 256, 0)):
        assert L.moe_layer_mxfp4_workspace(*bad) == 0, bad
    assert L.moe_layer_mxfp4_workspace(0, 8, 2, 256, 512) > 0 and L.moe_expert_ffn_workspace(0, 8, 256, 512, F32) > 0
    # a prompt's rows and h in bf16 and the experts' rows in fp32 fit
    assert L.moe_layer_mxfp4_workspace(4096, 8, 2, 4096, 14336) >= 8192 * (2 * 4096 + 2 * 14336 + 4 * 4096)


def test_plan(L):
    plan = binding.FfnPlan()

    def path(N, E, d, f, p=0):
        rc = L.moe_expert_ffn_plan(N, E, d, f, MXFP4, p, C.byref(plan))
        return (rc, plan.path, plan.n_parts) if rc == 0 else rc
    stream, grouped, mid = 1, 2, 3
    assert path(2, 8, 4096, 14336) == (0, stream, 1) and path(32, 8, 4096, 14336) == (0, stream, 1)
    assert path(33, 8, 4096, 14336) == (0, grouped, 1) and path(72, 64, 2048, 1408) == (0, stream, 1)
    assert path(73, 64, 2048, 1408) == (0, grouped, 1) and path(8192, 8, 4096, 14336) == (0, grouped, 1)
    # forced: up to 72 rows of at most 4096 values
    assert path(72, 8, 4096, 14336, stream) == (0, stream, 1) and path(1, 8, 4096, 14336, grouped) == (0, grouped, 1)
    assert path(73, 8, 4096, 14336, stream) == UNSUPPORTED and path(2, 8, 4160, 512, stream) == UNSUPPORTED
    assert path(2, 8, 4160, 512) == (0, grouped, 1) and path(2, 8, 256, 512, mid) == UNSUPPORTED
    assert path(2, 8, 256, 512, 9) == INVALID


def test_block_query(L):
    # (needs no device: the bf16 kernels ask for the number of compute units, these do not)
    assert L.moe_decode_block_supported(1, 8, 2, 4096, 14336, MXFP4) == 1
    assert L.moe_decode_block_supported(2, 16, 2, 4096, 6400, MXFP4) == 1   # 34 sums
    assert L.moe_decode_block_supported(4, 16, 1, 4096, 6400, MXFP4) == 1   # 68
    assert L.moe_decode_block_supported(3, 8, 2, 4096, 14336, MXFP4) == 0   # six routed rows
    assert L.moe_decode_block_supported(1, 17, 2, 4096, 6400, MXFP4) == 0
    assert L.moe_decode_block_supported(1, 8, 2, 8192, 6400, MXFP4) == 0
    for T, E in ((1, 8), (2, 16), (4, 16), (1, 1)):
        stride = L.moe_gate_sums_stride(T, E)
        assert stride >= T * (E + 1) and stride % 32 == 0


def test_ffn_refuses_what_the_handle_cannot(L, mem):
    p = mem[0]
    W = _MxWeights(E=8, d=256, f=512, dtype=MXFP4)
    need = L.moe_expert_ffn_workspace(8, 8, 256, 512, F32)

    def ffn(path, N=8, act=F32):
        return L.moe_expert_ffn_path(C.addressof(W), p, act, p + 65536, N, p + 131072, need, p + 100000 * 8, path, None)
    assert ffn(0) == HIP and ffn(1) == HIP and ffn(2) == HIP and ffn(2, act=BF16) == HIP
    assert ffn(3) == UNSUPPORTED and ffn(0, act=MXFP4) == INVALID and ffn(9) == INVALID
    assert ffn(1, N=73) in (UNSUPPORTED, WORKSPACE) and ffn(0, N=0) == 0


def test_python_refusals():
    import torch
    import paper_2402_07033_amd as moe
    cpu = torch.zeros((2, 64, 48))
    with pytest.raises(TypeError):
        moe.moe_mxfp4_quantize(cpu)
    with pytest.raises(TypeError):
        moe.moe_mxfp4_quantize(cpu.double())
    with pytest.raises(TypeError):
        moe.moe_mxfp4_dequantize(torch.zeros((1, 2, 16), dtype=torch.uint8), torch.zeros((1, 2, 1), dtype=torch.uint8))


@pytest.mark.parametrize("E,d,f,N", [(16, 8192, 28672, 1), (16, 8192, 28672, 8), (64, 5120, 14336, 2), (64, 8192, 8192, 4)])
def test_a_few_rows_of_wide_layers_need_no_workspace(L, mem, E, d, f, N):
    """Scratch is for the experts that N rows can be on: d > 4096 has no streaming kernels, and its single rows go
    through the GEMM."""
    p = mem[0]
    W = _MxWeights(E=E, d=d, f=f, dtype=MXFP4)
    assert L.moe_expert_ffn_noalloc(C.addressof(W), p, F32, p + 65536, N, p + 131072, None) == HIP
