"""Calls on another stream than the current one, without a workspace of the caller's: what the binding allocates for
them stays theirs until they have run.  The other stream is kept busy, and the memory that the allocator hands out
meanwhile is overwritten."""
import pytest
import torch

import mxfp4_ref as ref
import paper_2402_07033_amd as moe
from test_gpu_mxfp4 import pack

pytestmark = pytest.mark.gpu


def setup(bf16):
    E, d, f = 8, 256, 512
    conv, mats = ref.matrices(1, E, d, f)
    if bf16:
        return moe.moe_weights_pack(*[torch.from_numpy(m).to(torch.bfloat16).contiguous().cuda() for m in mats])
    return pack(conv)


def on_a_busy_stream(call):
    """call(stream) behind other work of the stream, its freed memory filled on the current stream meanwhile."""
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    out = call(side)
    held = []
    for shift in range(8, 28):
        for _ in range(2):
            held.append(torch.full((1 << shift,), 0xFF, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("T", [3, 40, 200])
def test_layer_calls(T, bf16):
    W = setup(bf16)
    x, logits = torch.randn((T, W.d), device="cuda"), torch.randn((T, W.E), device="cuda")
    calls = [lambda s: moe.moe_layer(W, x, logits, 2, stream=s)["y"]]
    if not bf16:
        calls.append(lambda s: moe.moe_layer_mxfp4(W, x, logits, 2, stream=s)["y"])
    if T <= 16:
        calls.append(lambda s: moe.moe_decode_layer(W, x, logits, 2, stream=s)["y"])
    offsets = torch.arange(W.E + 1, dtype=torch.int32, device="cuda") * (T // W.E)
    offsets[-1] = T
    perm = torch.randperm(T, dtype=torch.int32, device="cuda")
    calls.append(lambda s: moe.moe_expert_ffn(W, x, offsets, stream=s))
    calls.append(lambda s: moe.moe_expert_ffn_tokens(W, x, 1, perm, offsets, stream=s))
    for call in calls:
        want = call(None)
        assert torch.equal(on_a_busy_stream(call), want)
    W.free()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("T,fused", [(1, True), (3, True), (40, True), (5, False)])
def test_stack(T, fused, bf16):
    W = setup(bf16)
    x = torch.randn((T, W.d), device="cuda")
    layers = [(W, torch.randn((W.d, W.E), device="cuda") / 16) for _ in range(3)]
    ids, wanted = [], []
    want = moe.moe_stack_forward(layers, x.clone(), 2, idx_out=wanted, fused=fused)
    rows = x.clone()
    assert torch.equal(on_a_busy_stream(lambda s: moe.moe_stack_forward(layers, rows, 2, idx_out=ids, fused=fused, stream=s)), want)
    assert all(torch.equal(a, b) for a, b in zip(ids, wanted))
    W.free()


def test_gate_sums():
    x, wg = torch.randn((2, 256), device="cuda"), torch.randn((256, 8), device="cuda")
    want = moe.moe_gate_sums(x, wg)
    assert torch.equal(on_a_busy_stream(lambda s: moe.moe_gate_sums(x, wg, stream=s)), want)
