"""Which kernels a call over 4-bit expert matrices takes, and that the sizes around each choice are right."""
import numpy as np
import pytest
import torch

import mxfp4_ref as ref
import paper_2402_07033_amd as moe
from test_gpu_mxfp4 import check, cuda, pack, rows

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def random_handle(E, d, f, seed=3):
    """A handle of random codes, made on the device."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    conv = []
    for K, C in ((d, f), (d, f), (f, d)):
        codes = torch.randint(0, 256, (E, C, K // 2), dtype=torch.uint8, device="cuda", generator=gen)
        conv.append((codes, torch.randint(118, 121, (E, C, K // 32), dtype=torch.uint8, device="cuda", generator=gen)))
    return moe.moe_weights_pack_mxfp4(*conv)


@pytest.mark.parametrize("E,d,f,T,dtype,family", [
    (2, 4096, 14336, 10, F32, moe.MOE_FFN_STREAM),   # one pass over 187 MB
    (2, 4096, 14336, 11, F32, moe.MOE_FFN_GROUPED),  # two would be
    (2, 4096, 14336, 16, F32, moe.MOE_FFN_GROUPED),
    (2, 4096, 14336, 16, BF16, moe.MOE_FFN_STREAM),  # one
    (2, 2048, 1408, 16, F32, moe.MOE_FFN_STREAM)])   # small matrices
def test_layer_takes_the_faster_family(E, d, f, T, dtype, family):
    """With one expert per token and weight 1 the layer's rows are the expert FFN's, bit for bit, of the family that ran."""
    W = random_handle(E, d, f)
    x = torch.randn((T, d), device="cuda").to(dtype)
    logits = torch.zeros((T, E), device="cuda")
    logits[torch.arange(T), torch.arange(T) % E] = 1.0
    out = moe.moe_layer_mxfp4(W, x, logits, 1, y=torch.empty((T, d), device="cuda"))
    xg = x[out["perm"].long()]
    inv = out["inv_perm"].long()
    y = {p: moe.moe_expert_ffn(W, xg, out["offsets"], path=p)[inv] for p in (moe.MOE_FFN_STREAM, moe.MOE_FFN_GROUPED)}
    assert not torch.equal(*y.values())  # (the sums' orders differ)
    assert torch.equal(out["y"], y[family])
    W.free()
