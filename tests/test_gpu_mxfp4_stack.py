"""Stacks of blocks over 4-bit expert matrices beyond the two-launch form, and stacks whose blocks hold them in
different types, against 64 bits."""
import numpy as np
import pytest
import torch

import mxfp4_ref as ref
import paper_2402_07033_amd as moe
from test_gpu_mxfp4 import cuda, pack, rows

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def handle(kind, conv, mats):
    """The same matrices as a 4-bit, bf16 or fp32 handle (their values are exact in all three)."""
    if kind == "mx":
        return pack(conv)
    dt = BF16 if kind == "bf16" else F32
    return moe.moe_weights_pack(*[cuda(m.astype(np.float32)).to(dt) for m in mats])


def stack(T, E, k, d, f, kinds, fused=True, **kw):
    """-> rows after the stack: the library's, and in 64 bits; every choice of experts equal."""
    rng = np.random.default_rng(T + E)
    x, want = rows(rng, T, d, F32)
    layers, refs = [], []
    for n, kind in enumerate(kinds):
        conv, mats = ref.matrices(20 + n, E, d, f)
        wg = (rng.standard_normal((d, E)) / np.sqrt(d)).astype(np.float32)
        layers.append((handle(kind, conv, mats), cuda(wg)))
        refs.append((mats, wg.astype(np.float64)))
    idx = []
    got = moe.moe_stack_forward(layers, x.clone(), k, idx_out=idx, fused=fused, **kw)
    for n, (mats, wg) in enumerate(refs):
        h = want / np.sqrt((want * want).mean(axis=1, keepdims=True) + 1e-5)
        lg = h @ wg
        top = np.sort(lg, axis=1)
        out = ref.layer(h, lg.astype(np.float32), mats, k, ref.SPLIT, ref.SPLIT)
        clear = top[:, E - k] - top[:, E - k - 1] > 1e-3  # (no choice that hangs on a rounding)
        assert clear.mean() > 0.9 and np.array_equal(np.sort(idx[n].cpu().numpy()[clear]), np.sort(out["idx"][clear]))
        # an unclear token may differ from here on; it is left out of the comparison
        want = want + out["y"]
        want[~clear] = np.nan
    for W, _ in layers:
        W.free()
    return got.cpu().numpy(), want


def relative(got, want):
    rows_ = np.isfinite(want).all(axis=1)
    assert rows_.mean() > 0.7
    return np.linalg.norm(got[rows_] - want[rows_]) / np.linalg.norm(want[rows_])


# Routed rows above four, experts above 16, d above 4096: the separate calls.  24-bit rows, so what remains are the fp32
# sums of the norms and router sums (d * 2^-24 at most) in three blocks, as in the two-launch form's test.
@pytest.mark.parametrize("fused", [True, False])
@pytest.mark.parametrize("T,E,k,d,f", [(3, 8, 2, 256, 512), (4, 16, 2, 320, 448), (2, 20, 2, 256, 320), (6, 8, 2, 256, 2112),
                                       (40, 8, 2, 256, 512), (200, 8, 2, 256, 320), (1, 8, 2, 4160, 192), (5, 8, 2, 4160, 192)])
def test_stack_in_separate_calls(T, E, k, d, f, fused):
    assert not moe.moe_decode_block_supported(T, E, k, d, f, moe.MOE_MXFP4)
    assert relative(*stack(T, E, k, d, f, ["mx"] * 3, fused)) <= 2.0 ** -15


# bf16 blocks split fp32 rows into two bf16 parts, 2^-16 each at most; twice that for three blocks' sums
@pytest.mark.parametrize("T,E,k,d,f", [(1, 8, 2, 256, 512), (2, 16, 2, 256, 512), (4, 8, 2, 256, 2112), (6, 8, 2, 256, 2112),
                                       (30, 8, 2, 256, 2112)])
@pytest.mark.parametrize("kinds", [("mx", "bf16", "mx"), ("bf16", "mx", "bf16"), ("mx", "f32", "bf16")])
def test_stack_of_mixed_handles(T, E, k, d, f, kinds):
    assert relative(*stack(T, E, k, d, f, kinds)) <= 2.0 ** -14


def test_buffers_of_mixed_handles():
    bufs = moe.StackBuffers(6, 8, 2, 256, 2112, w_dtype=(moe.MOE_MXFP4, moe.MOE_BF16))
    assert bufs.max_parts == moe.moe_expert_ffn_plan(12, 8, 256, 2112, moe.MOE_BF16)["n_parts"] > 1
    got, want = stack(6, 8, 2, 256, 2112, ("mx", "bf16"), bufs=bufs)
    assert relative(got, want) <= 2.0 ** -14
