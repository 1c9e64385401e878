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


# ---- rows of more than 4096 values: no streaming kernels, single tokens go through the GEMM ----

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d,f,E,N", [(4160, 192, 3, 1), (4160, 192, 3, 5), (4160, 192, 3, 72), (4160, 192, 3, 150), (5120, 320, 4, 7)])
def test_wide_rows(d, f, E, N, dtype):
    rng = np.random.default_rng(d + N)
    conv, mats = ref.matrices(d, E, d, f)
    W = pack(conv)
    x, x64 = rows(rng, N, d, dtype)
    offsets = np.concatenate([[0], np.sort(rng.integers(0, N + 1, size=E - 1)), [N]]).astype(np.int32)
    assert moe.moe_expert_ffn_plan(N, E, d, f, moe.MOE_MXFP4)["path"] == moe.MOE_FFN_GROUPED
    want, bound = ref.ffn(x64, offsets, mats, 0.0 if dtype == BF16 else ref.SPLIT, ref.SPLIT)
    yg = moe.moe_expert_ffn(W, x, cuda(offsets))
    check(yg, want, bound, what=(d, f, E, N))
    again = torch.empty_like(yg)
    moe.moe_expert_ffn_noalloc(W, x, cuda(offsets), again)
    assert torch.equal(again, yg)
    with pytest.raises(moe.MoeError):
        moe.moe_expert_ffn(W, x, cuda(offsets), path=moe.MOE_FFN_STREAM)
    W.free()


@pytest.mark.parametrize("xd,yd", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("T,d,f,E,k", [(1, 4160, 192, 8, 2), (2, 4160, 192, 8, 2), (16, 4608, 128, 12, 4), (90, 4160, 64, 3, 1)])
def test_layer_of_wide_rows(T, d, f, E, k, xd, yd):
    rng = np.random.default_rng(T + d)
    conv, mats = ref.matrices(d + f, E, d, f)
    W = pack(conv)
    x, x64 = rows(rng, T, d, xd)
    logits = rng.standard_normal((T, E)).astype(np.float32)
    parts = ref.SPLIT if yd == F32 else ref.PAIR
    want = ref.layer(x64, logits, mats, k, 0.0 if xd == BF16 else parts, parts)
    out = moe.moe_layer_mxfp4(W, x, cuda(logits), k, y=torch.empty((T, d), dtype=yd, device="cuda"))
    for n in ("idx", "counts", "offsets", "perm", "inv_perm"):
        assert np.array_equal(out[n].cpu().numpy(), want[n]), n
    check(out["y"], want["y"], want["bound"], yd, (T, d, f, E, k))
    if T <= 16:
        with pytest.raises(moe.MoeError):
            moe.moe_decode_layer(W, x.float(), cuda(logits), k)
    W.free()


# ---- more than 1024 rows of one expert: a second group of eight row tiles, of 128 rows or of 32 ----

@pytest.mark.parametrize("xd,yd", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("T,hot", [(300, 250), (600, 500), (1100, 1030), (2300, 2200)])
def test_rows_of_a_hot_expert(T, hot, xd, yd):
    """hot of T tokens on expert 1 of 3, the others on 0 and 2."""
    d, f, E = 192, 320, 3
    rng = np.random.default_rng(T)
    conv, mats = ref.matrices(T, E, d, f)
    W = pack(conv)
    x, x64 = rows(rng, T, d, xd)
    logits = rng.standard_normal((T, E)).astype(np.float32)
    logits[:, 1] = -20.0
    logits[rng.permutation(T)[:hot], 1] = 20.0
    parts = ref.SPLIT if yd == F32 else ref.PAIR
    want = ref.layer(x64, logits, mats, 1, 0.0 if xd == BF16 else parts, parts)
    assert want["counts"][1] == hot
    out = moe.moe_layer_mxfp4(W, x, cuda(logits), 1, y=torch.empty((T, d), dtype=yd, device="cuda"))
    assert np.array_equal(out["perm"].cpu().numpy(), want["perm"])
    check(out["y"], want["y"], want["bound"], yd, (T, hot))
    W.free()


def test_workspace_and_outputs_in_host_memory_are_refused():
    E, d, T, k = 4, 64, 6, 2
    W = pack(ref.matrices(11, E, d, 64)[0])
    x, logits = torch.randn((T, d), device="cuda"), torch.randn((T, E), device="cuda")
    need = moe.moe_layer_mxfp4_workspace(T, E, k, d, 64)
    for bad in (dict(workspace=torch.empty(need, dtype=torch.uint8)), dict(y=torch.empty((T, d))),
                dict(workspace=torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2]),
                dict(idx=torch.empty((T, k), dtype=torch.int32)), dict(weights=torch.empty((T, k)))):
        with pytest.raises(TypeError):
            moe.moe_layer_mxfp4(W, x, logits, k, **bad)
    W.free()
