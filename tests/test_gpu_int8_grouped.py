"""8-bit experts of many rows each: the persistent grouped GEMM against the streaming kernels.  Sums of integers have no
order and the epilogues are the same functions, so the results are the same bits (the streaming kernels are held to 64-bit
references in test_gpu_int8.py)."""
import numpy as np
import pytest
import torch

from test_gpu_int8 import BF16, F32, _dev, _rng, _same, _host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    import paper_2402_07033_amd as m
    m.lib()
    return m


def _handle(moe, E, d, f, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def mat(K, C):
        return (torch.randint(-127, 128, (E, C, K), dtype=torch.int8, device="cuda", generator=g),
                torch.rand((E, C), device="cuda", generator=g) * (2e-2 / K ** 0.5))
    return moe.moe_weights_pack_int8(mat(d, f), mat(d, f), mat(f, d))


# d, f, rows of each expert, tile rows of both projections that the plan names (256 twice, 192: the persistent loop)
CASES = [
    (2048, 2048, [1800, 1600, 1777, 1423], 256),           # odd counts
    (2048, 2304, [5000, 0, 1, 1500], 256),                 # an empty expert, one of a single row, left-over tiles
    (4096, 512, [257, 15, 16, 17, 2000, 31, 33, 4000], (128, 256)),  # too few tiles of 256 x 256 in the first
    (512, 4096, [12000, 12345], (256, 128)),               # ... in the second
    (4096, 512, [257, 15, 16, 17, 4000, 31, 33, 6500], 256),   # short reduction of the second projection
    (512, 4096, [13000, 13345], 256),                      # short reduction of the first, two column tiles
    (2304, 2048, [150, 140, 160, 133] * 8, 192),           # the tile of 192 rows
    (2048, 2048, [240, 256, 255, 233] * 4, 192),
    (2048, 2048, [6500], 256),                             # one expert
]


@pytest.mark.parametrize("d,f,counts,rows", CASES)
def test_same_bits(moe, d, f, counts, rows):
    E, N = len(counts), sum(counts)
    W = _handle(moe, E, d, f, d + f + N)
    plan = moe.moe_expert_ffn_plan(N + 3, E, d, f, moe.MOE_INT8, moe.MOE_FFN_GROUPED)
    assert (plan["up_tile_rows"], plan["down_tile_rows"]) == (rows if isinstance(rows, tuple) else (rows, rows))
    off = _dev(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))
    for dt in (F32, BF16):
        x = torch.randn((N + 3, d), device="cuda", generator=torch.Generator("cuda").manual_seed(5)).to(dt)
        x[N:] = float("nan")  # rows behind the last segment
        x[7, 3] = float("inf")  # a row that is all NaN, and no other
        want = torch.full((N + 3, d), 9.0, device="cuda")
        got = want.clone()
        moe.moe_expert_ffn(W, x, off, yg=want, path=moe.MOE_FFN_STREAM)
        ws = torch.full((moe.moe_expert_ffn_workspace(N + 3, E, d, f, moe.MOE_BF16),), 0x7F, dtype=torch.uint8, device="cuda")
        for _ in range(2):  # a used workspace as well as a fresh one
            got.fill_(9.0)
            moe.moe_expert_ffn(W, x, off, yg=got, workspace=ws, path=moe.MOE_FFN_GROUPED)
            assert (got[N:] == 9.0).all() and (want[N:] == 9.0).all()
            bad = torch.isnan(want).any(dim=1)
            assert torch.isnan(got[7]).all() and bad.sum() == 1 and torch.equal(torch.isnan(got).any(dim=1), bad)
            assert torch.equal(got[~bad], want[~bad])


@pytest.mark.parametrize("T,k", [(3300, 2), (6601, 1)])
def test_layer(moe, T, k):
    d, f, E = 2048, 2048, 4
    W = _handle(moe, E, d, f, T)
    g = torch.Generator("cuda").manual_seed(T)
    x = torch.randn((T, d), device="cuda", generator=g)
    logits = torch.randn((T, E), device="cuda", generator=g) - torch.arange(E, device="cuda") * 0.7
    want = moe.moe_layer(W, x, logits, k, path=moe.MOE_FFN_STREAM)
    out = moe.moe_layer_int8(W, x, logits, k)
    assert torch.equal(out["y"], want["y"]) and torch.equal(out["perm"], want["perm"])
    again = moe.moe_layer_int8(W, moe.moe_int8_quantize_rows(x), logits, k, dtype=F32)
    assert torch.equal(again["y"], want["y"])
    small = torch.empty(moe.moe_layer_int8_workspace(T, E, k, d, f) - 1, dtype=torch.uint8, device="cuda")
    with pytest.raises(moe.MoeError):
        moe.moe_layer_int8(W, x, logits, k, workspace=small)
