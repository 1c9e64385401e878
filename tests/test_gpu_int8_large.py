"""8-bit products and experts over matrices that are read past the caches (more than 96 MiB in use, up to 128 rows of an expert
on average), and products in tiles of 224 channels with an odd number of channels.  Results of a product are
one sum of integers and two fp32 multiplications, so the same bits by any order of the sum: the oracle takes the sums
in 64-bit floats, which hold them exactly.  Experts: tiles against the streaming kernels, the same bits too."""
import numpy as np
import pytest
import torch

from test_gpu_int8 import BF16, F32, _dev, moe  # noqa: F401
from test_gpu_int8_grouped import _handle

pytestmark = pytest.mark.gpu

PAST_CACHES = 96 << 20


def _operands(seed, E, M, K, C):
    g = torch.Generator("cuda").manual_seed(seed)

    def codes(*shape):
        return torch.randint(-127, 128, shape, dtype=torch.int8, device="cuda", generator=g)

    def scales(*shape):
        return torch.rand(shape, device="cuda", generator=g) + 0.5
    return (codes(M, K), scales(M)), (codes(E, C, K), scales(E, C))


def _values(x, w, e, rows):
    sums = x[0][rows].double() @ w[0][e].double().t().contiguous()
    return sums.float() * x[1][rows, None] * w[1][e]


def _check(moe, x, w, offsets, dtype):  # noqa: F811
    """Rows behind offsets[-1] stay; offsets None: one matrix."""
    M, C = x[0].shape[0], w[0].shape[1]
    y = torch.full((M, C), 7.0, dtype=dtype, device="cuda")
    moe.moe_int8_matmul(x, w, offsets=None if offsets is None else _dev(np.array(offsets, dtype=np.int32)), y=y)
    ends = [0, M] if offsets is None else offsets
    for e, (a, b) in enumerate(zip(ends, ends[1:])):
        assert torch.equal(y[a:b], _values(x, w, e, slice(a, b)).to(dtype)), e
    assert (y[ends[-1]:] == 7.0).all()


# E, K, C, rows of each expert
PRODUCTS = [
    # streaming, four waves: K no multiple of 64, C odd
    (16, 2064, 3333, [5, 0, 16, 1, 7, 3, 17, 2, 0, 4, 4, 4, 1, 1, 9, 3]),
    # streaming, eight waves
    (4, 8208, 3334, [1, 0, 17, 9]),
    (1, 16400, 6501, [17]),
    # tiles of 32 x 128
    (4, 8208, 3334, [99, 0, 33, 170]),
    (1, 16400, 6501, [101]),
    # tiles of 128 x 128
    (16, 2064, 3333, [50, 0, 129, 1, 7, 3, 300, 2, 0, 64, 65, 127, 1, 1, 91, 3]),
    (16, 2112, 3332, [127] * 15 + [129]),
]


@pytest.mark.parametrize("E,K,C,counts", PRODUCTS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_product_past_the_caches(moe, E, K, C, counts, dtype):  # noqa: F811
    M = sum(counts)
    used = min(M, E)
    assert used * ((C + 15) // 16) * 16 * K > PAST_CACHES and M <= 128 * used
    behind = 0 if E == 1 else 5
    x, w = _operands(M, E, M + behind, K, C)
    _check(moe, x, w, None if E == 1 else [0] + np.cumsum(counts).tolist(), dtype)


# d, f, rows of each expert, tile rows of both projections
EXPERTS = [
    (2304, 2048, [37, 0, 128, 1, 17, 99, 64, 65] * 4, (128, 128)),
    (4096, 14336, [9, 100, 0, 33, 128, 1, 77, 16], (128, 128)),
    (16384, 2048, [100, 60], (32, 128)),     # few features in the first projection
    (2048, 32768, [99, 121], (128, 32)),     # ... in the second
    (2048, 32768, [33, 0, 17], (128, 32)),
]


@pytest.mark.parametrize("d,f,counts,rows", EXPERTS)
def test_experts_past_the_caches(moe, d, f, counts, rows):  # noqa: F811
    E, N = len(counts), sum(counts) + 3
    assert N <= 128 * E and min(N, E) * 2 * f * d > PAST_CACHES
    plan = moe.moe_expert_ffn_plan(N, E, d, f, moe.MOE_INT8)
    assert (plan["path"], plan["up_tile_rows"], plan["down_tile_rows"]) == (moe.MOE_FFN_GROUPED, *rows)
    W = _handle(moe, E, d, f, d + f + N)
    off = _dev(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))
    for dt in (F32, BF16):
        x = torch.randn((N, d), device="cuda", generator=torch.Generator("cuda").manual_seed(N)).to(dt)
        x[N - 3:] = float("nan")  # rows behind the last segment
        got, want = (torch.full((N, d), 9.0, device="cuda") for _ in range(2))
        moe.moe_expert_ffn(W, x, off, yg=want, path=moe.MOE_FFN_STREAM)
        moe.moe_expert_ffn(W, x, off, yg=got, path=moe.MOE_FFN_GROUPED)
        assert torch.equal(got, want) and (got[N - 3:] == 9.0).all()
        assert torch.isfinite(got).all() and got[: N - 3].abs().amax(dim=1).min() > 0


@pytest.mark.parametrize("E,K,C,counts", [(1, 144, 14333, [3001]), (1, 80, 10033, [2049]), (3, 80, 14333, [1500, 0, 1500])])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_odd_channels_in_tiles_of_224(moe, E, K, C, counts, dtype):  # noqa: F811
    M = sum(counts)
    behind = 0 if E == 1 else 1
    # (the rule sees the rows and the channels, rounded up: as a second projection of such features)
    assert moe.moe_expert_ffn_plan(M + behind, E, (C + 63) // 64 * 64, 64, moe.MOE_INT8, moe.MOE_FFN_GROUPED)["down_tile_features"] == 224
    x, w = _operands(M, E, M + behind, K, C)
    _check(moe, x, w, None if E == 1 else [0] + np.cumsum(counts).tolist(), dtype)
