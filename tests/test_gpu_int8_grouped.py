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
    (4096, 4096, [2200, 2000], 256),                       # left-over tiles of both projections cut along the reduction
    (4096, 4096, [300, 0, 1900, 77, 1999, 1], 256),
    (2048, 1408, [370, 0, 400, 391, 383] * 8, 256),        # a reduction that is no multiple of 256: steps filled with zeros
    (2304, 1152, [2900, 3100, 17, 1111], 256),
    (3840, 4992, [1700, 1900], 256),
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


@pytest.mark.parametrize("M,K,C", [(2048, 128, 14336), (3000, 144, 14272), (2817, 4096, 10001)])
def test_products_of_whole_rounds(moe, M, K, C):
    """Tiles of 224 channels: the last rows and channels of a product are what a call on a few rows gives."""
    g = torch.Generator("cuda").manual_seed(M)
    x = torch.randint(-127, 128, (M, K), dtype=torch.int8, device="cuda", generator=g)
    w = torch.randint(-127, 128, (1, C, K), dtype=torch.int8, device="cuda", generator=g)
    s, t = torch.rand(M, device="cuda", generator=g) + 0.5, torch.rand((1, C), device="cuda", generator=g) + 0.5
    y = moe.moe_int8_matmul((x, s), (w, t), dtype=F32)
    for r in (0, 240, M // 64 * 32, (M - 1) // 32 * 32):
        n = min(32, M - r)
        assert torch.equal(y[r:r + n], moe.moe_int8_matmul((x[r:r + n], s[r:r + n]), (w, t), dtype=F32))


def test_second_projection_of_whole_rounds(moe):
    N, d, f = 2048, 14272, 64
    assert moe.moe_expert_ffn_plan(N, 1, d, f, moe.MOE_INT8, moe.MOE_FFN_GROUPED)["down_tile_features"] == 224
    W = _handle(moe, 1, d, f, 5)
    x = torch.randn((N, d), device="cuda", generator=torch.Generator("cuda").manual_seed(6))
    off = torch.tensor([0, N - 3], dtype=torch.int32, device="cuda")
    got, want = (torch.full((N, d), 4.0, device="cuda") for _ in range(2))
    moe.moe_expert_ffn(W, x, off, yg=got, path=moe.MOE_FFN_GROUPED)
    moe.moe_expert_ffn(W, x, off, yg=want, path=moe.MOE_FFN_STREAM)
    assert torch.equal(got, want) and (got[N - 3:] == 4.0).all()


# ---- more rows than a launch takes, and offsets past 32 bits: the last rows are what a call on them alone gives ----

def test_product_past_4_gib(moe):
    M, K, C = 1100000, 4096, 64
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.empty((M, K), dtype=torch.int8, device="cuda")
    x[:2000] = torch.randint(-127, 128, (2000, K), dtype=torch.int8, device="cuda", generator=g)
    x[2000:-2000] = 1
    x[-2000:] = torch.randint(-127, 128, (2000, K), dtype=torch.int8, device="cuda", generator=g)
    xs = torch.rand(M, device="cuda", generator=g)
    w = (torch.randint(-127, 128, (1, C, K), dtype=torch.int8, device="cuda", generator=g), torch.rand((1, C), device="cuda", generator=g))
    y = moe.moe_int8_matmul((x, xs), w, dtype=F32)
    for part in (slice(0, 2000), slice(M - 2000, M)):
        assert torch.equal(y[part], moe.moe_int8_matmul((x[part].clone(), xs[part].clone()), w, dtype=F32))


def test_experts_past_4_gib(moe):
    N, d, f = 80000, 512, 14336  # h: 4.6 GB
    W = _handle(moe, 1, d, f, 3)
    x = torch.randn((N, d), device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    y = moe.moe_expert_ffn(W, x, _dev(np.array([0, N], dtype=np.int32)))
    for part in (slice(0, 40), slice(N - 700, N)):
        n = part.stop - part.start
        assert torch.equal(y[part], moe.moe_expert_ffn(W, x[part].clone(), _dev(np.array([0, n], dtype=np.int32))))


def test_rows_past_a_launch(moe):
    T, d = (1 << 20) + 37, 64
    g = torch.Generator("cuda").manual_seed(4)
    x, y = (torch.randn((T, d), device="cuda", generator=g) for _ in range(2))
    gate = torch.rand(T, device="cuda", generator=g)
    whole = moe.moe_block_norm(x, y, norm_after=True, row_gate=gate, int8=True, h_dtype=BF16)
    codes, scales = moe.moe_int8_quantize_rows(x)
    back = moe.moe_int8_dequantize_rows(codes, scales, dtype=F32)
    part = slice((1 << 20) - 5, T)
    px, py, pg = x[part].clone(), y[part].clone(), gate[part].clone()
    alone = moe.moe_block_norm(px, py, norm_after=True, row_gate=pg, int8=True, h_dtype=BF16)
    for n in ("x", "h", "codes", "scales"):
        assert torch.equal(whole[n][part], alone[n])
    q, s = moe.moe_int8_quantize_rows(px)
    assert torch.equal(codes[part], q) and torch.equal(scales[part], s)
    assert torch.equal(back[part], moe.moe_int8_dequantize_rows(q, s, dtype=F32))
