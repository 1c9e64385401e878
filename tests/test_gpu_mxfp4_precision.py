"""What the kernels over 4-bit expert matrices keep of rows and of h = silu(a)*b: 24 bits where the result is
fp32, 16 where it is bf16, at any number of rows.

Two kinds of inputs.  `Picked`: every row has one value and every column of w2 one element, so that no sum
hides what an operand lost, and the result is held to a few fp32 roundings.  Dense ones: against the bounds
of mxfp4_ref, after a look (in the reference, on the CPU) that the bounds would show a result of zeros and
one that leaves out a scale block of the rows."""
import numpy as np
import pytest
import torch

import mxfp4_ref as ref
import paper_2402_07033_amd as moe
from test_gpu_mxfp4 import check, cuda, pack, rows, split_rows

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def keep(v, parts):
    """fp64 values with what `parts` bf16 parts hold of them."""
    out = np.zeros_like(v)
    for _ in range(parts):
        out = out + ref.bf16((v - out).astype(np.float32)).astype(np.float64)
    return out


class Picked:
    """Row n is x[n] in column at[n], else zero; column c of an expert's w2 has one element, in row src[c].
    w1 is positive, so a > 0 and silu is no worse conditioned than 1.3."""

    def __init__(self, seed, E, d, f, N):
        rng = np.random.default_rng(seed)

        def codes(shape, low):
            c = rng.integers(1, 8, size=shape, dtype=np.uint8) | (rng.integers(0, 2, size=shape, dtype=np.uint8) << 3) * low
            return c[..., 0::2] | (c[..., 1::2] << 4)

        def scales(shape):
            return rng.integers(125, 129, size=shape).astype(np.uint8)
        w1 = codes((E, f, d), 0), scales((E, f, d // 32))
        w3 = codes((E, f, d), 1), scales((E, f, d // 32))
        self.src = rng.integers(0, f, size=(E, d))
        c2 = np.zeros((E, d, f), dtype=np.uint8)
        np.put_along_axis(c2, self.src[..., None], rng.integers(1, 8, size=(E, d, 1), dtype=np.uint8), axis=2)
        w2 = c2[..., 0::2] | (c2[..., 1::2] << 4), scales((E, d, f // 32))
        self.conv = [w1, w3, w2]
        self.vals = [ref.dequantize(*m) for m in self.conv]
        self.at = rng.integers(0, d, size=N)
        # 24 bits each, the lowest set
        self.x = np.zeros((N, d), dtype=np.float32)
        top = np.ldexp((rng.integers(1 << 23, 1 << 24, size=N) | 1).astype(np.float64), -23 - rng.integers(0, 3, size=N))
        self.x[np.arange(N), self.at] = top

    def result(self, expert, x_parts=3, h_parts=3, bf16_rows=False):
        """yg in 64 bits, rows and h as so many bf16 parts (3: all of an fp32 value)."""
        n = np.arange(len(expert))
        v = self.x[n, self.at].astype(np.float64)
        v = keep(v, 1 if bf16_rows else x_parts)
        a = v[:, None] * self.vals[0][expert, self.at]
        b = v[:, None] * self.vals[1][expert, self.at]
        h = keep((ref.silu(a) * b).astype(np.float32).astype(np.float64), h_parts)
        src = self.src[expert]
        return np.take_along_axis(h, src, axis=1) * np.take_along_axis(self.vals[2][expert], src[:, None], axis=1)[:, 0]


# Roundings of a result over `Picked`, in steps of 2^-22 relative: the exact parts of x are added in two steps of
# 2^-23 for each of a and b; silu carries 1.3 times that on, its exp counts at most half a step of 2^-23 (|a e^-a| is
# below 0.3, so the argument's rounding counts less) and its sum and division 2^-24 each, the product 2^-24 and the
# parts of h two more steps of 2^-23: 1.3 + 1 + 0.5 + 0.75 + 1 = 4.55, so 2^-19.8.  Without the third part of x or h
# some elements are off by close to 2^-16.
PICKED_BOUND = 2.0 ** -19


def off(got, want):
    return float(np.max(np.abs(got - want) / np.abs(want)))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,path", [(7, moe.MOE_FFN_STREAM), (72, moe.MOE_FFN_STREAM), (7, moe.MOE_FFN_GROUPED),
                                    (72, moe.MOE_FFN_GROUPED), (73, moe.MOE_FFN_GROUPED), (200, moe.MOE_FFN_GROUPED),
                                    (1100, moe.MOE_FFN_GROUPED)])
@pytest.mark.parametrize("d,f,E", [(256, 512, 5), (320, 192, 3), (64, 4160, 2)])
def test_fp32_results_keep_24_bits(d, f, E, N, path, dtype):
    p = Picked(d + f + N, E, d, f, N)
    offsets = split_rows(np.random.default_rng(N), N, E, "some")
    expert = np.searchsorted(offsets[1:], np.arange(N), side="right")
    want = p.result(expert, bf16_rows=dtype == BF16)
    if dtype == F32:
        assert off(p.result(expert, x_parts=2), want) > 2 * PICKED_BOUND
    assert off(p.result(expert, h_parts=2, bf16_rows=dtype == BF16), want) > 2 * PICKED_BOUND
    W = pack(p.conv)
    yg = moe.moe_expert_ffn(W, cuda(p.x).to(dtype), cuda(offsets), path=path)
    assert off(yg.cpu().numpy().astype(np.float64), want) <= PICKED_BOUND
    W.free()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d,f,E,N,how", [(2048, 1408, 6, 73, "some"), (2048, 1408, 6, 200, "some"), (512, 6400, 2, 200, "some"),
                                         (4096, 448, 2, 330, "some"), (192, 4160, 3, 530, "one"), (256, 512, 8, 517, "some")])
def test_dense_rows_of_prompts(d, f, E, N, how, dtype):
    rng = np.random.default_rng(d + f + N)
    conv, mats = ref.matrices(d + f, E, d, f)
    x, x64 = rows(rng, N, d, dtype)
    offsets = split_rows(rng, N, E, how)
    want, bound = ref.ffn(x64, offsets, mats, 0.0 if dtype == BF16 else ref.SPLIT, ref.SPLIT)
    assert np.max(np.abs(want) / bound) > 2.0  # zeros
    cut = x64.copy()
    cut[:, -32:] = 0.0
    assert np.max(np.abs(ref.ffn(cut, offsets, mats, 0.0, 0.0)[0] - want) / bound) > 2.0
    W = pack(conv)
    check(moe.moe_expert_ffn(W, x, cuda(offsets), path=moe.MOE_FFN_GROUPED), want, bound, what=(d, f, E, N, how))
    W.free()


@pytest.mark.parametrize("xd", [F32, BF16])
@pytest.mark.parametrize("T,d,f,E,k", [(40, 256, 512, 8, 2), (130, 320, 192, 16, 3), (90, 64, 4160, 4, 1)])
def test_the_layer_in_fp32(T, d, f, E, k, xd):
    rng = np.random.default_rng(T)
    conv, mats = ref.matrices(T, E, d, f)
    x, x64 = rows(rng, T, d, xd)
    logits = rng.standard_normal((T, E)).astype(np.float32)
    want = ref.layer(x64, logits, mats, k, 0.0 if xd == BF16 else ref.SPLIT, ref.SPLIT)
    W = pack(conv)
    out = moe.moe_layer_mxfp4(W, x, cuda(logits), k, y=torch.empty((T, d), device="cuda"))
    check(out["y"], want["y"], want["bound"], what=(T, d, f, E, k))
    W.free()


# A bf16 result over `Picked`: h to 16 bits and fp32 rows to 16 at least (2^-16 each, times 1, and 1.3 + 1 for the
# rows' part in h: 2^-14.3), with the steps above 2^-14, and y's own rounding, 2^-8.  Rows or h in one part are off by
# up to 2^-8 before that rounding.
Y_BOUND = 2.0 ** -8 + 2.0 ** -14


@pytest.mark.parametrize("xd", [F32, BF16])
@pytest.mark.parametrize("T", [5, 60, 90, 300, 1500])
@pytest.mark.parametrize("d,f,E", [(256, 512, 6), (320, 192, 5), (64, 4160, 2)])
def test_bf16_results_keep_16_bits(d, f, E, T, xd):
    p = Picked(d + f + T, E, d, f, T)
    logits = np.random.default_rng(T).standard_normal((T, E)).astype(np.float32)
    expert = logits.argmax(axis=1)  # (k = 1: weight 1)
    want = p.result(expert, bf16_rows=xd == BF16)
    assert off(ref.bf16(p.result(expert, h_parts=1, bf16_rows=xd == BF16).astype(np.float32)), want) > 1.2 * Y_BOUND
    if xd == F32:
        assert off(ref.bf16(p.result(expert, x_parts=1).astype(np.float32)), want) > 1.2 * Y_BOUND
    W = pack(p.conv)
    out = moe.moe_layer_mxfp4(W, cuda(p.x).to(xd), cuda(logits), 1, y=torch.empty((T, d), dtype=BF16, device="cuda"))
    assert np.array_equal(out["idx"].cpu().numpy()[:, 0], expert)
    assert off(out["y"].float().cpu().numpy().astype(np.float64), want) <= Y_BOUND
    W.free()


# ---- scales at the ends of the format: other converters write them, 0 for blocks of zeros among others ----

def test_every_scale_byte():
    scales = np.arange(256, dtype=np.uint8).reshape(1, 256, 1)
    codes = np.tile(np.arange(16, dtype=np.uint8) * 0x11, (1, 256, 1))
    want = ref.dequantize(codes, scales)
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
    want[..., 255] = np.nan
    for dtype in (F32, BF16):
        got = moe.moe_mxfp4_dequantize(cuda(codes), cuda(scales), dtype=dtype).float().cpu().numpy()
        assert np.array_equal(got.astype(np.float64), want, equal_nan=True)


@pytest.mark.parametrize("path", [moe.MOE_FFN_STREAM, moe.MOE_FFN_GROUPED])
@pytest.mark.parametrize("byte,dtype", [(0, F32), (0, BF16), (1, F32), (230, F32), (252, BF16)])
def test_scales_at_the_ends_in_products(byte, dtype, path):
    """w1 and w3 of one scale, rows that undo it: subnormal weights are not lost on the matrix cores.  (fp32 rows end at
    2^-104 here: what lies below 2^-133 of a row is none of its parts'.)"""
    p = Picked(byte, 2, 64, 64, 9)
    for n in (0, 1):
        p.conv[n] = (p.conv[n][0], np.full_like(p.conv[n][1], byte))
        p.vals[n] = ref.dequantize(*p.conv[n])
    p.x *= np.float32(2.0) ** np.float32(min(127 - byte, 126))
    assert np.isfinite(p.x).all()
    # a block of zeros, as a converter may write it: scale 0, codes 0
    p.conv[2][1][:, :, 1][(p.conv[2][0].reshape(2, 64, 2, 16)[:, :, 1] == 0).all(axis=2)] = 0
    p.vals[2] = ref.dequantize(*p.conv[2])
    offsets = np.array([0, 4, 9], dtype=np.int32)
    want = p.result(np.repeat([0, 1], [4, 5]), bf16_rows=dtype == BF16)
    W = pack(p.conv)
    yg = moe.moe_expert_ffn(W, cuda(p.x).to(dtype), cuda(offsets), path=path)
    assert off(yg.cpu().numpy().astype(np.float64), want) <= PICKED_BOUND
    W.free()


@pytest.mark.parametrize("path", [moe.MOE_FFN_STREAM, moe.MOE_FFN_GROUPED])
@pytest.mark.parametrize("d,f", [(64, 192), (320, 64), (4096, 64)])
def test_zero_padding_is_kept_from_infinite_weights(d, f, path):
    """Infinite weights in the last block of a reduction that ends inside a fragment reach the rows that have them only."""
    E, N = 2, 5
    conv, mats = ref.matrices(1, E, d, f)
    conv[0][1][1, :, -1] = 254   # expert 1's first projection
    conv[0][0][1, :, -16:] = 0x77
    W = pack(conv)
    x, x64 = rows(np.random.default_rng(0), N, d, F32)
    offsets = np.array([0, 3, 5], dtype=np.int32)
    yg = moe.moe_expert_ffn(W, x, cuda(offsets), path=path).cpu().numpy().astype(np.float64)
    want, bound = ref.ffn(x64[:3], offsets[[0, 1]], [m[:1] for m in mats], ref.SPLIT, ref.SPLIT)
    assert (np.abs(yg[:3] - want) <= bound + 2.0 ** -24 * np.abs(want)).all()
    assert not np.isfinite(yg[3:]).any()
    W.free()


# ---- values past the types: what is infinite in 64-bit arithmetic rounded to the result's type is infinite ----

def positive(seed, E, d, f):
    """Matrices without a zero and without a sign: no sum is inf - inf or inf * 0."""
    rng = np.random.default_rng(seed)
    conv = []
    for K, C in ((d, f), (d, f), (f, d)):
        c = rng.integers(1, 8, size=(E, C, K), dtype=np.uint8)
        conv.append((c[..., 0::2] | (c[..., 1::2] << 4), rng.integers(120, 123, size=(E, C, K // 32)).astype(np.uint8)))
    return conv, [ref.dequantize(*m) for m in conv]


@pytest.mark.parametrize("xd,yd", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("T", [4, 60, 300])
@pytest.mark.parametrize("d,f", [(192, 320), (256, 512)])
def test_infinite_rows_and_products(d, f, T, xd, yd):
    """Row 1 holds an infinity, row 2 overflows h, row 3 holds a NaN; the others are ordinary."""
    E = 3
    conv, mats = positive(d + T, E, d, f)
    W = pack(conv)
    rng = np.random.default_rng(T)
    x = ref.bf16(rng.uniform(0.0, 1.0, size=(T, d)).astype(np.float32))
    x[1, 7], x[2], x[3, d - 1] = np.inf, 2.0 ** 90, np.nan
    logits = rng.standard_normal((T, E)).astype(np.float32)
    ordinary = np.arange(T)
    ordinary = ordinary[(ordinary < 1) | (ordinary > 3)]
    safe = x.astype(np.float64)
    safe[1:4] = 0.0
    parts = ref.SPLIT if yd == F32 else ref.PAIR
    want = ref.layer(safe, logits, mats, 1, 0.0, parts)
    calls = [moe.moe_layer_mxfp4(W, cuda(x).to(xd), cuda(logits), 1, y=torch.empty((T, d), dtype=yd, device="cuda"))["y"]]
    if yd == F32:  # either family, whatever the layer took
        xg, offsets, inv = cuda(x).to(xd)[cuda(want["perm"]).long()], cuda(want["offsets"]), cuda(want["inv_perm"]).long()
        for path in (moe.MOE_FFN_STREAM, moe.MOE_FFN_GROUPED)[T > 72:]:
            calls.append(moe.moe_expert_ffn(W, xg, offsets, path=path)[inv])
    for y in calls:
        check(y[cuda(ordinary)], want["y"][ordinary], want["bound"][ordinary], yd)
        got = y[1:4].float().cpu().numpy()
        assert np.isposinf(got[:2]).all() and np.isnan(got[2]).all()
    W.free()
