"""4-bit (MXFP4) expert matrices on the GPU against 64-bit references: the conversions, the expert
FFN of either kernel family, the layer in one call, and the layer calls on such a handle."""
import numpy as np
import pytest
import torch

import mxfp4_ref as ref
import paper_2402_07033_amd as moe
from gpu_util import to_dev, to_host

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def pack(conv):
    return moe.moe_weights_pack_mxfp4(*[(cuda(c), cuda(s)) for c, s in conv])


def rows(rng, n, d, dtype):
    """Activations as the kernels get them, and their 64-bit values."""
    x = rng.standard_normal((n, d)).astype(np.float32)
    if dtype == BF16:
        x = ref.bf16(x)
        return cuda(x).to(BF16), x.astype(np.float64)
    return cuda(x), x.astype(np.float64)


def check(got, want, bound, dtype=F32, what=""):
    got = got.float().cpu().numpy().astype(np.float64)
    # y is rounded once more to its type
    room = bound + (2.0 ** -8 if dtype == BF16 else 2.0 ** -24) * (np.abs(want) + bound) + 1e-30
    worst = float(np.max(np.abs(got - want) / room)) if want.size else 0.0
    assert np.isfinite(got).all() and worst <= 1.0, (what, worst)


# ---- the conversions -------------------------------------------------------------------

def special_matrix(E, K, C, seed):
    """Blocks of every kind: ordinary, zeros, ties of every pair of neighbours, values that
    saturate, powers of two and their neighbours, tiny ones."""
    rng = np.random.default_rng(seed)
    w = rng.standard_normal((E, K, C)).astype(np.float32)
    w *= np.exp2(rng.integers(-20, 20, size=(E, K // 32, 1, C))).astype(np.float32).repeat(32, axis=2).reshape(E, K, C)
    b = w.reshape(E, K // 32, 32, C)
    kind = rng.integers(0, 7, size=(E, K // 32, C))
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5, 7.0, 7.5, 0.0, -0.0, 0.5, 1.0, 6.0, 4.0], dtype=np.float32)
    for e, blk, c in zip(*np.nonzero(kind < 5)):
        col = {0: np.zeros(32), 1: np.concatenate([ties, -ties]) * 2.0 ** rng.integers(-30, 30),
               2: np.exp2(rng.integers(-6, 3, size=32)) * rng.choice([-1, 1], size=32),
               3: np.nextafter(np.exp2(rng.integers(-4, 3, size=32)).astype(np.float32), np.float32(rng.choice([0, 9]))),
               4: rng.standard_normal(32) * 2.0 ** -120}[int(kind[e, blk, c])]
        b[e, blk, :, c] = col.astype(np.float32)
    return w


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("E,K,C", [(1, 32, 1), (2, 64, 13), (1, 96, 64), (3, 256, 65), (2, 288, 200), (1, 4096, 48)])
def test_conversion_is_exact(E, K, C, dtype):
    w = special_matrix(E, K, C, seed=E * 1000 + K + C)
    if dtype == BF16:
        w = ref.bf16(w)
    codes, scales = ref.quantize(w)
    got_c, got_s = moe.moe_mxfp4_quantize(cuda(w).to(dtype))
    assert np.array_equal(got_s.cpu().numpy(), scales)
    assert np.array_equal(got_c.cpu().numpy(), codes)
    for out in (F32, BF16):
        v = moe.moe_mxfp4_dequantize(got_c, got_s, dtype=out)
        assert v.dtype == out and np.array_equal(v.float().cpu().numpy(), ref.dequantize(codes, scales).astype(np.float32))


def test_every_code_and_scale_widens_exactly():
    scales = np.arange(1, 253, dtype=np.uint8).reshape(1, 252, 1)
    codes = np.tile(np.arange(16, dtype=np.uint8) * 0x11, (1, 252, 1))
    v = moe.moe_mxfp4_dequantize(cuda(codes), cuda(scales))
    want = ref.dequantize(codes, scales)
    got = v.float().cpu().numpy()
    # bf16 holds them all; the smallest is 0.5 * 2^-126, and fp32 holds it as a subnormal
    assert np.array_equal(got.astype(np.float64), want)


def test_conversion_writes_nothing_else():
    w = torch.randn((2, 96, 13), device="cuda")
    codes = torch.full((2 * 13 * 48 + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((2 * 13 * 3 + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    c, s = codes[:2 * 13 * 48].view(2, 13, 48), scales[:2 * 13 * 3].view(2, 13, 3)
    moe.moe_mxfp4_quantize(w, c, s)
    assert (codes[2 * 13 * 48:] == 0xA5).all() and (scales[2 * 13 * 3:] == 0xA5).all()
    out = torch.full((2 * 96 * 13 + 64,), 7.0, device="cuda")
    moe.moe_mxfp4_dequantize(c, s, w=out[:2 * 96 * 13].view(2, 96, 13))
    assert (out[2 * 96 * 13:] == 7.0).all()


# ---- the expert FFN --------------------------------------------------------------------

SHAPES = [(64, 64, 1), (256, 512, 8), (320, 192, 5), (2048, 1408, 6), (4096, 448, 2), (512, 6400, 2), (192, 4160, 3)]


def split_rows(rng, N, E, how):
    if how == "one":      # all rows on one expert
        counts = np.zeros(E, dtype=np.int64)
        counts[rng.integers(E)] = N
    else:                 # uneven, some experts empty
        counts = np.bincount(rng.choice(E, size=N, p=rng.dirichlet(np.full(E, 0.5))), minlength=E)
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,how", [(1, "some"), (2, "some"), (8, "one"), (9, "one"), (16, "one"), (17, "one"), (33, "some"),
                                   (72, "some"), (72, "one")])
@pytest.mark.parametrize("d,f,E", SHAPES)
def test_stream(d, f, E, N, how, dtype):
    rng = np.random.default_rng(d + f + N)
    conv, mats = ref.matrices(d + f, E, d, f)
    W = pack(conv)
    x, x64 = rows(rng, N, d, dtype)
    offsets = split_rows(rng, N, E, how)
    assert moe.moe_expert_ffn_plan(N, E, d, f, moe.MOE_MXFP4, moe.MOE_FFN_STREAM)["path"] == moe.MOE_FFN_STREAM
    yg = moe.moe_expert_ffn(W, x, cuda(offsets), path=moe.MOE_FFN_STREAM)
    want, bound = ref.ffn(x64, offsets, mats, 0.0 if dtype == BF16 else ref.SPLIT, ref.SPLIT)
    check(yg, want, bound, what=(d, f, E, N, how))
    # the family that the library takes, without allocation and through the parts' call: the same bits
    auto = moe.moe_expert_ffn(W, x, cuda(offsets))
    check(auto, want, bound, what=(d, f, E, N, how))
    again = torch.empty_like(yg)
    moe.moe_expert_ffn_noalloc(W, x, cuda(offsets), again)
    assert torch.equal(again, auto)
    parts = torch.empty((1,) + tuple(yg.shape), device="cuda")
    assert moe.moe_expert_ffn_parts(W, x, cuda(offsets), parts) == 1 and torch.equal(parts[0], auto)
    W.free()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,how", [(1, "some"), (15, "one"), (65, "one"), (73, "some"), (200, "some"), (517, "some"), (530, "one")])
@pytest.mark.parametrize("d,f,E", SHAPES)
def test_grouped(d, f, E, N, how, dtype):
    if N > 300 and d * f > 1 << 21:
        pytest.skip("the small shapes cover it")
    rng = np.random.default_rng(d + f + N)
    conv, mats = ref.matrices(d + f, E, d, f)
    W = pack(conv)
    x, x64 = rows(rng, N, d, dtype)
    offsets = split_rows(rng, N, E, how)
    yg = moe.moe_expert_ffn(W, x, cuda(offsets), path=moe.MOE_FFN_GROUPED)
    # up to 72 rows of a result in fp32 nothing is rounded to bf16
    exact = N <= 72
    want, bound = ref.ffn(x64, offsets, mats, 0.0 if dtype == BF16 else (ref.SPLIT if exact else ref.ROUND),
                          ref.SPLIT if exact else ref.ROUND)
    check(yg, want, bound, what=(d, f, E, N, how))
    W.free()


@pytest.mark.parametrize("T,k", [(5, 2), (90, 3)])
def test_rows_through_perm(T, k):
    """The rows read through perm: the same bits as from the gathered copy."""
    rng = np.random.default_rng(T)
    conv, _ = ref.matrices(3, 8, 320, 192)
    W = pack(conv)
    x, _ = rows(rng, T, 320, F32)
    logits = cuda(rng.standard_normal((T, 8)).astype(np.float32))
    idx, _ = moe.moe_route(logits, k)
    _, offsets, perm, _, xg = moe.moe_permute(idx, 8, x)
    a = moe.moe_expert_ffn(W, xg, offsets)
    b = moe.moe_expert_ffn_tokens(W, x, k, perm, offsets)
    assert torch.equal(a, b)
    W.free()


# ---- the layer -------------------------------------------------------------------------

LAYERS = [(1, 256, 512, 8, 2), (1, 320, 192, 64, 8), (3, 256, 512, 8, 2), (8, 192, 4160, 5, 3), (9, 256, 320, 16, 2),
          (10, 2048, 1408, 64, 6), (16, 512, 256, 20, 4), (16, 256, 512, 8, 2), (17, 256, 512, 8, 2), (11, 256, 512, 33, 6),
          (24, 320, 192, 3, 3), (40, 256, 512, 8, 1), (300, 320, 192, 64, 6), (700, 256, 448, 8, 2), (2, 64, 64, 1, 1)]


@pytest.mark.parametrize("xd,yd", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("T,d,f,E,k", LAYERS)
def test_layer(T, d, f, E, k, xd, yd):
    rng = np.random.default_rng(T + d + E)
    conv, mats = ref.matrices(d + f, E, d, f)
    W = pack(conv)
    x, x64 = rows(rng, T, d, xd)
    logits = rng.standard_normal((T, E)).astype(np.float32)
    if E > 4:
        logits[:, 1] = logits[:, 3]  # ties go to the lower index
        logits[:, E - 1] = -30.0     # an expert that nobody takes (unless k says so)
    # up to 72 rows of an fp32 result nothing is rounded to bf16; streamed bf16 results keep 16 bits of h
    exact = T * k <= 72 and yd == F32
    streams = T <= 16 and T * k <= 64 or T * k <= min(72, 4 * E)
    out = moe.moe_layer_mxfp4(W, x, cuda(logits), k, y=torch.empty((T, d), dtype=yd, device="cuda"))
    u = 0.0 if xd == BF16 else (ref.SPLIT if exact or streams else ref.ROUND)
    want = ref.layer(x64, logits, mats, k, u, ref.SPLIT if exact else ref.PAIR if streams else ref.ROUND)
    for n in ("idx", "counts", "offsets", "perm", "inv_perm"):
        assert np.array_equal(out[n].cpu().numpy(), want[n]), n
    assert np.max(np.abs(out["w"].cpu().numpy() - want["w"])) <= 2.0 ** -20
    check(out["y"], want["y"], want["bound"], yd, (T, d, f, E, k))
    # the routing calls on their own give the same bits
    idx, w = moe.moe_route(cuda(logits), k)
    assert torch.equal(idx, out["idx"]) and torch.equal(w, out["w"])
    # and so does the call itself, again
    again = moe.moe_layer_mxfp4(W, x, cuda(logits), k, y=torch.empty((T, d), dtype=yd, device="cuda"))
    assert torch.equal(again["y"], out["y"])
    W.free()


def test_layer_of_no_tokens():
    conv, _ = ref.matrices(1, 8, 64, 64)
    W = pack(conv)
    out = moe.moe_layer_mxfp4(W, torch.empty((0, 64), device="cuda"), torch.empty((0, 8), device="cuda"), 2)
    assert out["y"].shape == (0, 64) and int(out["offsets"].abs().sum()) == 0 and int(out["counts"].abs().sum()) == 0
    W.free()


@pytest.mark.parametrize("T,E,k", [(1, 8, 2), (5, 8, 2), (16, 16, 4), (10, 64, 6)])
def test_the_other_layer_calls(T, E, k):
    """moe_decode_layer and moe_layer on a 4-bit handle."""
    d, f = 320, 448
    rng = np.random.default_rng(T + E)
    conv, mats = ref.matrices(T, E, d, f)
    W = pack(conv)
    x, x64 = rows(rng, T, d, F32)
    logits = rng.standard_normal((T, E)).astype(np.float32)
    want = ref.layer(x64, logits, mats, k, ref.SPLIT, ref.SPLIT)
    yg = torch.empty((T * k, d), device="cuda")
    a = moe.moe_decode_layer(W, x, cuda(logits), k, yg=yg, want_xg=True)
    b = moe.moe_layer(W, x, cuda(logits), k)
    for out in (a, b):
        check(out["y"], want["y"], want["bound"])
        check(out["yg"], want["yg"], want["yg_bound"])
        for n in ("idx", "counts", "offsets", "perm", "inv_perm"):
            assert np.array_equal(out[n].cpu().numpy(), want[n]), n
        assert torch.equal(out["xg"], x[(out["perm"] // k).long()])
    one = moe.moe_layer_mxfp4(W, x, cuda(logits), k)
    assert torch.equal(one["y"], a["y"])
    W.free()


@pytest.mark.parametrize("T,E,k,d,f", [(1, 8, 2, 256, 512), (2, 16, 2, 320, 448), (4, 4, 1, 1024, 192), (1, 8, 4, 2048, 1408),
                                       (4, 16, 1, 320, 192), (1, 3, 1, 64, 4160), (2, 16, 2, 4096, 192)])
def test_stack(T, E, k, d, f):
    """A stack of blocks in two launches each, against the same stack in separate calls and in 64 bits."""
    rng = np.random.default_rng(T + E)
    layers, want = [], None
    x, x64 = rows(rng, T, d, F32)
    for n in range(3):
        conv, mats = ref.matrices(10 + n, E, d, f)
        wg = (rng.standard_normal((d, E)) / np.sqrt(d)).astype(np.float32)
        layers.append((pack(conv), cuda(wg), mats, wg.astype(np.float64)))
    assert moe.moe_decode_block_supported(T, E, k, d, f, moe.MOE_MXFP4)
    dev = [(W, wg) for W, wg, _, _ in layers]
    idx = []
    fused = moe.moe_stack_forward(dev, x.clone(), k, idx_out=idx)
    apart = moe.moe_stack_forward(dev, x.clone(), k, fused=False)
    want = x64
    for n, (_, _, mats, wg) in enumerate(layers):
        h = want / np.sqrt((want * want).mean(axis=1, keepdims=True) + 1e-5)
        lg = h @ wg
        top = np.sort(lg, axis=1)
        assert (top[:, E - k] - top[:, E - k - 1] > 1e-3).all() if k < E else True  # no choice hangs on a rounding
        out = ref.layer(h, lg.astype(np.float32), mats, k, ref.SPLIT, ref.SPLIT)
        assert np.array_equal(idx[n].cpu().numpy(), out["idx"])
        want = want + out["y"]
    # the norms and sums of a block are fp32 (K * 2^-24 at most, K up to 2048), in three blocks
    for got in (fused, apart):
        err = np.linalg.norm(got.cpu().numpy() - want) / np.linalg.norm(want)
        assert err <= 2.0 ** -15, err
    for W, *_ in layers:
        W.free()


# ---- streams, graphs, neighbours ---------------------------------------------------------

@pytest.mark.parametrize("T,E,k", [(1, 8, 2), (7, 16, 2), (30, 8, 2), (200, 8, 2)])
def test_graph_replays(T, E, k):
    """Captured, replayed with other inputs and other work between the replays: every replay as the eager call."""
    d, f = 256, 2112
    conv, _ = ref.matrices(5, E, d, f)
    W = pack(conv)
    ws = torch.empty(moe.moe_layer_mxfp4_workspace(T, E, k, d, f), dtype=torch.uint8, device="cuda")
    x, logits = torch.randn((T, d), device="cuda"), torch.randn((T, E), device="cuda")
    out = moe.moe_layer_mxfp4(W, x, logits, k, workspace=ws)
    bufs = dict(idx=out["idx"], weights=out["w"], out=tuple(out[n] for n in ("counts", "offsets", "perm", "inv_perm")),
                workspace=ws, y=out["y"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        moe.moe_layer_mxfp4(W, x, logits, k, **bufs)
    for _ in range(4):
        x.normal_()
        logits.normal_()
        want = moe.moe_layer_mxfp4(W, x, logits, k)
        torch.cuda.synchronize()
        out["y"].fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out["y"], want["y"]) and torch.equal(out["idx"], want["idx"])
    W.free()


def test_two_streams():
    """Two calls at once on one handle, each with its own workspace."""
    conv, _ = ref.matrices(6, 8, 512, 2112)
    W = pack(conv)
    xs = [torch.randn((4, 512), device="cuda") for _ in range(2)]
    ls = [torch.randn((4, 8), device="cuda") for _ in range(2)]
    want = [moe.moe_layer_mxfp4(W, x, lg, 2)["y"] for x, lg in zip(xs, ls)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        for s, x, lg in zip(streams, xs, ls):
            with torch.cuda.stream(s):
                got.append(moe.moe_layer_mxfp4(W, x, lg, 2)["y"])
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i % 2]) for i, y in enumerate(got))
    W.free()


@pytest.mark.parametrize("path", [moe.MOE_FFN_STREAM, moe.MOE_FFN_GROUPED])
def test_scratch_is_written_before_it_is_read(path):
    """A workspace full of NaN and one full of zeros give the same bits, and nothing past yg is written."""
    conv, _ = ref.matrices(7, 5, 320, 448)
    W = pack(conv)
    x = torch.randn((37, 320), device="cuda")
    offsets = cuda(np.array([0, 5, 5, 22, 36, 37], dtype=np.int32))
    need = moe.moe_expert_ffn_workspace(37, 5, 320, 448)
    got = []
    for fill in (0xFF, 0):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        yg = torch.full((37 * 320 + 64,), 7.0, device="cuda")
        moe.moe_expert_ffn(W, x, offsets, workspace=ws, yg=yg[:37 * 320].view(37, 320), path=path)
        assert (yg[37 * 320:] == 7.0).all()
        got.append(yg)
    assert torch.equal(*got)
    W.free()


def test_quantize_then_layer():
    """As a program uses them together: bf16 matrices converted, packed, and a layer run on them."""
    E, d, f, T, k = 4, 256, 512, 6, 2
    rng = np.random.default_rng(0)
    ws = [ref.bf16(rng.standard_normal(s).astype(np.float32) / np.sqrt(s[1])) for s in ((E, d, f), (E, d, f), (E, f, d))]
    W = moe.moe_weights_pack_mxfp4(*[moe.moe_mxfp4_quantize(cuda(w).to(BF16)) for w in ws])
    x, x64 = rows(rng, T, d, BF16)
    logits = rng.standard_normal((T, E)).astype(np.float32)
    out = moe.moe_layer_mxfp4(W, x, cuda(logits), k)
    mats = [ref.dequantize(*ref.quantize(w)) for w in ws]
    want = ref.layer(x64, logits, mats, k, 0.0, ref.PAIR)
    check(out["y"], want["y"], want["bound"], BF16)
    W.free()


# ---- calls that the documentation allows and that go wrong easily -----------------------

@pytest.mark.parametrize("N,path", [(7, moe.MOE_FFN_STREAM), (7, moe.MOE_FFN_GROUPED), (200, moe.MOE_FFN_GROUPED)])
def test_rows_behind_the_last_expert_stay(N, path):
    """A padded batch: what offsets do not cover is left as it was, whatever the workspace holds."""
    E, d, f = 3, 256, 4096  # both families cut the second projection's reduction at this f
    conv, mats = ref.matrices(8, E, d, f)
    W = pack(conv)
    rng = np.random.default_rng(N)
    x, x64 = rows(rng, N, d, BF16)
    used = N - 3
    offsets = np.array([0, 1, 1, used], dtype=np.int32)
    ws = torch.full((moe.moe_expert_ffn_workspace(N, E, d, f),), 0xFF, dtype=torch.uint8, device="cuda")
    yg = torch.full((N, d), 7.0, device="cuda")
    moe.moe_expert_ffn(W, x, cuda(offsets), workspace=ws, yg=yg, path=path)
    assert (yg[used:] == 7.0).all()
    want, bound = ref.ffn(x64, offsets, mats, 0.0, ref.SPLIT if N <= 72 else ref.ROUND)
    check(yg[:used], want[:used], bound[:used])
    # and none at all
    yg.fill_(7.0)
    moe.moe_expert_ffn(W, x, cuda(np.zeros(E + 1, dtype=np.int32)), workspace=ws, yg=yg, path=path)
    assert (yg == 7.0).all()
    W.free()


@pytest.mark.parametrize("T", [5, 40])
@pytest.mark.parametrize("what", ["nan logits", "masked logits", "nan row", "infinite row"])
def test_a_bad_token_stays_alone(T, what):
    """Logits that are NaN or -infinity, rows that are NaN or infinite: the other tokens' results hold."""
    E, d, f, k = 8, 320, 448, 2
    conv, mats = ref.matrices(9, E, d, f)
    W = pack(conv)
    rng = np.random.default_rng(T)
    x, x64 = rows(rng, T, d, F32)
    logits = rng.standard_normal((T, E)).astype(np.float32)
    bad = 3
    given = logits.copy()
    if what == "nan logits":
        given[bad] = np.nan
    elif what == "masked logits":
        given[bad] = -np.inf
        given[:, 5] = logits[:, 5] = -np.inf  # an expert that nobody may take
    else:
        x[bad] = float("nan") if what == "nan row" else float("inf")
    out = moe.moe_layer_mxfp4(W, x, cuda(given), k)
    idx = out["idx"].cpu().numpy()
    # (moe_route, which more than 16 tokens go through, leaves the ids of NaN logits unspecified; the batching
    # clamps them, so the slots' order is one all the same)
    if what != "nan logits" or T <= 16:
        assert idx.min() >= 0 and idx.max() < E
    assert np.array_equal(np.sort(out["perm"].cpu().numpy()), np.arange(T * k))
    others = np.arange(T) != bad
    exact = T * k <= 72
    streams = T <= 16 or T * k <= min(72, 4 * E)
    want = ref.layer(x64, np.where(np.isfinite(logits), logits, -1e30), mats, k,
                     ref.SPLIT if exact or streams else ref.ROUND, ref.SPLIT if exact else ref.ROUND)
    assert np.array_equal(idx[others], want["idx"][others])
    check(out["y"][cuda(others)], want["y"][others], want["bound"][others])
    W.free()


@pytest.mark.parametrize("T", [3, 200])
def test_two_graphs_share_a_workspace(T):
    """Replayed in turn on one stream, neither keeps anything in it for its next replay."""
    E, k, d, f = 8, 2, 256, 2112
    conv, _ = ref.matrices(10, E, d, f)
    W = pack(conv)
    ws = torch.empty(moe.moe_layer_mxfp4_workspace(T, E, k, d, f), dtype=torch.uint8, device="cuda")
    small = max(1, T // 2)  # the second graph has another layout of the same memory
    runs = []
    for n in (T, small):
        x, logits = torch.randn((n, d), device="cuda"), torch.randn((n, E), device="cuda")
        out = moe.moe_layer_mxfp4(W, x, logits, k, workspace=ws)
        want = out["y"].clone()
        bufs = dict(idx=out["idx"], weights=out["w"], out=tuple(out[m] for m in ("counts", "offsets", "perm", "inv_perm")),
                    workspace=ws, y=out["y"])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            moe.moe_layer_mxfp4(W, x, logits, k, **bufs)
        runs.append((g, out["y"], want, x, logits, bufs))
    for _ in range(4):
        for g, y, want, *_ in runs:
            y.fill_(float("nan"))
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, want) for _, y, want, *_ in runs)
        ws.fill_(0xFF)
    W.free()


@pytest.mark.parametrize("path", [moe.MOE_FFN_STREAM, moe.MOE_FFN_GROUPED])
def test_matrices_past_32_bits(path):
    """64 experts of 4096 x 16384: 4 GiB of first-projection codes, and rows on the last experts."""
    E, d, f, N = 64, 4096, 16384, 3
    gen = torch.Generator(device="cuda").manual_seed(3)
    conv = []
    for K, C in ((d, f), (d, f), (f, d)):
        codes = torch.randint(0, 256, (E, C, K // 2), dtype=torch.uint8, device="cuda", generator=gen)
        scales = torch.randint(119, 121, (E, C, K // 32), dtype=torch.uint8, device="cuda", generator=gen)
        conv.append((codes, scales))
    W = moe.moe_weights_pack_mxfp4(*conv)
    rng = np.random.default_rng(0)
    x, x64 = rows(rng, N, d, BF16)
    offsets = np.zeros(E + 1, dtype=np.int32)
    offsets[E - 1], offsets[E] = 1, N  # expert 62: row 0, expert 63: rows 1 and 2
    yg = moe.moe_expert_ffn(W, x, cuda(offsets), path=path)
    for e, lo, hi in ((62, 0, 1), (63, 1, 3)):
        mats = [ref.dequantize(c[e:e + 1].cpu().numpy(), s[e:e + 1].cpu().numpy())[0] for c, s in conv]
        want, bound = ref.expert(x64[lo:hi], *mats, 0.0, ref.SPLIT)
        check(yg[lo:hi], want, bound, what=e)
    W.free()


def test_tensors_that_are_refused():
    conv, _ = ref.matrices(11, 4, 64, 64)
    W = pack(conv)
    x, logits = torch.randn((6, 64), device="cuda"), torch.randn((6, 4), device="cuda")
    for bad in (dict(x=torch.randn((64, 6), device="cuda").t()), dict(logits=torch.randn((4, 6), device="cuda").t()),
                dict(x=x.cpu()), dict(logits=logits.double()), dict(x=x[:, :32].contiguous()), dict(logits=logits[:, :3].contiguous()),
                dict(x=x.half())):
        with pytest.raises((ValueError, TypeError)):
            moe.moe_layer_mxfp4(W, **{**dict(x=x, logits=logits), **bad}, k=2)
    # the layer may not write where it reads
    with pytest.raises(moe.MoeError):
        moe.moe_layer_mxfp4(W, x, logits, 2, y=x)
    W.free()
