"""8-bit integer conversions, products, experts and the layer over them against 64-bit references."""
import numpy as np
import pytest
import torch

import int8_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    import paper_2402_07033_amd as m
    m.lib()
    return m


def _rng(*seed):
    return np.random.Generator(np.random.Philox(key=[sum(v * 1009 ** i for i, v in enumerate(seed)), 77]))


def _values(rng, shape, dtype, std=1.0):
    v = (rng.standard_normal(shape) * std).astype(np.float32)
    return ref.bf16(v) if dtype == torch.bfloat16 else v


def _dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _pair(q, s):
    return _dev(q), _dev(s)


def _host(t):
    return t.float().cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy()


def _same(got, want):
    np.testing.assert_array_equal(got.view(np.int32) if got.dtype == np.float32 else got,
                                  want.view(np.int32) if want.dtype == np.float32 else want)


F32, BF16 = torch.float32, torch.bfloat16


# ---- conversions -----------------------------------------------------------------------

@pytest.mark.parametrize("T,K", [(1, 16), (3, 48), (17, 64), (5, 1408), (2, 4096), (3, 14336), (2, 20000), (1, 131072)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows(moe, T, K, dtype):
    rng = _rng(1, T, K)
    x = _values(rng, (T, K), dtype)
    x[0, : K // 2] *= 2.0 ** -20
    q, s = ref.quantize(x)
    codes, scales = moe.moe_int8_quantize_rows(_dev(x, dtype))
    _same(_host(scales), s)
    _same(_host(codes), q)
    back = (q.astype(np.float32) * s[:, None]).astype(np.float32)
    _same(_host(moe.moe_int8_dequantize_rows(codes, scales, dtype=F32)), back)
    _same(_host(moe.moe_int8_dequantize_rows(codes, scales, dtype=BF16)), ref.bf16(back))


def test_rows_special(moe):
    """Borders between codes, all zeros, subnormal and huge rows, NaN and infinities."""
    K, rows = 256, []
    half = np.arange(-127, 127, dtype=np.float32) + np.float32(0.5)
    for step in (1.0, 2.0 ** -30, 2.0 ** 90, 2.0 ** -149, 3 * 2.0 ** -147):   # ties exactly on the borders
        r = np.zeros(K, dtype=np.float64)
        r[:254], r[254] = half * step, 127.0 * step
        rows.append(r.astype(np.float32))
    for s in (np.float32(0.0123456), np.float32(7.7e-39), np.float32(1.7e36)):  # next to them
        r = np.zeros(K, dtype=np.float32)
        r[0] = np.float32(127) * s
        b = (half[:250].astype(np.float64) * float((np.abs(r[0]) / np.float32(127)).astype(np.float32))).astype(np.float32)
        r[1:251] = np.nextafter(b, np.where(np.arange(250) % 3 == 0, np.float32(np.inf), np.where(np.arange(250) % 3 == 1, np.float32(-np.inf), b)).astype(np.float32))
        rows.append(r)
    rows += [np.zeros(K), np.full(K, -0.0), np.full(K, 1e-45), np.full(K, 3.4e38)]
    for bad in (np.nan, np.inf, -np.inf):
        r = np.ones(K)
        r[77] = bad
        rows.append(r)
    x = np.stack([np.asarray(r, dtype=np.float32) for r in rows])
    q, s = ref.quantize(x)
    codes, scales = moe.moe_int8_quantize_rows(_dev(x))
    got = _host(scales)
    assert np.array_equal(np.isnan(got), np.isnan(s)) and np.isnan(s[-3:]).all() and not np.isnan(s[:-3]).any()
    _same(np.nan_to_num(got), np.nan_to_num(s))
    _same(_host(codes), q)
    # the same values as channels of a matrix
    codes, scales = moe.moe_int8_quantize(_dev(x.T[None]))
    _same(np.nan_to_num(_host(scales))[0], np.nan_to_num(s))
    _same(_host(codes)[0], q)


@pytest.mark.parametrize("E,K,C", [(1, 16, 1), (2, 48, 63), (3, 256, 65), (1, 272, 129), (2, 528, 100), (1, 4096, 200), (5, 64, 64),
                                   (1, 6144, 33), (1, 20000, 17)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_matrices(moe, E, K, C, dtype):
    w = _values(_rng(2, E, K, C), (E, K, C), dtype, K ** -0.5)
    w[0, :, 0] = 0.0
    q, s = ref.matrix(w)
    codes, scales = moe.moe_int8_quantize(_dev(w, dtype))
    _same(_host(scales), s)
    _same(_host(codes), q)
    back = np.ascontiguousarray((q.astype(np.float32) * s[..., None]).transpose(0, 2, 1))
    _same(_host(moe.moe_int8_dequantize(codes, scales, dtype=F32)), back)
    _same(_host(moe.moe_int8_dequantize(codes, scales, dtype=BF16)), ref.bf16(back))


# ---- products --------------------------------------------------------------------------

def _offsets(rng, E, M, empty=()):
    c = np.zeros(E, dtype=np.int64)
    live = [e for e in range(E) if e not in empty]
    np.add.at(c, rng.choice(live, size=M), 1)
    return np.concatenate([[0], np.cumsum(c)]).astype(np.int32)


def _check_product(moe, q, s, codes, scales, offsets, dtype, M_used=None):
    M, C = q.shape[0], codes.shape[1]
    y = torch.full((M, C), 7.0, dtype=dtype, device="cuda")
    off = None if offsets is None else _dev(offsets)
    moe.moe_int8_matmul(_pair(q, s), _pair(codes, scales), offsets=off, y=y)
    got = _host(y).astype(np.float64)
    ends = [0, M] if offsets is None else [int(v) for v in offsets]
    for e, (a, b) in enumerate(zip(ends, ends[1:])):
        want = ref.product(q[a:b], s[a:b], codes[e], scales[e])
        bound = (ref.PRODUCT + (ref.BF16 if dtype == BF16 else 0)) * 1.01 * np.abs(want) + 1e-44
        assert (np.abs(got[a:b] - want) <= bound).all(), (e, np.max(np.abs(got[a:b] - want) - bound))
    assert (got[ends[-1]:] == 7.0).all()
    return y


@pytest.mark.parametrize("M,K,C", [(1, 16, 1), (1, 4096, 4096), (2, 64, 16), (3, 80, 17), (7, 112, 255), (15, 192, 256), (16, 256, 257),
                                   (17, 1024, 100), (33, 2048, 1407), (64, 96, 513), (65, 320, 64), (77, 4096, 48), (129, 576, 300),
                                   (255, 256, 256), (257, 128, 511), (300, 1408, 96), (513, 272, 130), (1000, 64, 33)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_product(moe, M, K, C, dtype):
    rng = _rng(3, M, K, C)
    q, s = ref.quantize(_values(rng, (M, K), F32))
    codes, scales = ref.quantize(_values(rng, (1, C, K), F32, K ** -0.5))
    _check_product(moe, q, s, codes, scales, None, dtype)


@pytest.mark.parametrize("E,M,K,C,empty", [(4, 1, 64, 48, ()), (16, 9, 128, 33, (0, 15)), (8, 40, 4096, 80, (3,)), (64, 100, 80, 64, ()),
                                           (3, 600, 192, 100, (1,)), (16, 333, 2048, 1407, ()), (2, 1200, 64, 257, ())])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_product_of_experts(moe, E, M, K, C, empty, dtype):
    rng = _rng(4, E, M, K, C)
    q, s = ref.quantize(_values(rng, (M + 5, K), F32))
    codes, scales = ref.quantize(_values(rng, (E, C, K), F32, K ** -0.5))
    _check_product(moe, q, s, codes, scales, _offsets(rng, E, M, empty), dtype)  # five rows behind the last


def test_product_extremes(moe):
    """The longest sums at their largest, and rows and channels with a NaN scale."""
    M, K, C = 3, 131072, 18
    q = np.full((M, K), 127, dtype=np.int8)
    q[1] = -127
    q[2, ::2] = -127
    codes = np.full((1, C, K), 127, dtype=np.int8)
    codes[0, 5] = -127
    s, scales = np.array([1.0, 0.5, 2.0], dtype=np.float32), np.linspace(0.5, 2, C, dtype=np.float32)[None]
    _check_product(moe, q, s, codes, scales, None, F32)
    q = np.zeros((40, 64), dtype=np.int8)
    q[:] = np.arange(64)
    codes = np.ones((1, 20, 64), dtype=np.int8)
    s, scales = np.ones(40, dtype=np.float32), np.ones((1, 20), dtype=np.float32)
    s[3], scales[0, 7] = np.nan, np.nan
    y = _host(moe.moe_int8_matmul(_pair(q, s), _pair(codes, scales), dtype=F32))
    bad = np.zeros((40, 20), dtype=bool)
    bad[3], bad[:, 7] = True, True
    assert np.array_equal(np.isnan(y), bad) and (y[~bad] == 2016.0).all()


def test_no_rows(moe):
    w = (torch.ones((2, 32, 64), dtype=torch.int8, device="cuda"), torch.ones((2, 32), device="cuda"))
    x = (torch.ones((0, 64), dtype=torch.int8, device="cuda"), torch.ones((0,), device="cuda"))
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert moe.moe_int8_matmul(x, w, offsets=off).shape == (0, 32)
    y = torch.full((4, 32), 3.0, device="cuda")
    x = (torch.ones((4, 64), dtype=torch.int8, device="cuda"), torch.ones((4,), device="cuda"))
    moe.moe_int8_matmul(x, w, offsets=off, y=y)
    assert (y == 3.0).all()
    q, s = moe.moe_int8_quantize_rows(torch.empty((0, 64), device="cuda"))
    assert q.shape == (0, 64) and moe.moe_int8_dequantize_rows(q, s).shape == (0, 64)


# ---- experts and the layer -------------------------------------------------------------

def _mats(rng, E, d, f):
    return [ref.quantize(_values(rng, (E, c, k), F32, k ** -0.5)) for k, c in ((d, f), (d, f), (f, d))]


def _pack(moe, mats):
    return moe.moe_weights_pack_int8(*(_pair(*m) for m in mats))


SHAPES = [(64, 64, 1, 1), (64, 128, 3, 2), (128, 192, 8, 2), (320, 448, 16, 4), (512, 64, 5, 1), (256, 1088, 4, 2)]


@pytest.mark.parametrize("d,f,E,k", SHAPES)
@pytest.mark.parametrize("T,x_dtype", [(1, F32), (1, BF16), (2, BF16), (5, "codes"), (16, F32), (33, BF16), (90, "codes"), (301, BF16)])
def test_layer(moe, d, f, E, k, T, x_dtype):
    rng = _rng(5, d, f, E, T)
    mats = _mats(rng, E, d, f)
    W = _pack(moe, mats)
    x = _values(rng, (T, d), BF16 if x_dtype is BF16 else F32)
    q, s = ref.quantize(x)
    logits = (rng.standard_normal((T, E)) * 1.5).astype(np.float32)
    for dt in (F32, BF16):
        out = moe.moe_layer_int8(W, _pair(q, s) if x_dtype == "codes" else _dev(x, x_dtype), _dev(logits), k, dtype=dt)
        idx, w, y, bound = ref.layer(q, s, logits, k, mats, dt == BF16)
        _same(_host(out["idx"]), idx)
        assert np.abs(_host(out["w"]) - w).max() <= 1e-6
        err = np.abs(_host(out["y"]).astype(np.float64) - y) - bound
        assert (err <= 0).all(), err.max()
    # the four calls, whatever kernels they take, give the same bits: sums of integers have no order
    if x_dtype != "codes":
        lay = moe.moe_layer(W, _dev(x, x_dtype), _dev(logits), k)
        for n in ("idx", "counts", "offsets", "perm", "inv_perm"):
            _same(_host(lay[n]), _host(out[n]))
        y32 = moe.moe_layer_int8(W, _dev(x, x_dtype), _dev(logits), k, dtype=F32)["y"]
        _same(_host(lay["y"]), _host(y32))
        yg = moe.moe_expert_ffn_tokens(W, _dev(x, x_dtype), k, lay["perm"], lay["offsets"])
        _same(_host(yg), _host(lay["yg"]))


@pytest.mark.parametrize("d,f,E", [(128, 192, 4), (2048, 1408, 8)])
@pytest.mark.parametrize("N", [1, 4, 16, 17, 40, 72, 200])
def test_families_give_the_same_bits(moe, d, f, E, N):
    rng = _rng(6, d, f, N)
    W = _pack(moe, _mats(rng, E, d, f))
    off = _dev(_offsets(rng, E, N, (1,)))
    for dt in (F32, BF16):
        x = _dev(_values(rng, (N, d), dt), dt)
        auto = moe.moe_expert_ffn(W, x, off)
        for path in (moe.MOE_FFN_STREAM, moe.MOE_FFN_GROUPED):
            try:
                moe.moe_expert_ffn_plan(N, E, d, f, moe.MOE_INT8, path)
            except moe.MoeError:
                with pytest.raises(moe.MoeError):
                    moe.moe_expert_ffn(W, x, off, path=path)
                continue
            _same(_host(moe.moe_expert_ffn(W, x, off, path=path)), _host(auto))
        yg = torch.empty((N, d), dtype=F32, device="cuda")
        _same(_host(moe.moe_expert_ffn_noalloc(W, x, off, yg)), _host(auto))
        parts = torch.empty((2, N, d), dtype=F32, device="cuda")
        assert moe.moe_expert_ffn_parts(W, x, off, parts) == 1
        _same(_host(parts[0]), _host(auto))


def test_uncovered_rows_stay(moe):
    d, f, E, N = 128, 64, 3, 40
    rng = _rng(7)
    W = _pack(moe, _mats(rng, E, d, f))
    x = _values(rng, (N, d), F32)
    x[30:] = np.nan
    off = np.array([0, 11, 11, 30], dtype=np.int32)
    for path in (moe.MOE_FFN_AUTO, moe.MOE_FFN_GROUPED):
        yg = torch.full((N, d), 5.0, device="cuda")
        moe.moe_expert_ffn(W, _dev(x), _dev(off), yg=yg, path=path)
        assert (yg[30:] == 5.0).all() and torch.isfinite(yg[:30]).all()


def test_a_bad_token_stays_alone(moe):
    d, f, E, k, T = 128, 192, 4, 2, 9
    rng = _rng(8)
    W = _pack(moe, _mats(rng, E, d, f))
    x = _values(rng, (T, d), F32)
    logits = _dev(rng.standard_normal((T, E)).astype(np.float32))
    good = _host(moe.moe_layer_int8(W, _dev(x), logits, k)["y"])
    for bad in (np.nan, np.inf):
        x2 = x.copy()
        x2[4, 3] = bad
        y = _host(moe.moe_layer_int8(W, _dev(x2), logits, k)["y"])
        assert np.isnan(y[4]).all()
        _same(np.delete(y, 4, 0), np.delete(good, 4, 0))
    assert (_host(moe.moe_layer_int8(W, _dev(np.zeros((T, d), dtype=np.float32)), logits, k)["y"]) == 0).all()


def test_layer_of_no_tokens(moe):
    W = _pack(moe, _mats(_rng(9), 4, 64, 64))
    out = moe.moe_layer_int8(W, torch.empty((0, 64), device="cuda"), torch.empty((0, 4), device="cuda"), 2)
    assert out["y"].shape == (0, 64) and (out["offsets"] == 0).all() and (out["counts"] == 0).all()


def test_streams_and_graph(moe):
    """A side stream, and a captured layer replayed between eager work, give the eager bits."""
    d, f, E, k, T = 256, 448, 8, 2, 6
    rng = _rng(10)
    W = _pack(moe, _mats(rng, E, d, f))
    xs = [_dev(_values(rng, (T, d), F32)) for _ in range(3)]
    lg = [_dev(rng.standard_normal((T, E)).astype(np.float32)) for _ in range(3)]
    wm = moe.moe_int8_quantize(_dev(_values(rng, (1, d, 100), F32)))
    eager = [moe.moe_layer_int8(W, x, l, k)["y"].clone() for x, l in zip(xs, lg)]
    prod = [moe.moe_int8_matmul(moe.moe_int8_quantize_rows(x), wm).clone() for x in xs]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y = moe.moe_layer_int8(W, xs[0], lg[0], k, stream=side)["y"]
    side.synchronize()
    assert torch.equal(y, eager[0])
    x, l = xs[0].clone(), lg[0].clone()
    ws = torch.empty(moe.moe_layer_int8_workspace(T, E, k, d, f), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = moe.moe_layer_int8(W, x, l, k, workspace=ws)["y"]
        p = moe.moe_int8_matmul(moe.moe_int8_quantize_rows(x), wm)
    for i in (0, 1, 2, 1, 0):
        x.copy_(xs[i])
        l.copy_(lg[i])
        g.replay()
        other = moe.moe_layer_int8(W, xs[(i + 1) % 3], lg[(i + 1) % 3], k)["y"]
        torch.cuda.synchronize()
        assert torch.equal(y, eager[i]) and torch.equal(p, prod[i]) and torch.equal(other, eager[(i + 1) % 3])
