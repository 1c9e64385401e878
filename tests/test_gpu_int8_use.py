"""8-bit layers as a program uses them: many experts at the edge of the one-launch front, logits that leave experts or
tokens out, calls on two streams at once, and captured graphs."""
import numpy as np
import pytest
import torch

import int8_ref as ref
from test_gpu_int8 import BF16, F32, _dev, _host, _mats, _pack, _pair, _rng, _same, _values, moe  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 8, 63, 64, 65])
def test_eight_of_64_experts(moe, T):  # noqa: F811
    """T * 8 slots: 512 are routed and batched in one launch, 520 in two.  Of a third of the tokens all
    but k logits are -infinity, and many are equal."""
    d, f, E, k = 128, 64, 64, 8
    rng = _rng(20, T)
    mats = _mats(rng, E, d, f)
    W = _pack(moe, mats)
    q, s = ref.quantize(_values(rng, (T, d), F32))
    logits = rng.integers(-3, 4, (T, E)).astype(np.float32)
    for t in range(0, T, 3):
        logits[t, rng.permutation(E)[: E - k]] = -np.inf
    out = moe.moe_layer_int8(W, _pair(q, s), _dev(logits), k, dtype=F32)
    idx, w, y, bound = ref.layer(q, s, logits, k, mats, False)
    _same(_host(out["idx"]), idx)
    assert np.abs(_host(out["w"]) - w).max() <= 1e-6
    assert (np.abs(_host(out["y"]).astype(np.float64) - y) <= bound).all()
    flat = idx.reshape(-1)
    perm = np.argsort(flat, kind="stable").astype(np.int32)
    inv = np.empty_like(perm)
    inv[perm] = np.arange(perm.size)
    counts = np.bincount(flat, minlength=E).astype(np.int32)
    _same(_host(out["perm"]), perm)
    _same(_host(out["inv_perm"]).reshape(-1), inv)
    _same(_host(out["counts"]), counts)
    _same(_host(out["offsets"]), np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))


@pytest.mark.parametrize("T", [2, 9, 300])
def test_logits_of_nan(moe, T):  # noqa: F811
    """A token whose logits hold NaN leaves the other tokens as they are without it."""
    d, f, E, k = 128, 192, 8, 2
    rng = _rng(21, T)
    W = _pack(moe, _mats(rng, E, d, f))
    x = _dev(_values(rng, (T, d), BF16), BF16)
    lg = rng.standard_normal((T, E)).astype(np.float32)
    good = _host(moe.moe_layer_int8(W, x, _dev(lg), k)["y"])
    for bad in (np.full(E, np.nan), np.full(E, -np.inf), np.where(np.arange(E) < 7, lg[1], np.nan)):
        lg2 = lg.copy()
        lg2[1] = bad
        out = moe.moe_layer_int8(W, x, _dev(lg2), k)
        _same(np.delete(_host(out["y"]), 1, 0), np.delete(good, 1, 0))
        assert sorted(_host(out["perm"]).tolist()) == list(range(T * k))


def _big(moe, E, d, f, seed):  # noqa: F811
    g = torch.Generator("cuda").manual_seed(seed)
    def mat(k, c):
        return (torch.randint(-127, 128, (E, c, k), dtype=torch.int8, device="cuda", generator=g),
                (torch.rand((E, c), device="cuda", generator=g) + 0.5) * (k ** -0.5 / 64))
    return moe.moe_weights_pack_int8(mat(d, f), mat(d, f), mat(f, d))


def test_two_streams_at_once(moe):  # noqa: F811
    """Layers of few and of many rows (the persistent loop) over one handle on two streams, a workspace each."""
    E, d, f, k = 4, 2048, 1408, 2
    W = _big(moe, E, d, f, 1)
    g = torch.Generator("cuda").manual_seed(2)
    jobs = []
    for T in (1, 40, 3300):
        x = torch.randn((T, d), device="cuda", generator=g).to(BF16)
        lg = torch.randn((T, E), device="cuda", generator=g)
        jobs.append((x, lg, moe.moe_layer_int8(W, x, lg, k)["y"]))
    assert moe.moe_expert_ffn_plan(6600, E, d, f, moe.MOE_INT8)["down_tile_rows"] == 256
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for i in range(6):
        for n, s in enumerate(streams):
            j = (i + n) % 3
            with torch.cuda.stream(s):
                got.append((j, moe.moe_layer_int8(W, jobs[j][0], jobs[j][1], k)["y"]))
    torch.cuda.synchronize()
    for j, y in got:
        assert torch.equal(y, jobs[j][2])


@pytest.mark.parametrize("T", [1, 600, 3300])
def test_graphs_of_one_workspace(moe, T):  # noqa: F811
    """Two captured layers that share a workspace, replayed in turn between eager work."""
    E, d, f, k = 4, 2048, 1408, 2
    Ws = [_big(moe, E, d, f, n) for n in (3, 4)]
    g = torch.Generator("cuda").manual_seed(T)
    xs = [torch.randn((T, d), device="cuda", generator=g) for _ in range(3)]
    lg = [torch.randn((T, E), device="cuda", generator=g) for _ in range(3)]
    eager = [[moe.moe_layer_int8(W, x, l, k, dtype=BF16)["y"].clone() for x, l in zip(xs, lg)] for W in Ws]
    ws = torch.empty(moe.moe_layer_int8_workspace(T, E, k, d, f), dtype=torch.uint8, device="cuda")
    x, l = xs[0].clone(), lg[0].clone()
    torch.cuda.synchronize()
    graphs = []
    for W in Ws:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = moe.moe_layer_int8(W, x, l, k, workspace=ws, dtype=BF16)["y"]
        graphs.append((graph, y))
    for i in (0, 2, 1, 1, 0):
        x.copy_(xs[i])
        l.copy_(lg[i])
        for graph, _ in graphs:
            graph.replay()
        other = moe.moe_layer_int8(Ws[0], xs[(i + 1) % 3], lg[(i + 1) % 3], k, dtype=BF16)["y"]
        torch.cuda.synchronize()
        for n in range(2):
            assert torch.equal(graphs[n][1], eager[n][i])
        assert torch.equal(other, eager[0][(i + 1) % 3])


@pytest.mark.parametrize("d", [256, 4096, 20032])
def test_norms_and_conversions_captured(moe, d):  # noqa: F811
    """A chain of norm, rows to 8 bits and back, and a product on a side stream and in a graph whose norm updates x in
    place: replays give the eager bits."""
    T = 37
    g = torch.Generator("cuda").manual_seed(d)
    x0 = torch.randn((T, d), device="cuda", generator=g)
    y = torch.randn((T, d), device="cuda", generator=g).to(BF16)
    gain = torch.rand(d, device="cuda", generator=g) + 0.5
    wm = moe.moe_int8_quantize(torch.randn((1, d, 72), device="cuda", generator=g))

    def chain(x, stream=None):
        n = moe.moe_block_norm(x, y, True, gain, gain_before=gain, x_out=x, int8=True, stream=stream)
        rows = moe.moe_int8_quantize_rows(n["h"], stream=stream)
        back = moe.moe_int8_dequantize_rows(*rows, dtype=F32, stream=stream)
        return (x, n["h"], n["codes"], n["scales"], back, moe.moe_int8_matmul((n["codes"], n["scales"]), wm, stream=stream))

    first = [t.clone() for t in chain(x0.clone())]
    second = [t.clone() for t in chain(first[0].clone())]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    x = x0.clone()
    torch.cuda.synchronize()
    got = chain(x, side)
    side.synchronize()
    for a, b in zip(got, first):
        assert torch.equal(a, b)
    x = x0.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = chain(x)
    for _ in range(3):
        x.copy_(x0)
        for want in (first, second):
            graph.replay()
            chain(x0.clone())
            torch.cuda.synchronize()
            for a, b in zip(out, want):
                assert torch.equal(a, b)


@pytest.mark.parametrize("E,K,C", [(1, 4112, 1), (2, 4112, 66), (1, 5120, 8202), (3, 4352, 100), (2, 4112, 4098), (1, 14336, 63), (4, 4128, 4100)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_long_reductions_to_codes(moe, E, K, C, dtype):  # noqa: F811
    """Matrices whose channels are too long for one workgroup's registers (scales and codes in a launch each), with
    channels of zeros, of one large value and with a NaN or an infinity."""
    rng = _rng(22, E, K, C)
    w = _values(rng, (E, K, C), dtype, K ** -0.5)
    w[0, :, 0] = 0.0
    if C > 8:
        w[0, K - 1, C - 1] = -1000.0
        w[-1, 7, 3], w[-1, K - 2, 5] = np.nan, np.inf
    bad = ~np.isfinite(w).all(axis=1)
    q, s = ref.matrix(np.where(bad[:, None], 0, w).astype(np.float32))
    codes, scales = (_host(t) for t in moe.moe_int8_quantize(_dev(w, dtype)))
    assert np.array_equal(np.isnan(scales), bad)
    _same(scales[~bad], s[~bad])
    _same(codes, q)  # (codes 0 where the scale is NaN)
