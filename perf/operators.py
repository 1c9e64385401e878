"""Expert matrices held in 4 bits, as measurable cases: the conversion of a matrix, the expert
FFN over batched rows, the whole layer from tokens and router logits, and a stack of blocks.

The format is OCP Microscaling MXFP4: an element is four bits -- sign, two exponent bits, one
mantissa bit, so 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives -- and every 32 consecutive
elements along the reduction share one scale 2^(s-127), s one byte.  A matrix W [K,C] (y = x.W)
is codes [C,K/2] (element 2i in the low half of byte i) and scales [C,K/32].

Shapes (d, f, E, k): the Mixtral-shaped layer (4096, 14336, 8, 2), the 16-expert layer
(4096, 6400, 16, 2), a generic layer of many small experts (2048, 1408, 64, 6) and small ones.
Expert matrices are N(0, 1/fan_in) before their conversion, activations N(0, 1), router logits
N(0, 1), with `zipf` > 0 skewed by the log of a Zipf pmf over the experts (expert 0 hottest).
Programs in fp32 get fp32 results, programs in bf16 get the layer's result in bf16."""
import math

import numpy as np
import torch

own = False

MIXTRAL = dict(d=4096, f=14336, E=8, k=2)
SIXTEEN = dict(d=4096, f=6400, E=16, k=2)
SIXTYFOUR = dict(d=2048, f=1408, E=64, k=6)
SMALL = dict(d=256, f=512, E=8, k=2)
EPS = 1e-5


def listed():
    return [
        # converting a small all-fp32 layer's matrix: one launch each way
        dict(name="convert_small", kind="convert", E=8, K=256, C=512, x="f32"),
        # converting a large layer's first matrix when a checkpoint is loaded
        dict(name="convert_layer", kind="convert", E=8, K=4096, C=14336, x="bf16"),
        # the expert FFN of a program that batches for itself: a few rows of a small layer,
        # where latency is everything
        dict(name="ffn_small_n7", kind="ffn", N=7, x="f32", zipf=0.0, **SMALL),
        # the same for a beam of 16: every expert's matrices read once
        dict(name="ffn_n32", kind="ffn", N=32, x="f32", zipf=1.2, **MIXTRAL),
        # single-batch decoding, one token per step
        dict(name="layer_t1", kind="layer", T=1, x="f32", zipf=0.0, **MIXTRAL),
        # a few concurrent sequences of a bf16 program on smaller experts
        dict(name="layer_e16_t5", kind="layer", T=5, x="bf16", zipf=1.2, **SIXTEEN),
        # the same on many small experts
        dict(name="layer_e64_t10", kind="layer", T=10, x="bf16", zipf=0.0, **SIXTYFOUR),
        # a short prompt of odd length: tens of rows per expert
        dict(name="layer_t77", kind="layer", T=77, x="bf16", zipf=1.2, **MIXTRAL),
        # a chunk of a prompt on many small experts
        dict(name="layer_e64_t300", kind="layer", T=300, x="bf16", zipf=0.0, **SIXTYFOUR),
        # the longest prefill step
        dict(name="layer_t4096", kind="layer", T=4096, x="bf16", zipf=1.2, **MIXTRAL),
        # single-batch decoding through consecutive blocks (norm, router, experts, residual)
        dict(name="stack_t1", kind="stack", T=1, layers=4, x="f32", zipf=0.0, **MIXTRAL),
        # two sequences on the 16-expert layer
        dict(name="stack_e16_t2", kind="stack", T=2, layers=3, x="f32", zipf=0.0, **SIXTEEN),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_shape(rng):
    """One of the named shapes, or a small one with d and f any multiples of 64."""
    if rng.random() < 0.6:
        return dict(rng.choice([MIXTRAL, SIXTEEN, SIXTYFOUR]))
    E = rng.randint(2, 32)
    return dict(d=64 * rng.randint(1, 24), f=64 * rng.randint(1, 32), E=E, k=rng.randint(1, min(4, E)))


def draw(rng):
    kind = rng.choice(["convert", "ffn", "ffn", "layer", "layer", "layer", "layer", "stack"])
    zipf = rng.choice([0.0, 0.6, 1.2])
    if kind == "convert":
        return dict(kind=kind, E=rng.randint(1, 8), K=32 * _log_int(rng, 1, 128), C=_log_int(rng, 1, 14336),
                    x=rng.choice(["f32", "bf16"]))
    if kind == "stack":
        return dict(kind=kind, T=rng.randint(1, 2), layers=rng.randint(2, 4), x="f32", zipf=zipf,
                    **rng.choice([MIXTRAL, SIXTEEN]))
    shape = _draw_shape(rng)
    if kind == "ffn":
        return dict(kind=kind, N=_log_int(rng, 1, 72), x=rng.choice(["f32", "bf16"]), zipf=zipf, **shape)
    T = _log_int(rng, 1, 4096)
    f32 = T * shape["k"] <= 72 and rng.random() < 0.5
    return dict(kind=kind, T=T, x="f32" if f32 else "bf16", zipf=zipf, **shape)


# ---- inputs ----------------------------------------------------------------------------

def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _generator(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000 + stream)
    return g


def _normal(gen, shape, std, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)


def _converted_matrices(E, K, C, gen):
    """codes [E,C,K/2] and scales [E,C,K/32] of E matrices [K,C] with N(0, 1/K) elements."""
    codes = torch.empty((E, C, K // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((E, C, K // 32), dtype=torch.uint8, device="cuda")
    for e in range(E):
        codes[e], scales[e] = _quantize(_normal(gen, (K, C), K ** -0.5, torch.float32))
    return codes, scales


def _expert_matrices(case, seed, layer):
    g, d, f, E = _generator(seed, 100 + layer), case["d"], case["f"], case["E"]
    return (_converted_matrices(E, d, f, g), _converted_matrices(E, d, f, g), _converted_matrices(E, f, d, g))


def _log_pmf(case):
    p = np.arange(1, case["E"] + 1, dtype=np.float64) ** -case["zipf"]
    return np.log(p / p.sum())


def _tokens(case, seed):
    g = _generator(seed, 1)
    x = _normal(g, (case["T"], case["d"]), 1.0, _dtype(case["x"]))
    logits = _normal(g, (case["T"], case["E"]), 1.0, torch.float32)
    return x, logits + torch.from_numpy(_log_pmf(case).astype(np.float32)).cuda()


def _batched_rows(case, seed):
    """Rows in expert order and the experts' offsets, as a batching step leaves them."""
    g = _generator(seed, 1)
    x = _normal(g, (case["N"], case["d"]), 1.0, _dtype(case["x"]))
    p = torch.from_numpy(np.exp(_log_pmf(case)).astype(np.float32)).cuda()
    counts = torch.bincount(torch.multinomial(p, case["N"], replacement=True, generator=g), minlength=case["E"])
    return x, torch.cat([counts.new_zeros(1), torch.cumsum(counts, 0)]).int()


def _source_matrix(case, seed):
    return _normal(_generator(seed, 1), (case["E"], case["K"], case["C"]), case["K"] ** -0.5, _dtype(case["x"]))


def _router_matrix(case, seed, layer):
    return _normal(_generator(seed, 50 + layer), (case["d"], case["E"]), case["d"] ** -0.5, torch.float32)


def _weights(case, seed, layer=0):
    """What a program keeps of a layer's experts: the converted matrices, or the library's handle."""
    mats = _expert_matrices(case, seed, layer)
    if own:
        import paper_2402_07033_amd as moe
        return moe.moe_weights_pack_mxfp4(*mats)
    return mats


def prepare(case, seed):
    st = dict(case=case)
    if case["kind"] == "convert":
        st["w"] = _source_matrix(case, seed)
        return st
    d, f, E, k = (case[n] for n in ("d", "f", "E", "k"))
    if case["kind"] == "stack":
        st["layers"] = [(_weights(case, seed, n), _router_matrix(case, seed, n)) for n in range(case["layers"])]
        st["x"] = _tokens(case, seed)[0]
        if own:
            import paper_2402_07033_amd as moe
            st["bufs"] = moe.StackBuffers(case["T"], E, k, d, f, w_dtype=moe.MOE_MXFP4)
        return st
    st["W"] = _weights(case, seed)
    if case["kind"] == "ffn":
        st["x"], st["offsets"] = _batched_rows(case, seed)
    else:
        st["x"], st["logits"] = _tokens(case, seed)
    if own:
        import paper_2402_07033_amd as moe
        act = moe.MOE_BF16 if case["x"] == "bf16" else moe.MOE_F32
        N = case["N"] if case["kind"] == "ffn" else case["T"] * k
        st["ws"] = torch.empty(moe.moe_expert_ffn_workspace(N, E, d, f, act) if case["kind"] == "ffn"
                               else moe.moe_layer_mxfp4_workspace(case["T"], E, k, d, f), dtype=torch.uint8,
                               device="cuda")
    return st


# ---- one pass --------------------------------------------------------------------------

def run(state):
    case, k = state["case"], state["case"].get("k")
    if own:
        import paper_2402_07033_amd as moe
        if case["kind"] == "convert":
            codes, scales = moe.moe_mxfp4_quantize(state["w"])
            return moe.moe_mxfp4_dequantize(codes, scales, dtype=state["w"].dtype)
        if case["kind"] == "ffn":
            return moe.moe_expert_ffn(state["W"], state["x"], state["offsets"], workspace=state["ws"])
        if case["kind"] == "stack":
            return moe.moe_stack_forward(state["layers"], state["x"].clone(), k, EPS, bufs=state["bufs"])
        out = moe.moe_layer_mxfp4(state["W"], state["x"], state["logits"], k, workspace=state["ws"])
        return dict(y=out["y"], idx=out["idx"], w=out["w"], offsets=out["offsets"], perm=out["perm"],
                    inv_perm=out["inv_perm"])
    if case["kind"] == "convert":
        return _convert_plain(state["w"])
    if case["kind"] == "ffn":
        rows = torch.arange(case["N"], device="cuda")
        expert = torch.searchsorted(state["offsets"][1:].contiguous(), rows.int(), right=True)
        return _experts_plain(state["x"].float(), expert[:, None], torch.ones((case["N"], 1), device="cuda"),
                              state["W"])
    if case["kind"] == "stack":
        x = state["x"]
        for mats, w_gate in state["layers"]:
            h = x / torch.sqrt((x * x).mean(dim=1, keepdim=True) + EPS)
            idx, w = _route_plain(h @ w_gate, k)
            x = x + _experts_plain(h, idx, w, mats)
        return x
    idx, w = _route_plain(state["logits"], k)
    flat = idx.reshape(-1)
    perm = torch.sort(flat, stable=True)[1]
    inv = torch.empty_like(perm)
    inv[perm] = torch.arange(perm.numel(), device="cuda")
    counts = (flat[:, None] == torch.arange(case["E"], device="cuda")).sum(dim=0)
    offsets = torch.cat([counts.new_zeros(1), torch.cumsum(counts, 0)])
    y = _experts_plain(state["x"].float(), idx, w, state["W"])
    return dict(y=y.to(state["x"].dtype), idx=idx.int(), w=w, offsets=offsets.int(), perm=perm.int(),
                inv_perm=inv.int())


# ---- the plain forms -------------------------------------------------------------------

# the element values of the codes 0 .. 15
_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _quantize(w):
    """w [K,C] fp32 -> codes [C,K/2], scales [C,K/32].  The scale's exponent is the largest
    magnitude's, less 2 (the exponent of the largest element); elements round to nearest, ties to
    the even code, and saturate."""
    K, C = w.shape
    b = w.t().reshape(C, K // 32, 32)
    top = b.abs().amax(dim=2)
    e = (torch.frexp(top)[1] - 1 - 2).clamp(-126, 127)  # frexp's mantissa is in [0.5, 1)
    e = torch.where(top > 0, e, torch.full_like(e, -126))
    m = torch.ldexp(b.abs(), -e[:, :, None])
    # a step of 0.5 up to 2, of 1 up to 4, of 2 up to 6; the codes of the three pieces follow on
    # one another, and torch.round takes ties to the even number
    code = torch.where(m < 2, torch.round(m * 2), torch.where(m < 4, torch.round(m) + 2, torch.round(m / 2) + 4))
    code = code.clamp(max=7).to(torch.uint8) + 8 * torch.signbit(b).to(torch.uint8)
    code = code.reshape(C, K // 2, 2)
    return code[:, :, 0] + 16 * code[:, :, 1], (e + 127).to(torch.uint8)


def _dequantize(codes, scales):
    """codes [..., K/2], scales [..., K/32] -> fp32 [..., K]."""
    table = torch.tensor(_VALUES, dtype=torch.float32, device=codes.device)
    v = torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], dim=-1)
    v = v.reshape(scales.shape + (32,))
    return torch.ldexp(v, scales.int()[..., None] - 127).reshape(codes.shape[:-1] + (-1,))


def _convert_plain(w):
    E, K, C = w.shape
    codes, scales = _quantize(w.float().transpose(1, 2).reshape(E * C, K).t())
    return _dequantize(codes, scales).reshape(E, C, K).transpose(1, 2).contiguous().to(w.dtype)


def _route_plain(logits, k):
    v, idx = torch.sort(logits, dim=1, descending=True, stable=True)
    u = torch.exp(v[:, :k] - v[:, :1])
    return idx[:, :k], u / u.sum(dim=1, keepdim=True)


def _experts_plain(x, idx, w, mats):
    """y[t] = sum_j w[t,j] * expert idx[t,j] of x[t], every expert's matrices widened in turn."""
    y = torch.zeros_like(x)
    for e in range(mats[0][0].shape[0]):
        tok, slot = torch.nonzero(idx == e, as_tuple=True)
        if tok.numel() == 0:
            continue
        w1, w3, w2 = (_dequantize(codes[e], scales[e]) for codes, scales in mats)
        a = x[tok] @ w1.t()
        h = a / (1 + torch.exp(-a)) * (x[tok] @ w3.t())
        y.index_add_(0, tok, (h @ w2.t()) * w[tok, slot, None])
    return y


# ---- what a pass cannot do without -------------------------------------------------------

def _active_experts(E, T, k, zipf):
    """Experts that get at least one row, on average over draws."""
    if k > 1 and (T == 1 or T * k >= 64 * E):
        return float(min(E, T * k))
    rng, n = np.random.default_rng(7), []
    p = np.arange(1, E + 1, dtype=np.float64) ** -zipf
    p /= p.sum()
    for _ in range(32):
        if k == 1:
            n.append(len(np.unique(rng.choice(E, size=T, p=p))))
        else:
            lg = rng.standard_normal((T, E)) + np.log(p)[None, :]
            n.append(len(np.unique(np.argsort(-lg, axis=1)[:, :k])))
    return float(np.mean(n))


def work(case):
    xb = 2 if case["x"] == "bf16" else 4
    if case["kind"] == "convert":
        n = case["E"] * case["K"] * case["C"]
        return {"bytes": 2 * n * (xb + 0.5 + 1 / 32), "flops": 4 * n}
    d, f, E, k, L = case["d"], case["f"], case["E"], case["k"], case.get("layers", 1)
    ffn = case["kind"] == "ffn"
    T = case["N"] if ffn else case["T"]
    N = T if ffn else T * k
    experts = _active_experts(E, T, 1 if ffn else k, case["zipf"]) * 3 * d * f * (0.5 + 1 / 32)
    flops = 6 * N * d * f
    if case["kind"] == "stack":
        return {"bytes": L * (experts + d * E * 4) + 2 * T * d * 4, "flops": L * (flops + 2 * T * d * E + 2 * N * d)}
    if ffn:
        return {"bytes": experts + T * d * (xb + 4) + (E + 1) * 4, "flops": flops}
    return {"bytes": experts + T * d * 2 * xb + T * E * 4 + 4 * N * 4 + E * 4, "flops": flops + 2 * N * d}


# ---- the same in 64 bits -----------------------------------------------------------------

def _widen64(codes, scales):
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)
    ex, man = ((c >> 1) & 3).double(), (c & 1).double()
    mag = torch.where(ex == 0, man / 2, (1 + man / 2) * torch.exp2(ex - 1))
    sc = torch.exp2(scales.double() - 127).repeat_interleave(32, dim=-1)
    return torch.where(c >= 8, -mag, mag) * sc


def _nearest64(w):
    """The values that the converted w [K,C] stands for, by distance to each of the eight magnitudes."""
    K, C = w.shape
    b = w.double().t().reshape(C, K // 32, 32)
    top = b.abs().amax(dim=2, keepdim=True)
    e = torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top))))
    e = torch.where(torch.exp2(e) > top, e - 1, e)
    e = torch.where(torch.exp2(e + 1) <= top, e + 1, e)  # log2 next to a power of two
    sc = torch.exp2(torch.where(top > 0, (e - 2).clamp(-126, 127), torch.full_like(e, -126)))
    m = b.abs() / sc
    best, far = torch.zeros_like(m), m.clone()
    for value, even in ((0.5, False), (1.0, True), (1.5, False), (2.0, True), (3.0, False), (4.0, True), (6.0, False)):
        off = (m - value).abs()
        nearer = off <= far if even else off < far  # a tie goes to the even code
        best, far = torch.where(nearer, torch.full_like(m, value), best), torch.where(nearer, off, far)
    return (torch.where(b < 0, -best, best) * sc).reshape(C, K).t()


def _route64(logits, k):
    lg = logits.double()
    idx = torch.sort(lg, dim=1, descending=True, stable=True)[1][:, :k]
    return idx, torch.softmax(torch.gather(lg, 1, idx), dim=1)


def _experts64(x, idx, w, mats):
    y = torch.zeros((x.shape[0], mats[0][0].shape[2] * 2), dtype=torch.float64, device="cuda")
    for e in range(mats[0][0].shape[0]):
        tok, slot = torch.nonzero(idx == e, as_tuple=True)
        if tok.numel() == 0:
            continue
        a = x[tok]
        h = torch.nn.functional.silu(a @ _widen64(mats[0][0][e], mats[0][1][e]).t())
        h = h * (a @ _widen64(mats[1][0][e], mats[1][1][e]).t())
        y.index_add_(0, tok, (h @ _widen64(mats[2][0][e], mats[2][1][e]).t()) * w[tok, slot, None])
    return y


def exact(case, seed):
    if case["kind"] == "convert":
        w = _source_matrix(case, seed)
        out = torch.empty_like(w)  # the values fit the source's type
        for e in range(case["E"]):
            out[e] = _nearest64(w[e]).to(w.dtype)
        return out
    k = case["k"]
    if case["kind"] == "stack":
        x = _tokens(case, seed)[0].double()
        for n in range(case["layers"]):
            h = x / torch.sqrt((x * x).mean(dim=1, keepdim=True) + EPS)
            idx, w = _route64(h @ _router_matrix(case, seed, n).double(), k)
            x = x + _experts64(h, idx, w, _expert_matrices(case, seed, n))
        return x
    mats = _expert_matrices(case, seed, 0)
    if case["kind"] == "ffn":
        x, offsets = _batched_rows(case, seed)
        counts = (offsets[1:] - offsets[:-1]).long()
        expert = torch.repeat_interleave(torch.arange(case["E"], device="cuda"), counts)
        return _experts64(x.double(), expert[:, None], torch.ones((case["N"], 1), device="cuda").double(), mats)
    x, logits = _tokens(case, seed)
    idx, w = _route64(logits, k)
    flat = idx.reshape(-1)
    perm = torch.sort(flat, stable=True)[1]
    inv = torch.argsort(perm)
    offsets = torch.cat([flat.new_zeros(1), torch.cumsum(torch.bincount(flat, minlength=case["E"]), 0)])
    return dict(y=_experts64(x.double(), idx, w, mats), idx=idx.int(), w=w, offsets=offsets.int(), perm=perm.int(),
                inv_perm=inv.int())
