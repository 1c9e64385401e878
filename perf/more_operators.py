"""8-bit integer products with a scale for every token and every channel, the expert layer over
them, and the norms around a block, as measurable cases.

The 8-bit form of a row of values v (a token of x, or an output channel of a matrix W [K,C],
y = x.W) is q = v/s rounded to the nearest integer (ties to even) with s = max|v|/127 in fp32.
A matrix is codes [C,K] int8 and scales [C].  Products are sums of integers, scaled once:
y[t,c] = sx[t] * sw[c] * sum_k qx[t,k] qw[c,k].

  convert   a matrix to its 8-bit form and back
  matmul    rows to their 8-bit form and their product with a matrix, or with one matrix per expert
  layer     routing, the gated experts in 8 bits (x and h = silu(a)*b each in their 8-bit form),
            gate-weighted sum; results in bf16
  norm      x' = x + r * g * u, u = y or rmsnorm(y) * gain, and h = rmsnorm(x') * gain, the two
            norms around a block with its gate g and the residual scale r; h in fp32, bf16 or 8 bits
  block     the norms, the router on h in fp32 and the expert layer on h in 8 bits

Shapes (d, f, E, k): the Mixtral-shaped layer (4096, 14336, 8, 2), the 16-expert layer
(4096, 6400, 16, 2), a generic layer of many small experts (2048, 1408, 64, 6) and small ones.
Matrices are N(0, 1/fan_in) before their conversion, activations N(0, 1), router logits N(0, 1),
with `zipf` > 0 skewed by the log of a Zipf pmf over the experts (expert 0 hottest)."""
import math

import numpy as np
import torch

own = False

MIXTRAL = dict(d=4096, f=14336, E=8, k=2)
SIXTEEN = dict(d=4096, f=6400, E=16, k=2)
SIXTYFOUR = dict(d=2048, f=1408, E=64, k=6)
EPS = 1e-5


def listed():
    return [
        # converting a large layer's first matrix when a checkpoint is loaded
        dict(name="convert_layer", kind="convert", E=8, K=4096, C=14336, x="bf16"),
        # one token of an fp32 program through a square projection: latency and 16 MB of codes
        dict(name="matmul_m1", kind="matmul", M=1, K=4096, C=4096, E=1, x="f32", zipf=0.0),
        # rows that a program batched for itself, an odd number on each of 16 experts, odd width
        dict(name="matmul_e16_m333", kind="matmul", M=333, K=2048, C=1407, E=16, x="bf16", zipf=0.6),
        # the longest prefill step through one wide projection
        dict(name="matmul_m4096", kind="matmul", M=4096, K=4096, C=14336, E=1, x="bf16", zipf=0.0),
        # single-batch decoding, one token per step
        dict(name="layer_t1", kind="layer", T=1, x="bf16", zipf=0.0, **MIXTRAL),
        # a few concurrent sequences on many small experts
        dict(name="layer_e64_t10", kind="layer", T=10, x="bf16", zipf=0.0, **SIXTYFOUR),
        # a short prompt of odd length: tens of rows per expert
        dict(name="layer_t77", kind="layer", T=77, x="bf16", zipf=1.2, **MIXTRAL),
        # the longest prefill step
        dict(name="layer_t4096", kind="layer", T=4096, x="bf16", zipf=1.2, **MIXTRAL),
        # the place between two blocks at single-batch decoding, residual stream in fp32
        dict(name="norm_t1", kind="norm", T=1, d=4096, x="f32", y="f32", after=True, gate="feature", out="f32"),
        # the same of a prompt of odd length in bf16, a gate per token, rows for 8-bit products
        dict(name="norm_t301", kind="norm", T=301, d=2048, x="bf16", y="bf16", after=False, gate="token", out="int8"),
        # the longest prefill step
        dict(name="norm_t4096", kind="norm", T=4096, d=4096, x="f32", y="bf16", after=True, gate="feature", out="bf16"),
        # two sequences through the place between two blocks and the next block's experts
        dict(name="block_e16_t2", kind="block", T=2, x="f32", y="bf16", after=True, gate="feature", zipf=0.0, **SIXTEEN),
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
    kind = rng.choice(["convert", "matmul", "matmul", "layer", "layer", "layer", "norm", "norm", "block"])
    zipf = rng.choice([0.0, 0.6, 1.2])
    if kind == "convert":
        return dict(kind=kind, E=rng.randint(1, 8), K=16 * _log_int(rng, 1, 256), C=_log_int(rng, 1, 14336),
                    x=rng.choice(["f32", "bf16"]))
    if kind == "matmul":
        E = rng.choice([1, 1, rng.randint(2, 32)])
        return dict(kind=kind, M=_log_int(rng, 1, 4096), K=16 * _log_int(rng, 1, 256),
                    C=_log_int(rng, 1, 14336 if E == 1 else 4096), E=E, x=rng.choice(["f32", "bf16"]),
                    zipf=0.0 if E == 1 else zipf)
    norms = dict(x=rng.choice(["f32", "bf16"]), y=rng.choice(["f32", "bf16"]), after=rng.random() < 0.6,
                 gate=rng.choice(["none", "feature", "token"]))
    if kind == "norm":
        return dict(kind=kind, T=_log_int(rng, 1, 4096), d=64 * _log_int(rng, 1, 128),
                    out=rng.choice(["f32", "bf16", "int8"]), **norms)
    shape = _draw_shape(rng)
    if kind == "block":
        return dict(kind=kind, T=_log_int(rng, 1, 64), zipf=zipf, **norms, **shape)
    return dict(kind=kind, T=_log_int(rng, 1, 4096), x=rng.choice(["f32", "bf16", "bf16"]), zipf=zipf, **shape)


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
    """codes [E,C,K] and scales [E,C] of E matrices [K,C] with N(0, 1/K) elements."""
    codes = torch.empty((E, C, K), dtype=torch.int8, device="cuda")
    scales = torch.empty((E, C), dtype=torch.float32, device="cuda")
    for e in range(E):
        codes[e], scales[e] = _quantize(_normal(gen, (C, K), K ** -0.5, torch.float32))
    return codes, scales


def _expert_matrices(case, seed):
    g, d, f, E = _generator(seed, 100), case["d"], case["f"], case["E"]
    return (_converted_matrices(E, d, f, g), _converted_matrices(E, d, f, g), _converted_matrices(E, f, d, g))


def _log_pmf(case):
    p = np.arange(1, case["E"] + 1, dtype=np.float64) ** -case["zipf"]
    return torch.from_numpy(np.log(p / p.sum()).astype(np.float32)).cuda()


def _tokens(case, seed):
    g = _generator(seed, 1)
    x = _normal(g, (case["T"], case["d"]), 1.0, _dtype(case["x"]))
    return x, _normal(g, (case["T"], case["E"]), 1.0, torch.float32) + _log_pmf(case)


def _batched_rows(case, seed):
    """Rows in expert order and, with several experts, their offsets as a batching step leaves them."""
    g = _generator(seed, 1)
    x = _normal(g, (case["M"], case["K"]), 1.0, _dtype(case["x"]))
    if case["E"] == 1:
        return x, None
    counts = torch.bincount(torch.multinomial(torch.exp(_log_pmf(case)), case["M"], replacement=True, generator=g),
                            minlength=case["E"])
    return x, torch.cat([counts.new_zeros(1), torch.cumsum(counts, 0)]).int()


def _source_matrix(case, seed):
    return _normal(_generator(seed, 1), (case["E"], case["K"], case["C"]), case["K"] ** -0.5, _dtype(case["x"]))


def _norm_inputs(case, seed):
    """The residual stream, the block's output, the gains (near 1) and the gate of the place between two blocks."""
    g, T, d = _generator(seed, 2), case["T"], case["d"]
    st = dict(x=_normal(g, (T, d), 1.0, _dtype(case["x"])), y=_normal(g, (T, d), 0.5, _dtype(case["y"])),
              gain_after=1 + _normal(g, (d,), 0.1, torch.float32), gain_before=1 + _normal(g, (d,), 0.1, torch.float32),
              gate=None, row_gate=None, scale=0.7)
    if case["gate"] == "feature":
        st["gate"] = _normal(g, (d,), 0.5, torch.float32)
    elif case["gate"] == "token":
        st["row_gate"] = torch.empty((T,), dtype=torch.float32, device="cuda").uniform_(0.0, 1.0, generator=g)
    return st


def _router_matrix(case, seed):
    w = _normal(_generator(seed, 50), (case["d"], case["E"]), case["d"] ** -0.5, torch.float32)
    return w * (1 + torch.arange(case["E"], 0, -1, device="cuda") * (0.1 * case["zipf"]))


def prepare(case, seed):
    st = dict(case=case)
    if case["kind"] == "convert":
        st["w"] = _source_matrix(case, seed)
    elif case["kind"] == "matmul":
        st["x"], st["offsets"] = _batched_rows(case, seed)
        st["w"] = _converted_matrices(case["E"], case["K"], case["C"], _generator(seed, 100))
    elif case["kind"] == "norm":
        st.update(_norm_inputs(case, seed))
    else:
        mats = _expert_matrices(case, seed)
        if case["kind"] == "layer":
            st["x"], st["logits"] = _tokens(case, seed)
        else:
            st.update(_norm_inputs(case, seed))
            st["w_gate"] = _router_matrix(case, seed)
        st["W"] = mats
        if own:  # what a program keeps: the library's handle and a workspace
            import paper_2402_07033_amd as moe
            st["W"] = moe.moe_weights_pack_int8(*mats)
            st["ws"] = torch.empty(moe.moe_layer_int8_workspace(*(case[n] for n in ("T", "E", "k", "d", "f"))),
                                   dtype=torch.uint8, device="cuda")
    return st


# ---- one pass --------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(st):
    import paper_2402_07033_amd as moe
    case = st["case"]
    kind = case["kind"]
    if kind == "convert":
        codes, scales = moe.moe_int8_quantize(st["w"])
        return moe.moe_int8_dequantize(codes, scales, dtype=st["w"].dtype)
    if kind == "matmul":
        return moe.moe_int8_matmul(moe.moe_int8_quantize_rows(st["x"]), st["w"], offsets=st["offsets"],
                                   dtype=st["x"].dtype)
    if kind == "layer":
        out = moe.moe_layer_int8(st["W"], st["x"], st["logits"], case["k"], dtype=torch.bfloat16, workspace=st["ws"])
        return {n: out[n] for n in ("y", "idx", "w", "offsets", "perm", "inv_perm")}
    out = "both" if kind == "block" else case["out"]
    n = moe.moe_block_norm(st["x"], y=st["y"], norm_after=case["after"], gain_after=st["gain_after"] if case["after"] else None,
                           gate=st["gate"], row_gate=st["row_gate"], residual_scale=st["scale"],
                           gain_before=st["gain_before"], eps=EPS, int8=out in ("int8", "both"),
                           h_dtype=None if out == "int8" else torch.bfloat16 if out == "bf16" else torch.float32)
    if kind == "block":
        logits = moe.moe_router_logits(n["h"], st["w_gate"])
        lay = moe.moe_layer_int8(st["W"], (n["codes"], n["scales"]), logits, case["k"], dtype=torch.bfloat16,
                                 workspace=st["ws"])
        return dict(x=n["x"], y=lay["y"])
    if out == "int8":
        return dict(x=n["x"], h=moe.moe_int8_dequantize_rows(n["codes"], n["scales"], dtype=torch.bfloat16))
    return dict(x=n["x"], h=n["h"])


def _run_plain(st):
    case = st["case"]
    kind = case["kind"]
    if kind == "convert":
        w = st["w"]
        codes, scales = _quantize(w.transpose(1, 2).float())
        return (codes.float() * scales[..., None]).transpose(1, 2).contiguous().to(w.dtype)
    if kind == "matmul":
        q, s = _quantize(st["x"].float())
        codes, scales = st["w"]
        if case["E"] == 1:
            return _product(q, s, codes[0], scales[0]).to(st["x"].dtype)
        rows = torch.arange(case["M"], device="cuda")
        expert = torch.searchsorted(st["offsets"][1:].contiguous(), rows.int(), right=True)
        y = torch.empty((case["M"], case["C"]), dtype=torch.float32, device="cuda")
        for e in range(case["E"]):
            at = torch.nonzero(expert == e)[:, 0]
            y[at] = _product(q[at], s[at], codes[e], scales[e])
        return y.to(st["x"].dtype)
    if kind == "layer":
        k = case["k"]
        idx, w = _route_plain(st["logits"], k)
        flat = idx.reshape(-1)
        perm = torch.sort(flat, stable=True)[1]
        inv = torch.empty_like(perm)
        inv[perm] = torch.arange(perm.numel(), device="cuda")
        counts = (flat[:, None] == torch.arange(case["E"], device="cuda")).sum(dim=0)
        offsets = torch.cat([counts.new_zeros(1), torch.cumsum(counts, 0)])
        y = _experts_plain(*_quantize(st["x"].float()), idx, w, st["W"])
        return dict(y=y.bfloat16(), idx=idx.int(), w=w, offsets=offsets.int(), perm=perm.int(), inv_perm=inv.int())
    out = "both" if kind == "block" else case["out"]
    # codes are taken next to the borders between them: 64 bits up to there
    wide = torch.float64 if out in ("int8", "both") else torch.float32
    x = st["x"].to(wide)
    u = st["y"].to(wide)
    if case["after"]:
        u = u / torch.sqrt((u * u).mean(dim=1, keepdim=True) + EPS) * st["gain_after"]
    if st["gate"] is not None:
        u = u * st["gate"]
    if st["row_gate"] is not None:
        u = u * st["row_gate"][:, None]
    x = x + st["scale"] * u
    h = x / torch.sqrt((x * x).mean(dim=1, keepdim=True) + EPS) * st["gain_before"]
    x = x.to(st["x"].dtype)
    if out == "bf16" or out == "f32":
        return dict(x=x, h=h.to(_dtype(out)))
    q, s = _quantize(h)
    if out == "int8":
        return dict(x=x, h=(q.float() * s[:, None]).bfloat16())
    idx, w = _route_plain((h @ st["w_gate"].double()).float(), case["k"])
    return dict(x=x, y=_experts_plain(q, s, idx, w, st["W"]).bfloat16())


# ---- the plain forms -------------------------------------------------------------------

def _quantize(v):
    """v [..., K] -> codes int8 [..., K], scales fp32 [...].  The quotient of two fp32 numbers in 64 bits is on
    the right side of every border between two codes."""
    s = (v.abs().amax(dim=-1) / 127).float()
    safe = torch.where(s > 0, s, torch.ones_like(s)).double()
    q = torch.round(v.double() / safe[..., None]).clamp(-127, 127)
    return torch.where(s[..., None] > 0, q, torch.zeros_like(q)).to(torch.int8), s


def _product(q, s, codes, scales):
    """q [M,K], s [M], codes [C,K], scales [C] -> fp32 [M,C]."""
    return (q.float() @ codes.float().t()) * s[:, None] * scales


def _route_plain(logits, k):
    v, idx = torch.sort(logits, dim=1, descending=True, stable=True)
    u = torch.exp(v[:, :k] - v[:, :1])
    return idx[:, :k], u / u.sum(dim=1, keepdim=True)


def _experts_plain(q, s, idx, w, mats):
    """y[t] = sum_j w[t,j] * expert idx[t,j] of token t in its 8-bit form, fp32 [T,d]."""
    y = torch.zeros(q.shape, dtype=torch.float32, device=q.device)
    for e in range(mats[0][0].shape[0]):
        tok, slot = torch.nonzero(idx == e, as_tuple=True)
        if tok.numel() == 0:
            continue
        a, b = (_product(q[tok], s[tok], codes[e], scales[e]) for codes, scales in mats[:2])
        y.index_add_(0, tok, _product(*_quantize(a / (1 + torch.exp(-a)) * b), mats[2][0][e], mats[2][1][e])
                     * w[tok, slot, None])
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
    size = dict(f32=4, bf16=2, int8=2, both=0)
    xb = size[case["x"]]
    if case["kind"] == "convert":
        n = case["E"] * case["K"] * case["C"]
        return {"bytes": 2 * n * (xb + 1), "flops": 4 * n}
    if case["kind"] == "matmul":
        M, K, C, E = (case[n] for n in ("M", "K", "C", "E"))
        experts = 1 if E == 1 else _active_experts(E, M, 1, case["zipf"])
        return {"bytes": experts * C * (K + 4) + M * (K + C) * xb, "flops": 2 * M * K * C}
    T, d = case["T"], case["d"]
    norm_bytes = norm_flops = 0
    if case["kind"] != "layer":
        yb, hb = size[case["y"]], size["both" if case["kind"] == "block" else case["out"]]
        norm_bytes, norm_flops = T * d * (2 * xb + yb + hb) + 12 * d, 12 * T * d
        if case["kind"] == "norm":
            return {"bytes": norm_bytes, "flops": norm_flops}
    f, E, k = case["f"], case["E"], case["k"]
    experts = _active_experts(E, T, k, case["zipf"]) * 3 * d * f
    flops = T * k * (6 * d * f + 2 * d)
    if case["kind"] == "block":
        return {"bytes": norm_bytes + experts + d * E * 4 + T * d * 2, "flops": norm_flops + flops + 2 * T * d * E}
    return {"bytes": experts + T * d * (xb + 2) + T * E * 4 + 4 * T * k * 4 + E * 4, "flops": flops}


# ---- the same in 64 bits -----------------------------------------------------------------

def _codes64(v):
    """Codes and scales of the rows of v in 64 bits, by the distance to the integer below."""
    s = (v.abs().max(dim=-1, keepdim=True)[0] / 127).float().double()
    z = torch.where(s > 0, v / torch.where(s > 0, s, torch.ones_like(s)), torch.zeros_like(v))
    low = torch.floor(z)
    up = (z - low > 0.5) | ((z - low == 0.5) & (torch.remainder(low, 2) == 1))
    return torch.clamp(low + up, -127, 127), s


def _times64(v, codes, scales):
    q, s = _codes64(v)
    return torch.matmul(q, codes.double().t().contiguous()) * (s * scales.double()[None, :])


def _route64(logits, k):
    lg = logits.double()
    idx = torch.sort(lg, dim=1, descending=True, stable=True)[1][:, :k]
    return idx, torch.softmax(torch.gather(lg, 1, idx), dim=1)


def _experts64(x, idx, w, mats):
    y = torch.zeros_like(x)
    for e in range(mats[0][0].shape[0]):
        tok, slot = torch.nonzero(idx == e, as_tuple=True)
        if tok.numel():
            h = torch.nn.functional.silu(_times64(x[tok], mats[0][0][e], mats[0][1][e]))
            h = h * _times64(x[tok], mats[1][0][e], mats[1][1][e])
            y.index_add_(0, tok, _times64(h, mats[2][0][e], mats[2][1][e]) * w[tok, slot, None])
    return y


def _rms64(v):
    return v * torch.rsqrt(v.square().mean(dim=1, keepdim=True) + EPS)


def exact(case, seed):
    if case["kind"] == "convert":
        w = _source_matrix(case, seed)
        out = torch.empty(w.shape, dtype=torch.float64 if w.numel() < 1 << 26 else torch.float32, device="cuda")
        for e in range(case["E"]):
            q, s = _codes64(w[e].double().t())
            out[e] = (q * s).t()
        return out
    if case["kind"] == "matmul":
        x, offsets = _batched_rows(case, seed)
        codes, scales = _converted_matrices(case["E"], case["K"], case["C"], _generator(seed, 100))
        ends = [0, case["M"]] if offsets is None else offsets.tolist()
        return torch.cat([_times64(x[a:b].double(), codes[e], scales[e]) for e, (a, b) in enumerate(zip(ends, ends[1:]))])
    if case["kind"] == "layer":
        x, logits = _tokens(case, seed)
        idx, w = _route64(logits, case["k"])
        flat = idx.reshape(-1)
        perm = torch.sort(flat, stable=True)[1]
        offsets = torch.cat([flat.new_zeros(1), torch.cumsum(torch.bincount(flat, minlength=case["E"]), 0)])
        return dict(y=_experts64(x.double(), idx, w, _expert_matrices(case, seed)), idx=idx.int(), w=w,
                    offsets=offsets.int(), perm=perm.int(), inv_perm=torch.argsort(perm).int())
    st = _norm_inputs(case, seed)
    u = st["y"].double()
    u = _rms64(u) * st["gain_after"].double() if case["after"] else u
    gate = torch.ones((), dtype=torch.float64, device="cuda")
    gate = st["gate"].double()[None, :] if st["gate"] is not None else gate
    gate = st["row_gate"].double()[:, None] if st["row_gate"] is not None else gate
    x = torch.addcmul(st["x"].double(), u, gate, value=st["scale"])
    h = _rms64(x) * st["gain_before"].double()
    if case["kind"] == "block":
        idx, w = _route64(h @ _router_matrix(case, seed).double(), case["k"])
        return dict(x=x, y=_experts64(h, idx, w, _expert_matrices(case, seed)))
    if case["out"] == "int8":
        q, s = _codes64(h)
        h = q * s
    return dict(x=x, h=h)
