"""Cases over which the operators around the exchange are timed and checked:
routing, RMS norm with 8-bit output, the experts' 8-bit products, and one MoE
layer that runs them with layout, dispatch and combine.

A case names a kind of call and its shape (plain values); `prepare` makes what
a program holds before the call, `run` is one pass and returns every output,
`exact` gives the computed values in 64 bits.  With `own` false `run` computes
the operators in elementary torch operations in 32 bits, else it makes the
framework's calls.

Kinds:
  route       top-k experts and combine weights of router logits
  route_grad  gradient of the logits from that of the combine weights
  norm        residual addition, RMS norm, output in bf16 or 8 bits
  norm_grad   gradients of the norm's input and weight
  matmul      int8 products of the experts' windows (swiglu: gate and up
              channels joined in the epilogue)
  layer       norm, routing, layout, dispatch, product, quantisation, product,
              combine of one MoE layer

Shapes: T tokens, H hidden, E experts, k slots per token, rows routed rows,
K depth and N channels of a product, I an expert's inner width.
"""
from __future__ import annotations

import math

import torch

own = False

FP8_BLOCK = 128      # values that share one fp8 scale
FP8_MAX, INT8_MAX = 448.0, 127.0
AMAX_MIN = 2.0 ** -100
EPS = 1e-6


def _route(name, kind, T, E, k, f32=True, score="softmax", bias=False, groups=1, top=1,
           renorm=True, scale=1.0, dead=0.0, pad=0.0):
    """dead: share of experts masked by -inf logits, token by token; pad:
    share of tokens that are padding."""
    return _named(name, kind=kind, T=T, E=E, k=k, f32=f32, score=score, bias=bias,
                  groups=groups, top=top, renorm=renorm, scale=scale, dead=dead, pad=pad)


def _norm(name, kind, T, H, q="none", res="bf16", wf32=False):
    """q: "none" (bf16 output), "fp8" or "int8"; res: the residual's type."""
    return _named(name, kind=kind, T=T, H=H, q=q, res=res, wf32=wf32)


def _matmul(name, rows, E, K, N, swiglu=False, zipf=0.0, fixed=False):
    """fixed: windows of equal capacity, filled in part; else packed ones."""
    return _named(name, kind="matmul", rows=rows, E=E, K=K, N=N, swiglu=swiglu, zipf=zipf,
                  fixed=fixed)


def _layer(name, T, H, I, E, k, pad=0.0):
    return _named(name, kind="layer", T=T, H=H, I=I, E=E, k=k, f32=True, score="sigmoid",
                  bias=True, groups=1, top=1, renorm=True, scale=2.5, dead=0.0, pad=pad,
                  res="bf16", wf32=False, q="int8")


def _named(name, **c):
    return dict(c, name=name) if name else c


def listed():
    return [
        # routing of a small model's layer: bound by the launch
        _route("route_tiny", "route", 128, 16, 2),
        # a long prompt batch: sigmoid scores, a bias for balance, 4 of 8 groups
        _route("route_prefill", "route", 16384, 256, 8, score="sigmoid", bias=True, groups=8,
               top=4, scale=2.5),
        # training of a mid-width model: softmax weights as they are, bf16 logits
        _route("route_grad_large", "route_grad", 32768, 128, 8, f32=False, renorm=False),
        # a decode batch: rows for an fp8 dispatch
        _norm("norm_decode", "norm", 64, 7168, q="fp8"),
        # the same for a prompt batch
        _norm("norm_prefill", "norm", 16384, 7168, q="fp8"),
        # training: gradients at the largest batch, and at an odd small one
        _norm("norm_grad_large", "norm_grad", 32768, 4096),
        _norm("norm_grad_ragged", "norm_grad", 777, 2056, res="f32", wf32=True),
        # decode: few rows for each expert, bound by reading the weights
        _matmul("matmul_decode", 512, 32, 7168, 4096, swiglu=True),
        # a ragged batch over many small experts, some of them without rows
        _matmul("matmul_ragged", 4662, 96, 2064, 1416, zipf=0.5),
        # prompt batch: the first product of the experts, bound by arithmetic
        _matmul("matmul_prefill", 32768, 16, 7168, 4096, swiglu=True),
        # one MoE layer, low-latency decode ...
        _layer("layer_decode", 64, 7168, 2048, 32, 8),
        # ... and a prompt batch with some padding tokens
        _layer("layer_prefill", 4096, 7168, 2048, 32, 8, pad=0.05),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(["route", "route", "route_grad", "norm", "norm", "norm_grad", "matmul",
                       "matmul", "matmul", "layer"])
    if kind in ("route", "route_grad"):
        E = rng.choice([8, 16, 60, 64, 96, 128, 160, 256, 384, 512])
        k = rng.choice([1, 2, 4, 6, 8, 8, 10])
        k = min(k, E)
        T = round(_log(rng, 1, min(32768, 32768 * 256 // E)))
        groups, top = rng.choice([(1, 1), (1, 1), (4, 2), (8, 4)] if E % 8 == 0 else [(1, 1)])
        if k > E // groups * top:
            groups, top = 1, 1
        # one renormalised weight is 1 whatever its logit: no gradient to check
        renorm = rng.random() < 0.6 and (k > 1 or kind == "route")
        return _route(None, kind, T, E, k, rng.random() < 0.6, rng.choice(["softmax", "sigmoid"]),
                      rng.random() < 0.5, groups, top, renorm,
                      rng.choice([1.0, 2.5]), rng.choice([0.0, 0.0, 0.3]),
                      rng.choice([0.0, 0.05]))
    if kind in ("norm", "norm_grad"):
        q = rng.choice(["none", "fp8", "int8"]) if kind == "norm" else "none"
        step = {"none": 8, "fp8": 128, "int8": 16}[q]
        H = step * max(1, round(_log(rng, 128, 8192) / step))
        T = round(_log(rng, 1, min(32768, 16384 * 7168 // H)))
        return _norm(None, kind, T, H, q, rng.choice(["none", "bf16", "f32"]),
                     rng.random() < 0.4)
    if kind == "matmul":
        swiglu = rng.random() < 0.4
        K = 16 * round(_log(rng, 128, 8192) / 16)
        N = 16 * round(_log(rng, 64, 8192) / 16) + (0 if swiglu else rng.choice([0, 8]))
        E = round(_log(rng, 1, min(128, max(1, 470_000_000 // (K * N)))))
        zipf = rng.choice([0.0, 0.5])
        most = min(32768, int(6e11 / (K * N)))
        return _matmul(None, round(_log(rng, 1, most)), E, K, N, swiglu, zipf,
                       rng.random() < 0.3)
    H = 128 * round(_log(rng, 256, 7168) / 128)
    I = 16 * round(_log(rng, 128, 2048) / 16)
    E = rng.choice([4, 8, 16, 32])
    T = round(_log(rng, 1, 4096))
    return _layer(None, T, H, I, E, rng.choice([1, 2, 4]) if E < 8 else rng.choice([2, 4, 6, 8]),
                  rng.choice([0.0, 0.1]))


# ---------------------------------------------------------------- inputs
def _gen(seed, n):
    g = torch.Generator(device="cuda")
    g.manual_seed(16 * seed + n)
    return g


def _randn(g, *shape, dtype=torch.float32):
    """Normal values, drawn in pieces so that large ones need no second copy."""
    out = torch.empty(*shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    step = 1 << 26
    for i in range(0, flat.numel(), step):
        n = min(step, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, generator=g, device="cuda")
    return out


def _make_route(c, seed, s):
    g, T, E = _gen(seed, 1), c["T"], c["E"]
    x = torch.randn(T, E, generator=g, device="cuda") * 1.5
    if c["dead"]:
        x.masked_fill_(torch.rand(T, E, generator=g, device="cuda") < c["dead"], -math.inf)
        x[::97] = -math.inf                 # tokens that no expert may take
    s["logits"] = x if c["f32"] else x.bfloat16()
    s["bias"] = None
    if c["bias"]:                           # as steps of 0.001 leave it
        s["bias"] = torch.randint(-60, 61, (E,), generator=g, device="cuda").float() * 0.001
    s["live"] = None
    if c["pad"]:
        s["live"] = (torch.rand(T, generator=g, device="cuda") >= c["pad"]).to(torch.uint8)
    s["idx"] = torch.empty(T, c["k"], dtype=torch.int32, device="cuda")
    s["w"] = torch.empty(T, c["k"], device="cuda")


def _make_norm(c, seed, s):
    g, T, H = _gen(seed, 2), c["T"], c["H"]
    rt = torch.float32 if c["res"] == "f32" else torch.bfloat16
    gain = torch.exp(0.5 * torch.randn(T, 1, generator=g, device="cuda"))
    s["x"] = (_randn(g, T, H) * gain).bfloat16()
    s["residual"] = None if c["res"] == "none" else _randn(g, T, H, dtype=rt)
    wt = torch.float32 if c["wf32"] else torch.bfloat16
    s["weight"] = (1 + 0.2 * torch.randn(H, generator=g, device="cuda")).to(wt)
    s["rstd"] = torch.empty(T, device="cuda")
    s["sum"] = None if c["res"] == "none" else torch.empty(T, H, dtype=rt, device="cuda")
    if c["q"] == "none":
        s["y"] = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    else:
        s["q"] = torch.empty(T, H, dtype=torch.uint8 if c["q"] == "fp8" else torch.int8,
                             device="cuda")
        s["scales"] = torch.empty(T, H // FP8_BLOCK if c["q"] == "fp8" else 1, device="cuda")
        s["values"] = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")


def _make_norm_grad(c, seed, s):
    g, T, H = _gen(seed, 3), c["T"], c["H"]
    rt = torch.float32 if c["res"] == "f32" else torch.bfloat16
    s["h"] = _randn(g, T, H, dtype=rt)
    s["rstd"] = 1 / (s["h"].float().square().mean(1) + EPS).sqrt()
    s["grad_y"] = _randn(g, T, H, dtype=torch.bfloat16)
    s["grad_sum"] = None if c["res"] == "none" else _randn(g, T, H, dtype=rt)
    wt = torch.float32 if c["wf32"] else torch.bfloat16
    s["weight"] = (1 + 0.2 * torch.randn(H, generator=g, device="cuda")).to(wt)
    s["grad_x"] = torch.empty(T, H, dtype=rt, device="cuda")
    s["grad_w"] = torch.empty(H, device="cuda")


def _int8_weights(g, E, N, K):
    """Weights of about unit gain: int8 and one scale for each channel."""
    w = torch.randint(-127, 128, (E, N, K), generator=g, device="cuda", dtype=torch.int8)
    s = (0.5 + torch.rand(E, N, generator=g, device="cuda")) / (73.0 * math.sqrt(K))
    return w, s


def _counts(c, seed):
    """Rows of each expert: a multinomial draw, a few experts left out."""
    g = torch.Generator()
    g.manual_seed(seed)
    p = torch.arange(1, c["E"] + 1, dtype=torch.float64) ** -c["zipf"]
    p[7::11] = 0
    p = p[torch.randperm(c["E"], generator=g)]
    return torch.bincount(torch.multinomial(p, c["rows"], replacement=True, generator=g),
                          minlength=c["E"])


def _make_matmul(c, seed, s):
    g, E, N, K = _gen(seed, 4), c["E"], c["N"], c["K"]
    count = _counts(c, seed)
    if c["fixed"]:                          # twice the mean; rows beyond are dropped
        s["cap"] = max(8, -(-2 * c["rows"] // E))
        count = count.clamp(max=s["cap"])
    else:
        s["cap"] = int(count.max())
    start = torch.arange(E + 1) * s["cap"] if c["fixed"] else \
        torch.cat([torch.zeros(1, dtype=torch.long), count.cumsum(0)])
    rows = int(start[-1])
    s["a"] = (40 * _randn(g, rows, K)).round_().clamp_(-127, 127).to(torch.int8)
    s["a_scales"] = (0.5 + torch.rand(rows, 1, generator=g, device="cuda")) / 40
    s["wt"], s["wt_scales"] = _int8_weights(g, E, N, K)
    s["offset"] = start.to("cuda", torch.int32)
    s["count"] = count.to("cuda", torch.int32)
    out = N // 2 if c["swiglu"] else N
    s["y"] = torch.zeros(rows, out, dtype=torch.bfloat16, device="cuda")  # rows of no window stay


def _make_layer(c, seed, s):
    _make_route(c, seed, s)
    _make_norm(c, seed, s)
    g, H, I, E = _gen(seed, 5), c["H"], c["I"], c["E"]
    s["w13"], s["s13"] = _int8_weights(g, E, 2 * I, H)
    s["w2"], s["s2"] = _int8_weights(g, E, H, I)
    s["y"] = torch.empty(c["T"], H, dtype=torch.bfloat16, device="cuda")
    # rows that the fullest expert gets: how wide the plain form's batch is
    idx, _ = _route_plain(c, s)
    s["cap"] = max(1, int(torch.bincount(idx.reshape(-1).long() + 1, minlength=2)[1:].max()))


def prepare(case, seed):
    s, kind = {"case": case}, case["kind"]
    if kind in ("route", "route_grad"):
        _make_route(case, seed, s)
        if kind == "route_grad":
            s["idx"], s["w"] = _route_plain(case, s)
            s["grad_topk"] = torch.randn(case["T"], case["k"], generator=_gen(seed, 6),
                                         device="cuda")
            s["grad"] = torch.empty_like(s["logits"])
    elif kind == "layer":
        _make_layer(case, seed, s)
    else:
        {"norm": _make_norm, "norm_grad": _make_norm_grad, "matmul": _make_matmul}[kind](
            case, seed, s)
    return s


# ------------------------------------------------------------ plain forms
def _fold(x):
    """Sum over the last axis, padded with zeros to a power of two, the upper
    half added to the lower until one is left: the order in which the routing
    adds a softmax's terms."""
    n = 1 << max(0, x.shape[-1] - 1).bit_length()
    x = torch.nn.functional.pad(x, (0, n - x.shape[-1]))
    while n > 1:
        n //= 2
        x = x[..., :n] + x[..., n:]
    return x


def _scores(c, x, ok):
    """Softmax or sigmoid of the eligible logits, 0 elsewhere."""
    if c["score"] == "sigmoid":
        return torch.where(ok, 1 / (1 + torch.exp(-x)), 0.0)
    m = torch.where(ok, x, -math.inf).amax(-1, keepdim=True)
    e = torch.where(ok, torch.exp(x - m), 0.0)
    t = _fold(e)
    return e / torch.where(t > 0, t, 1.0)


def _first_max(v):
    """Largest value of the last axis and the first place that has it."""
    m = v.amax(-1, keepdim=True)
    n = torch.arange(v.shape[-1], device=v.device)
    return m, torch.where(v == m, n, v.shape[-1]).amin(-1, keepdim=True)


def _route_plain(c, s):
    E, k, G = c["E"], c["k"], c["groups"]
    x = s["logits"].float()
    ok = x > -math.inf
    if s["live"] is not None:
        ok = ok & (s["live"] != 0)[:, None]
    sc = _scores(c, x, ok)
    by_score = c["bias"] or (G > 1 and c["score"] == "sigmoid")
    key = x if not by_score else sc + s["bias"] if c["bias"] else sc
    key = torch.where(ok, key, -math.inf)
    if G > 1:
        gk = key.view(-1, G, E // G)
        best, at = _first_max(gk)
        if by_score:                        # the two highest keys of a group
            n = torch.arange(E // G, device=x.device)
            second = torch.where(n == at, -math.inf, gk).amax(-1, keepdim=True)
            best = torch.where(second > -math.inf, best + second, best)
        order = torch.sort(best[..., 0], dim=-1, descending=True, stable=True).indices
        keep = torch.zeros_like(best[..., 0], dtype=torch.bool).scatter_(
            1, order[:, :c["top"]], True)
        key = torch.where(keep[:, :, None], gk, -math.inf).view(-1, E)
    top = torch.sort(key, dim=-1, descending=True, stable=True)
    idx, used = top.indices[:, :k], top.values[:, :k] > -math.inf
    w = torch.where(used, sc.gather(1, idx), 0.0)
    if c["renorm"]:
        if c["score"] == "softmax":
            xc = torch.where(used, x.gather(1, idx), -math.inf)
            w = torch.where(used, torch.exp(xc - xc.amax(1, keepdim=True)), 0.0)
        t = w.sum(1, keepdim=True)
        w = w / torch.where(t > 0, t, 1.0)
    return torch.where(used, idx, -1).int(), w * c["scale"]


def _route_grad_plain(c, s):
    x, used = s["logits"].float(), s["idx"] >= 0
    idx = s["idx"].clamp(min=0).long()
    ok = x > -math.inf
    g = torch.where(used, s["grad_topk"] * c["scale"], 0.0)
    sc = _scores(c, x, ok)
    q = torch.where(used, sc.gather(1, idx), 0.0)
    if not c["renorm"] and c["score"] == "softmax":
        up = torch.zeros_like(x).scatter_add_(1, idx, g)
        return (sc * (up - (g * q).sum(1, keepdim=True))).to(s["logits"].dtype)
    d = g * q * (1 - q)
    if c["renorm"]:
        t = q.sum(1, keepdim=True)
        n = q / torch.where(t > 0, t, 1.0)
        d = n * (g - (g * n).sum(1, keepdim=True))
        if c["score"] == "sigmoid":
            d = d * (1 - q)
    return torch.zeros_like(x).scatter_add_(1, idx, torch.where(used, d, 0.0)).to(
        s["logits"].dtype)


def _quantise(y, q):
    """Codes (as float) and scales of rows y: fp8 per 128 values, int8 per row."""
    b = y.view(y.shape[0], -1, FP8_BLOCK) if q == "fp8" else y[:, None, :]
    most = FP8_MAX if q == "fp8" else INT8_MAX
    a = b.abs().amax(2, keepdim=True)
    low = a.clamp(min=AMAX_MIN)
    v = (b * (most / low)).clamp(-most, most)
    v = v.to(torch.float8_e4m3fn) if q == "fp8" else v.round()
    return v.view(y.shape), torch.where(a > 0, low / most, 1.0)[:, :, 0]


def _norm_plain(c, s):
    x = s["x"].float()
    h = x if s["residual"] is None else x + s["residual"].float()
    rstd = 1 / (h.square().mean(1) + EPS).sqrt()
    y = h * rstd[:, None] * s["weight"].float()
    out = {"rstd": rstd}
    if s["residual"] is not None:
        out["sum"] = h.to(s["residual"].dtype)
    return out, y


def _norm_out(c, s):
    out, y = _norm_plain(c, s)
    if c["q"] == "none":
        out["y"] = y.bfloat16()
    else:
        v, out["scales"] = _quantise(y, c["q"])
        if c["q"] == "fp8":
            out["q"] = v
        else:
            out["values"] = (v * out["scales"]).bfloat16()
    return out


def _norm_grad_plain(s):
    h, dy, rstd = s["h"].float(), s["grad_y"].float(), s["rstd"][:, None]
    u = dy * s["weight"].float()
    dx = rstd * (u - h * (rstd * rstd * (u * h).mean(1, keepdim=True)))
    if s["grad_sum"] is not None:
        dx = dx + s["grad_sum"].float()
    return {"grad_x": dx.to(s["h"].dtype), "grad_w": (dy * h * rstd).sum(0)}


def _matmul_plain(a, a_scales, w, w_scales, offset, count, cap, swiglu):
    """The windows as one padded batch; rows of no window give 0."""
    rows, E = a.shape[0], w.shape[0]
    n = torch.arange(cap, device=a.device)
    row = offset[:E, None].long() + n
    row = torch.where(n < count[:, None], row, rows)     # padding: one row past the end
    pad = torch.cat([a, a.new_zeros(1, a.shape[1])])[row].float()
    acc = torch.bmm(w.float(), pad.transpose(1, 2).contiguous()).transpose(1, 2)
    scale = torch.cat([a_scales, a_scales.new_ones(1, 1)])[row]
    v = acc * scale * w_scales[:, None, :]
    if swiglu:
        g, u = v.chunk(2, dim=-1)
        v = g / (1 + torch.exp(-g)) * u
    y = torch.zeros(rows + 1, v.shape[-1], dtype=torch.bfloat16, device=a.device)
    y[row.reshape(-1)] = v.reshape(-1, v.shape[-1]).bfloat16()
    return y[:rows]


def _layer_plain(c, s):
    T, E, k = c["T"], c["E"], c["k"]
    out, y = _norm_plain(c, s)
    q, scales = _quantise(y, "int8")
    idx, w = _route_plain(c, s)
    flat = idx.reshape(-1).long()
    key = torch.where(flat < 0, E, flat)
    order = torch.sort(key, stable=True).indices
    count = torch.bincount(key, minlength=E + 1)[:E]
    offset = count.cumsum(0) - count
    tok = order // k
    act = _matmul_plain(q[tok].to(torch.int8), scales[tok], s["w13"], s["s13"], offset, count,
                        s["cap"], True)
    q2, scales2 = _quantise(act.float(), "int8")
    rows = _matmul_plain(q2.to(torch.int8), scales2, s["w2"], s["s2"], offset, count, s["cap"],
                         False)
    slot = torch.empty_like(rows)
    slot[order] = rows
    y = (w[:, :, None] * slot.view(T, k, -1).float()).sum(1)
    return {"sum": out["sum"], "idx": idx, "w": w, "y": y.bfloat16()}


def _plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "route":
        return dict(zip(("idx", "w"), _route_plain(c, s)))
    if kind == "route_grad":
        return {"grad": _route_grad_plain(c, s)}
    if kind == "norm":
        return _norm_out(c, s)
    if kind == "norm_grad":
        return _norm_grad_plain(s)
    if kind == "matmul":
        return {"y": _matmul_plain(s["a"], s["a_scales"], s["wt"], s["wt_scales"], s["offset"],
                                   s["count"], s["cap"], c["swiglu"])}
    return _layer_plain(c, s)


# ------------------------------------------------------- framework's calls
def _route_args(c):
    """Keywords of the routing's options."""
    from paper_2607_26444_amd import moe
    by_score = c["bias"] or (c["groups"] > 1 and c["score"] == "sigmoid")
    return dict(score=moe.MOE_SCORE_SIGMOID if c["score"] == "sigmoid" else moe.MOE_SCORE_SOFTMAX,
                groups=c["groups"], top_groups=c["top"], group_top=2 if by_score else 1,
                renorm=c["renorm"], scale=c["scale"])


def _dtype(t):
    from paper_2607_26444_amd import moe
    return moe.MOE_DTYPE_F32 if t is not None and t.dtype == torch.float32 else moe.MOE_DTYPE_BF16


def _own_norm(c, s):
    from paper_2607_26444_amd import moe
    q = {"none": 0, "fp8": moe.MOE_DTYPE_FP8_E4M3, "int8": moe.MOE_DTYPE_INT8}[c["q"]]
    moe.moe_rmsnorm(s["x"], s["residual"], _dtype(s["residual"]), s["weight"],
                    _dtype(s["weight"]), EPS, c["T"], c["H"], s["sum"], s.get("y"), q,
                    s.get("q"), s.get("scales"), s["rstd"])
    out = {"rstd": s["rstd"]}
    if s["sum"] is not None:
        out["sum"] = s["sum"]
    if c["q"] == "none":
        out["y"] = s["y"]
    else:
        out["scales"] = s["scales"]
        if c["q"] == "fp8":
            out["q"] = s["q"].view(torch.float8_e4m3fn)
        else:
            out["values"] = torch.mul(s["q"], s["scales"], out=s["values"])
    return out


def _own(s):
    from paper_2607_26444_amd import moe
    c = s["case"]
    kind = c["kind"]
    if kind == "route":
        moe.moe_route(s["logits"], _dtype(s["logits"]), c["E"], s["bias"], s["live"], s["idx"],
                      s["w"], **s.setdefault("options", _route_args(c)))
        return {"idx": s["idx"], "w": s["w"]}
    if kind == "route_grad":
        o = s.setdefault("options", _route_args(c))
        moe.moe_route_backward(s["logits"], _dtype(s["logits"]), c["E"], s["idx"],
                               s["grad_topk"], s["grad"], score=o["score"], renorm=o["renorm"],
                               scale=o["scale"])
        return {"grad": s["grad"]}
    if kind == "norm":
        return _own_norm(c, s)
    if kind == "norm_grad":
        ws = torch.empty(moe.moe_rmsnorm_backward_workspace_bytes(c["T"], c["H"]),
                         dtype=torch.uint8, device="cuda")
        moe.moe_rmsnorm_backward(s["grad_y"], s["h"], _dtype(s["h"]), s["rstd"], s["weight"],
                                 _dtype(s["weight"]), s["grad_sum"], c["T"], c["H"],
                                 s["grad_x"], s["grad_w"], ws)
        return {"grad_x": s["grad_x"], "grad_w": s["grad_w"]}
    if kind == "matmul":
        moe.moe_expert_matmul(s["a"], s["a_scales"], s["a"].shape[0], s["wt"], s["wt_scales"],
                              c["E"], c["N"], c["K"], s["offset"], s["count"],
                              moe.MOE_ACT_SWIGLU if c["swiglu"] else moe.MOE_ACT_NONE, s["y"])
        return {"y": s["y"]}
    if "layer" not in s:                    # the handle that a program keeps
        from paper_2607_26444_amd.layer import MoeLayer
        s["layer"] = MoeLayer(c["T"], c["H"], c["I"], c["E"], c["k"], s["weight"], s["w13"],
                              s["s13"], s["w2"], s["s2"], bias=s["bias"], eps=EPS,
                              **_route_args(c))
    layer = s["layer"]
    y = layer.forward(s["x"], s["residual"], s["logits"], token_mask=s["live"])
    return {"sum": layer.sum, "idx": layer.topk_idx, "w": layer.topk_w, "y": y}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ work
def work(case):
    c, kind = case, case["kind"]
    if kind in ("route", "route_grad"):
        size = 4 if c["f32"] else 2
        b = c["T"] * (c["E"] * size * (1 if kind == "route" else 2) + 8 * c["k"])
        return {"bytes": float(b), "flops": 8.0 * c["T"] * c["E"]}
    if kind == "norm":
        r = {"none": 0, "bf16": 4, "f32": 8}[c["res"]]
        b = c["T"] * c["H"] * (2 + r + (2 if c["q"] == "none" else 1)) + 4 * c["T"]
        if c["q"] != "none":
            b += 4 * c["T"] * (c["H"] // FP8_BLOCK if c["q"] == "fp8" else 1)
        return {"bytes": float(b), "flops": 6.0 * c["T"] * c["H"]}
    if kind == "norm_grad":
        r = 4 if c["res"] == "f32" else 2
        b = c["T"] * c["H"] * (2 + r * (2 if c["res"] == "none" else 3)) + 4 * c["T"]
        return {"bytes": float(b), "flops": 10.0 * c["T"] * c["H"]}
    if kind == "matmul":
        return _product_work(c["rows"], min(c["E"], c["rows"]), c["K"], c["N"], c["swiglu"])
    rows = c["T"] * c["k"] * (1 - c["pad"])
    E = min(c["E"], rows)
    one = _product_work(rows, E, c["H"], 2 * c["I"], True)
    two = _product_work(rows, E, c["I"], c["H"], False)
    # outside the experts: x, residual, sum, logits, y
    b = c["T"] * (8 * c["H"] + 4 * c["E"])
    return {"bytes": b + E * 3.0 * c["I"] * c["H"], "flops": one["flops"] + two["flops"]}


def _product_work(rows, E, K, N, swiglu):
    out = N // 2 if swiglu else N
    return {"bytes": float(rows * (K + 4 + 2 * out) + E * N * (K + 4)),
            "flops": 2.0 * rows * K * N}


# ----------------------------------------------------------------- exact
def _best(v, n):
    """The n highest of the last axis, of equal ones the first."""
    values, at = torch.sort(v, dim=-1, descending=True, stable=True)
    return values[..., :n], at[..., :n]


def _exact_route(c, s):
    """Token by expert, in 64 bits: weights [T,k] (0 where a slot is unused)
    and, for the layer, the experts."""
    x = s["logits"].double()
    if s["live"] is not None:
        x = x.masked_fill(s["live"][:, None] == 0, -math.inf)
    if c["score"] == "softmax":
        p = torch.nan_to_num(torch.softmax(x, -1), nan=0.0)
    else:
        p = torch.sigmoid(x)
    rank = p if s["bias"] is None else p + s["bias"].double()
    rank = rank.masked_fill(x == -math.inf, -math.inf)
    G = c["groups"]
    if G > 1:
        parts = rank.view(x.shape[0], G, -1)
        n = min(2 if c["bias"] or c["score"] == "sigmoid" else 1, parts.shape[2])
        two, _ = _best(parts, n)
        total = two.masked_fill(two == -math.inf, 0.0).sum(-1)
        total = total.masked_fill(two[..., 0] == -math.inf, -math.inf)
        out = torch.ones_like(total, dtype=torch.bool)
        out.scatter_(1, _best(total, c["top"])[1], False)
        rank = parts.masked_fill(out[:, :, None], -math.inf).view_as(rank)
    values, idx = _best(rank, c["k"])
    w = p.gather(1, idx).masked_fill(values == -math.inf, 0.0)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    return w * c["scale"], idx.masked_fill(values == -math.inf, -1)


def _exact_route_grad(c, s):
    """By automatic differentiation of the weights in 64 bits."""
    x = s["logits"].double().requires_grad_()
    used = s["idx"] >= 0
    p = torch.softmax(x, -1) if c["score"] == "softmax" else torch.sigmoid(x)
    v = p.gather(1, s["idx"].clamp(min=0).long())
    v = torch.where(used, v, torch.zeros_like(v))
    if c["renorm"]:
        t = v.sum(1, keepdim=True)
        v = v / torch.where(t > 0, t, torch.ones_like(t))
    loss = torch.where(used, v * s["grad_topk"].double() * c["scale"], torch.zeros_like(v)).sum()
    (d,) = torch.autograd.grad(loss, x)
    return torch.where((x == -math.inf) | (used.sum(1, keepdim=True) == 0),
                       torch.zeros_like(d), d)


def _exact_norm(c, s, n=None):
    """Sum, reciprocal deviation and normed rows of the first n tokens."""
    h = s["x"][:n].double()
    if s["residual"] is not None:
        h = h + s["residual"][:n].double()
    r = torch.rsqrt(h.pow(2).sum(1) / c["H"] + EPS)
    return h, r, h * r[:, None] * s["weight"].double()


def _exact_codes(y, block, most):
    """Values in units of their scale, before rounding, and the scales."""
    b = y.view(y.shape[0], y.shape[1] // block, block)
    a = b.abs().amax(2)
    sc = torch.where(a > 0, a.clamp(min=AMAX_MIN) / most, torch.ones_like(a))
    return (b / sc[:, :, None]).view_as(y), sc


def _exact_expert(a, w, w_scales):
    return (a @ w.double().T) * w_scales.double()


def exact(case, seed):
    c, kind = case, case["kind"]
    s = prepare(case, seed)
    if kind == "route":
        return {"idx": None, "w": _exact_route(c, s)[0]}
    if kind == "route_grad":
        return {"grad": _exact_route_grad(c, s)}
    if kind == "norm":
        h, r, y = _exact_norm(c, s)
        out = {"rstd": r}
        if s["residual"] is not None:
            out["sum"] = h
        if c["q"] == "none":
            out["y"] = y
        else:
            v, out["scales"] = _exact_codes(y, FP8_BLOCK if c["q"] == "fp8" else c["H"],
                                            FP8_MAX if c["q"] == "fp8" else INT8_MAX)
            if c["q"] == "fp8":
                out["q"] = v
            else:
                out["values"] = y
        return out
    if kind == "norm_grad":
        h = s["h"].double().requires_grad_()
        w = s["weight"].double().requires_grad_()
        # the forward's reciprocal deviation is an input: its derivative is added
        r = s["rstd"].double()
        g = s["grad_y"].double()
        dh, dw = torch.autograd.grad((g * h * r[:, None] * w).sum(), (h, w))
        dr = (g * h * w).sum(1).detach()
        dh = dh - (dr * r.pow(3) / c["H"])[:, None] * h.detach()
        if s["grad_sum"] is not None:
            dh = dh + s["grad_sum"].double()
        return {"grad_x": dh, "grad_w": dw}
    if kind == "matmul":
        y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
        for e, (o, n) in enumerate(zip(s["offset"].tolist(), s["count"].tolist())):
            v = _exact_expert(s["a"][o:o + n].double() * s["a_scales"][o:o + n].double(),
                              s["wt"][e], s["wt_scales"][e])
            if c["swiglu"]:
                g, u = v.chunk(2, -1)
                v = g * torch.sigmoid(g) * u
            y[o:o + n] = v
        return {"y": y}
    h, _, normed = _exact_norm(c, s)
    w, idx = _exact_route(c, s)
    v, sc = _exact_codes(normed, c["H"], INT8_MAX)
    a = v.round() * sc
    y = torch.zeros_like(h)
    for e in range(c["E"]):
        tok, slot = torch.nonzero(idx == e, as_tuple=True)
        g, u = _exact_expert(a[tok], s["w13"][e], s["s13"][e]).chunk(2, -1)
        v, sc = _exact_codes(g * torch.sigmoid(g) * u, c["I"], INT8_MAX)
        rows = _exact_expert(v.round() * sc, s["w2"][e], s["s2"][e])
        y.index_add_(0, tok, rows * w[tok, slot][:, None])
    return {"sum": h, "idx": None, "w": w, "y": y}
