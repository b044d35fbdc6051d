"""Cases over which the operators of a balanced router and of 4-bit experts are
timed and checked: the balance loss of a routed batch with its gradient, the
quantisation of rows to microscaled 4-bit floats, the experts' products on them,
and one MoE layer with such weights.

A case names a kind of call and its shape (plain values); `prepare` makes what
a program holds before the call, `run` is one pass and returns every output,
`exact` gives the computed values in 64 bits.  With `own` false `run` computes
the operators in elementary torch operations in 32 bits, else it makes the
framework's calls.

Kinds:
  balance       slots of each expert, mean scores and the balance loss of every
                sequence
  balance_grad  gradient of the logits from that of the losses
  quantize      4-bit codes, block scales and the values they stand for
  matmul        products of the experts' windows (swiglu: gate and up channels
                joined in the epilogue)
  layer         norm, routing, layout, quantisation, dispatch, products, combine

Shapes: T tokens, H hidden, E experts, k slots per token, seq tokens of a
sequence, rows routed rows, K depth and N channels of a product, I an expert's
inner width.

Blocks of 32 neighbouring values of a row share a scale 2^(s - 127), s one byte;
a value is a sign and one of MAGNITUDES, two to a byte, the first in the low
half.  With a the block's largest magnitude the scale is the power of two that
puts a into [3.5, 7); values round to nearest even and end at 6.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 32                       # values that share a scale
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-6


def _named(name, **c):
    return dict(c, name=name) if name else c


def _balance(name, kind, T, E, k, seq=0, f32=True, score="softmax", pad=0.0, dead=0.0, add=False):
    """seq 0: the batch is one sequence; pad: share of padding at the sequences'
    ends; dead: share of experts masked by -inf logits; add: the gradient is added to
    another one of the same logits."""
    return _named(name, kind=kind, T=T, E=E, k=k, seq=seq or T, f32=f32, score=score, pad=pad,
                  dead=dead, add=add)


def _quantize(name, rows, H, skip=0.0):
    """skip: share of rows that no slot fills."""
    return _named(name, kind="quantize", rows=rows, H=H, skip=skip)


def _matmul(name, rows, E, K, N, swiglu=False, zipf=0.0, fixed=False):
    """rows: routed rows, spread over the experts with probabilities that fall
    as rank^-zipf; fixed: windows of equal capacity, filled in part."""
    return _named(name, kind="matmul", rows=rows, E=E, K=K, N=N, swiglu=swiglu, zipf=zipf,
                  fixed=fixed)


def _layer(name, T, H, I, E, k, pad=0.0):
    return _named(name, kind="layer", T=T, H=H, I=I, E=E, k=k, pad=pad)


def listed():
    return [
        # a small model's step: bound by the launch
        _balance("balance_tiny", "balance", 128, 16, 2, f32=False),
        # training on padded sequences, a loss for each
        _balance("balance_sequences", "balance", 32768, 256, 8, seq=4096, score="sigmoid", pad=0.1),
        # its gradient over a whole batch, added to that of the combine weights
        _balance("balance_grad_large", "balance_grad", 32768, 128, 8, f32=False, add=True),
        # an odd batch of short sequences
        _balance("balance_grad_ragged", "balance_grad", 777, 60, 6, seq=111, score="sigmoid",
                 pad=0.2),
        # rows of a decode batch
        _quantize("quantize_decode", 64, 7168),
        # rows of a prompt batch, a few of them padding
        _quantize("quantize_prefill", 16384, 7168, skip=0.05),
        # one token's eight slots
        _matmul("matmul_token", 8, 32, 7168, 4096, swiglu=True),
        # decode: few rows for each expert, bound by reading the weights
        _matmul("matmul_decode", 512, 32, 7168, 4096, swiglu=True),
        # a ragged batch over many small experts, some of them without rows
        _matmul("matmul_ragged", 4662, 96, 2080, 1416, zipf=0.5),
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
    kind = rng.choice(["balance", "balance", "balance_grad", "balance_grad", "quantize", "quantize",
                       "matmul", "matmul", "matmul", "layer"])
    if kind in ("balance", "balance_grad"):
        E = rng.choice([4, 8, 16, 60, 64, 96, 128, 160, 256, 384, 512])
        # with every expert chosen all loads are equal and the gradient is 0
        k = min(E - 1, rng.choice([1, 2, 4, 6, 8, 8, 10]))
        most = min(32768, 32768 * 256 // E)
        S = rng.choice([1, 1, round(_log(rng, 1, 64))])
        seq = max(1, round(_log(rng, 1, most // S)))
        return _balance(None, kind, S * seq, E, k, seq, rng.random() < 0.6,
                        rng.choice(["softmax", "sigmoid"]), rng.choice([0.0, 0.1, 0.3]),
                        rng.choice([0.0, 0.0, 0.3]), kind == "balance_grad" and rng.random() < 0.5)
    if kind == "quantize":
        H = BLOCK * round(_log(rng, 64, 8192) / BLOCK)
        return _quantize(None, round(_log(rng, 1, min(32768, 16384 * 7168 // H))), H,
                         rng.choice([0.0, 0.1]))
    if kind == "matmul":
        swiglu = rng.random() < 0.4
        K = BLOCK * round(_log(rng, 128, 8192) / BLOCK)
        N = 16 * round(_log(rng, 64, 8192) / 16) + (0 if swiglu else rng.choice([0, 8]))
        E = round(_log(rng, 1, min(128, max(1, 470_000_000 // (K * N)))))
        most = min(32768, int(6e11 / (K * N)))
        return _matmul(None, round(_log(rng, 1, most)), E, K, N, swiglu, rng.choice([0.0, 0.5]),
                       rng.random() < 0.3)
    H = BLOCK * round(_log(rng, 256, 7168) / BLOCK)
    I = BLOCK * round(_log(rng, 128, 2048) / BLOCK)
    E = rng.choice([4, 8, 16, 32])
    return _layer(None, round(_log(rng, 1, 4096)), H, I, E,
                  rng.choice([1, 2, 4]) if E < 8 else rng.choice([2, 4, 6, 8]),
                  rng.choice([0.0, 0.1]))


# ---------------------------------------------------------------- inputs
def _gen(seed, n):
    g = torch.Generator(device="cuda")
    g.manual_seed(16 * seed + n)
    return g


def _scale_cols(K):
    """Bytes of a row of scales: whole fours."""
    return -(-K // (4 * BLOCK)) * 4


def _make_balance(c, seed, s):
    g, T, E = _gen(seed, 1), c["T"], c["E"]
    x = torch.randn(T, E, generator=g, device="cuda") * 1.5
    x += 0.7 * torch.randn(E, generator=g, device="cuda")       # some experts are preferred
    if c["dead"]:
        x.masked_fill_(torch.rand(T, E, generator=g, device="cuda") < c["dead"], -math.inf)
        x[::97] = -math.inf                 # tokens that no expert may take
    s["logits"] = x if c["f32"] else x.bfloat16()
    S = T // c["seq"]
    s["live"] = None
    if c["pad"]:                            # sequences end early, one is empty at times
        lengths = (1 - 2 * c["pad"] * torch.rand(S, 1, generator=g, device="cuda")) * c["seq"]
        lengths[5::7] = 0
        n = torch.arange(c["seq"], device="cuda")
        s["live"] = (n < lengths.round()).to(torch.uint8).reshape(-1)
    s["idx"] = _choose(c, s)[0]
    new = dict(dtype=torch.int32, device="cuda")
    s["count"], s["tokens"] = torch.empty(S, E, **new), torch.empty(S, **new)
    s["mean"], s["loss"] = torch.empty(S, E, device="cuda"), torch.empty(S, device="cuda")


def _make_balance_grad(c, seed, s):
    _make_balance(c, seed, s)
    g, x = _gen(seed, 2), s["logits"]
    s["count"], s["tokens"] = _counts_plain(c, s)
    s["grad_loss"] = 0.5 + torch.rand(c["T"] // c["seq"], generator=g, device="cuda")
    s["sum"] = None
    if c["add"]:                            # of the size that the loss's gradient has
        s["sum"] = (torch.randn(x.shape, generator=g, device="cuda") / c["T"]).to(x.dtype)
    s["grad"] = torch.empty_like(x)


def _rows(g, rows, H):
    """bf16 rows of different gain, with a few columns of large values."""
    x = torch.randn(rows, H, generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))
    x[:, torch.randint(0, H, (max(1, H // 512),), generator=g, device="cuda")] *= 12
    return x.bfloat16()


def _make_quantize(c, seed, s):
    g, rows, H = _gen(seed, 3), c["rows"], c["H"]
    s["x"] = _rows(g, rows, H)
    s["src"] = None
    if c["skip"]:
        src = torch.arange(rows, device="cuda", dtype=torch.int32)
        s["src"] = torch.where(torch.rand(rows, generator=g, device="cuda") < c["skip"], -1, src)
    byte = dict(dtype=torch.uint8, device="cuda")       # rows that are skipped stay
    s["q"] = torch.zeros(rows, H // 2, **byte)
    s["scales"] = torch.zeros(rows, _scale_cols(H), **byte)
    s["values"] = torch.zeros(rows, H, dtype=torch.bfloat16, device="cuda")


def _codes(g, rows, K, exponent):
    """Codes as normal values have them, scales of three neighbouring exponents."""
    share = torch.tensor([0.14, 0.25, 0.2, 0.15, 0.13, 0.08, 0.035, 0.015])
    table = torch.multinomial(share, 256, replacement=True, generator=torch.Generator().manual_seed(1))
    table = (table + 8 * (torch.arange(256) % 2)).to("cuda", torch.uint8)
    q = torch.empty(rows, K // 2, dtype=torch.uint8, device="cuda")
    flat, step = q.view(-1), 1 << 26
    for i in range(0, flat.numel(), step):
        n = min(step, flat.numel() - i)
        r = torch.randint(0, 256, (2, n), generator=g, device="cuda", dtype=torch.int32)
        flat[i:i + n] = table[r[0]] | table[r[1]] << 4
    scales = torch.zeros(rows, _scale_cols(K), dtype=torch.uint8, device="cuda")
    scales[:, :K // BLOCK] = torch.randint(exponent - 1, exponent + 2, (rows, K // BLOCK),
                                           generator=g, device="cuda", dtype=torch.uint8)
    return q, scales


def _weights(g, E, N, K):
    """Weights of about unit gain."""
    q, scales = _codes(g, E * N, K, 126 - round(0.5 * math.log2(K)))
    return q.view(E, N, -1), scales.view(E, N, -1)


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
    s["a"], s["a_scales"] = _codes(g, rows, K, 126)
    s["wt"], s["wt_scales"] = _weights(g, E, N, K)
    s["offset"] = start.to("cuda", torch.int32)
    s["count"] = count.to("cuda", torch.int32)
    out = N // 2 if c["swiglu"] else N
    s["y"] = torch.zeros(rows, out, dtype=torch.bfloat16, device="cuda")  # rows of no window stay


def _make_layer(c, seed, s):
    g, T, H, I, E = _gen(seed, 5), c["T"], c["H"], c["I"], c["E"]
    s["x"] = _rows(g, T, H)
    s["residual"] = torch.randn(T, H, generator=g, device="cuda").bfloat16()
    s["weight"] = (1 + 0.2 * torch.randn(H, generator=g, device="cuda")).bfloat16()
    s["logits"] = torch.randn(T, E, generator=g, device="cuda") * 1.5
    s["live"] = None
    if c["pad"]:
        s["live"] = (torch.rand(T, generator=g, device="cuda") >= c["pad"]).to(torch.uint8)
    s["w13"], s["s13"] = _weights(g, E, 2 * I, H)
    s["w2"], s["s2"] = _weights(g, E, H, I)
    # rows that the fullest expert gets: how wide the plain form's batch is
    idx, _ = _choose(c, s)
    s["cap"] = max(1, int(torch.bincount(idx.reshape(-1).long() + 1, minlength=2)[1:].max()))


def prepare(case, seed):
    s = {"case": case}
    {"balance": _make_balance, "balance_grad": _make_balance_grad, "quantize": _make_quantize,
     "matmul": _make_matmul, "layer": _make_layer}[case["kind"]](case, seed, s)
    return s


# ------------------------------------------------------------ plain forms
def _choose(c, s):
    """The k experts of the highest logits, equal ones in their order, and weights that
    are a softmax over them; -1 and 0 where there is none."""
    x = s["logits"].float()
    if s["live"] is not None:
        x = torch.where(s["live"][:, None] != 0, x, -math.inf)
    top = torch.sort(x, dim=-1, descending=True, stable=True)
    v, idx = top.values[:, :c["k"]], top.indices[:, :c["k"]]
    used = v > -math.inf
    w = torch.where(used, torch.exp(v - torch.where(used[:, :1], v[:, :1], 0.0)), 0.0)
    t = w.sum(1, keepdim=True)
    return torch.where(used, idx, -1).int(), w / torch.where(t > 0, t, 1.0)


def _counts_plain(c, s):
    """Slots of each expert in each sequence, and the sequences' live tokens."""
    T, E, S = c["T"], c["E"], c["T"] // c["seq"]
    idx = s["idx"].long()
    live = torch.ones(T, dtype=torch.bool, device=idx.device) if s["live"] is None else s["live"] != 0
    ok = (idx >= 0) & (idx < E) & live[:, None]
    at = torch.arange(T, device=idx.device)[:, None] // c["seq"] * E + idx
    count = torch.bincount(torch.where(ok, at, S * E).reshape(-1), minlength=S * E + 1)[:S * E]
    return count.view(S, E).int(), live.view(S, -1).sum(1).int()


def _shares(c, s):
    """A token's scores over their sum (0 for an expert or a token that takes no
    part), and the share that sigmoid scores keep of a change, 1 - score."""
    x = s["logits"].float()
    ok = x > -math.inf
    if s["live"] is not None:
        ok = ok & (s["live"] != 0)[:, None]
    rest = None
    if c["score"] == "sigmoid":
        e = torch.where(ok, 1 / (1 + torch.exp(-x)), 0.0)
        rest = torch.where(ok, 1 / (1 + torch.exp(x)), 0.0)
    else:
        m = torch.where(ok, x, -math.inf).amax(-1, keepdim=True)
        e = torch.where(ok, torch.exp(x - m), 0.0)
    t = e.sum(-1, keepdim=True)
    return e / torch.where(t > 0, t, 1.0), rest


def _loads(count):
    """Slots of an expert over those of the mean one."""
    total = count.sum(-1, keepdim=True).float()
    return count.float() * count.shape[-1] / torch.where(total > 0, total, 1.0)


def _balance_plain(c, s):
    count, tokens = _counts_plain(c, s)
    p, _ = _shares(c, s)
    mean = p.view(-1, c["seq"], c["E"]).sum(1) / tokens.clamp(min=1)[:, None].float()
    return {"count": count, "tokens": tokens, "mean": mean, "loss": (_loads(count) * mean).sum(-1)}


def _balance_grad_plain(c, s):
    p, rest = _shares(c, s)
    p = p.view(-1, c["seq"], c["E"])
    f = _loads(s["count"])[:, None, :]
    d = p * (f - (f * p).sum(-1, keepdim=True))
    if rest is not None:
        d = d * rest.view(d.shape)
    d = (d * (s["grad_loss"] / s["tokens"].clamp(min=1).float())[:, None, None]).view(c["T"], c["E"])
    if s["sum"] is not None:
        d = d + s["sum"].float()
    return {"grad": d.to(s["logits"].dtype)}


def _quantise(x):
    """Codes [rows, H] and scale bytes [rows, H / BLOCK] of bf16 rows."""
    b = x.float().view(x.shape[0], -1, BLOCK)
    a = b.abs().amax(2)
    # the exponent of a, one more from 1.75 times a power of two on
    e = ((a.view(torch.int32) + 0x200000) >> 23) - 2
    e = torch.where(a > 0, e.clamp(0, 254), 127)
    m = (b * ((254 - e) << 23).view(torch.float32)[:, :, None]).abs()
    code = sum(cut.to(torch.uint8) for cut in (m > 0.25, m >= 0.75, m > 1.25, m >= 1.75, m > 2.5,
                                               m >= 3.5, m > 5.0))
    return (code + 8 * torch.signbit(b).to(torch.uint8)).view(x.shape), e.to(torch.uint8)


def _values(q, scales, K):
    """float32 values of packed codes [..., K / 2] and scales [..., cols]."""
    one = torch.tensor(MAGNITUDES, device=q.device)
    one = torch.cat([one, -one])
    n = torch.arange(256, device=q.device)
    pair = torch.stack([one[n & 15], one[n >> 4]], 1)
    v = pair[q.int()].view(*q.shape[:-1], K // BLOCK, BLOCK)
    scale = (scales[..., :K // BLOCK].int() << 23).view(torch.float32)
    return (v * scale[..., None]).view(*q.shape[:-1], K)


def _quantize_plain(c, s):
    code, e = _quantise(s["x"])
    scales = torch.nn.functional.pad(e, (0, _scale_cols(c["H"]) - e.shape[1]))
    q = code[:, 0::2] | code[:, 1::2] << 4
    values = _values(q, scales, c["H"]).bfloat16()
    if s["src"] is not None:
        keep = (s["src"] >= 0)[:, None]
        q, scales, values = (torch.where(keep, t, t.new_zeros(())) for t in (q, scales, values))
    return {"q": q, "scales": scales, "values": values}


def _matmul_plain(a, w, offset, count, cap, swiglu):
    """The windows of float32 rows a as one padded batch; rows of no window give 0."""
    rows, E = a.shape[0], w.shape[0]
    n = torch.arange(cap, device=a.device)
    row = offset[:E, None].long() + n
    row = torch.where(n < count[:, None], row, rows)     # padding: one row past the end
    pad = torch.cat([a, a.new_zeros(1, a.shape[1])])[row]
    v = torch.bmm(w, pad.transpose(1, 2).contiguous()).transpose(1, 2)
    if swiglu:
        g, u = v.chunk(2, dim=-1)
        v = g / (1 + torch.exp(-g)) * u
    y = torch.zeros(rows + 1, v.shape[-1], dtype=torch.bfloat16, device=a.device)
    y[row.reshape(-1)] = v.reshape(-1, v.shape[-1]).bfloat16()
    return y[:rows]


def _rounded(x):
    """float32 values that bf16 rows have after their quantisation."""
    code, e = _quantise(x)
    return _values(code[:, 0::2] | code[:, 1::2] << 4, e, x.shape[1])


def _layer_plain(c, s):
    T, E, k = c["T"], c["E"], c["k"]
    h = s["x"].float() + s["residual"].float()
    rstd = 1 / (h.square().mean(1, keepdim=True) + EPS).sqrt()
    x = _rounded((h * rstd * s["weight"].float()).bfloat16())
    idx, w = _choose(c, s)
    flat = idx.reshape(-1).long()
    key = torch.where(flat < 0, E, flat)
    order = torch.sort(key, stable=True).indices
    count = torch.bincount(key, minlength=E + 1)[:E]
    offset = count.cumsum(0) - count
    act = _matmul_plain(x[order // k], _values(s["w13"], s["s13"], c["H"]), offset, count, s["cap"],
                        True)
    rows = _matmul_plain(_rounded(act), _values(s["w2"], s["s2"], c["I"]), offset, count, s["cap"],
                         False)
    slot = torch.empty_like(rows)
    slot[order] = rows
    y = (w[:, :, None] * slot.view(T, k, -1).float()).sum(1)
    return {"sum": h.bfloat16(), "idx": idx, "w": w, "y": y.bfloat16()}


def _plain(s):
    c = s["case"]
    if c["kind"] == "balance":
        return _balance_plain(c, s)
    if c["kind"] == "balance_grad":
        return _balance_grad_plain(c, s)
    if c["kind"] == "quantize":
        return _quantize_plain(c, s)
    if c["kind"] == "matmul":
        return {"y": _matmul_plain(_values(s["a"], s["a_scales"], c["K"]),
                                   _values(s["wt"], s["wt_scales"], c["K"]), s["offset"],
                                   s["count"], s["cap"], c["swiglu"])}
    return _layer_plain(c, s)


# ------------------------------------------------------- framework's calls
def _own(s):
    from paper_2607_26444_amd import moe
    c = s["case"]
    kind = c["kind"]
    if kind in ("balance", "balance_grad"):
        dtype = moe.MOE_DTYPE_F32 if c["f32"] else moe.MOE_DTYPE_BF16
        score = moe.MOE_SCORE_SIGMOID if c["score"] == "sigmoid" else moe.MOE_SCORE_SOFTMAX
    if kind == "balance":
        if "workspace" not in s:            # as a training loop keeps it
            s["workspace"] = torch.empty(
                moe.moe_balance_workspace_bytes(c["T"], c["E"], c["seq"]), dtype=torch.uint8,
                device="cuda")
        moe.moe_balance(s["logits"], dtype, c["E"], s["idx"], s["live"], s["count"], s["tokens"],
                        s["mean"], s["loss"], s["workspace"], score=score, seq_len=c["seq"])
        return {"count": s["count"], "tokens": s["tokens"], "mean": s["mean"], "loss": s["loss"]}
    if kind == "balance_grad":
        moe.moe_balance_backward(s["logits"], dtype, c["T"], c["E"], s["live"], s["count"],
                                 s["tokens"], s["grad_loss"], s["sum"], s["grad"], score=score,
                                 seq_len=c["seq"])
        return {"grad": s["grad"]}
    if kind == "quantize":
        moe.moe_quantize_mx(s["x"], c["rows"], c["H"], s["q"], s["scales"], values=s["values"],
                            row_src=s["src"])
        return {"q": s["q"], "scales": s["scales"], "values": s["values"]}
    if kind == "matmul":
        moe.moe_expert_matmul_mx(s["a"], s["a_scales"], s["a"].shape[0], s["wt"], s["wt_scales"],
                                 c["E"], c["N"], c["K"], s["offset"], s["count"],
                                 moe.MOE_ACT_SWIGLU if c["swiglu"] else moe.MOE_ACT_NONE, s["y"])
        return {"y": s["y"]}
    if "layer" not in s:                    # the handle that a program keeps
        from paper_2607_26444_amd.layer import MoeLayer
        s["layer"] = MoeLayer(c["T"], c["H"], c["I"], c["E"], c["k"], s["weight"], s["w13"],
                              s["s13"], s["w2"], s["s2"], eps=EPS)
    layer = s["layer"]
    y = layer.forward(s["x"], s["residual"], s["logits"], token_mask=s["live"])
    return {"sum": layer.sum, "idx": layer.topk_idx, "w": layer.topk_w, "y": y}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ work
def work(case):
    c, kind = case, case["kind"]
    if kind in ("balance", "balance_grad"):
        size, n = 4 if c["f32"] else 2, c["T"] * c["E"]
        if kind == "balance":
            b = n * size + 4 * c["T"] * c["k"]
        else:
            b = n * size * (3 if c["add"] else 2)
        return {"bytes": float(b + 8 * c["E"] * c["T"] // c["seq"]), "flops": 10.0 * n}
    if kind == "quantize":
        rows = c["rows"] * (1 - c["skip"])
        return {"bytes": rows * c["H"] * (2 + 0.5 + 1 / BLOCK + 2), "flops": 6.0 * rows * c["H"]}
    if kind == "matmul":
        return _product_work(c["rows"], min(c["E"], c["rows"]), c["K"], c["N"], c["swiglu"])
    rows = c["T"] * c["k"] * (1 - c["pad"])
    E = min(c["E"], rows)
    one = _product_work(rows, E, c["H"], 2 * c["I"], True)
    two = _product_work(rows, E, c["I"], c["H"], False)
    # outside the experts: x, residual, sum, logits, y
    b = c["T"] * (8 * c["H"] + 4 * c["E"])
    return {"bytes": b + E * 3.0 * c["I"] * c["H"] * (0.5 + 1 / BLOCK),
            "flops": one["flops"] + two["flops"]}


def _product_work(rows, E, K, N, swiglu):
    out = N // 2 if swiglu else N
    deep = K * (0.5 + 1 / BLOCK)
    return {"bytes": float(rows * (deep + 2 * out) + E * N * deep), "flops": 2.0 * rows * K * N}


# ----------------------------------------------------------------- exact
def _exact_shares(c, x, live):
    """[T, E] in 64 bits, differentiable: scores over their sum."""
    off = x == -math.inf
    if live is not None:
        off = off | (live[:, None] == 0)
    if c["score"] == "sigmoid":
        v = torch.sigmoid(x).masked_fill(off, 0.0)
    else:
        top = x.detach().masked_fill(off, -1e30).amax(1, keepdim=True)
        v = torch.exp((x - top).masked_fill(off, -1e30))
    total = v.sum(1, keepdim=True)
    return v / total.masked_fill(total == 0, 1.0)


def _exact_losses(c, s, x, count):
    """Mean scores [S, E] and losses [S]."""
    S, E = c["T"] // c["seq"], c["E"]
    live = s["live"]
    n = torch.full((S, 1), float(c["seq"]), dtype=torch.float64, device=x.device) if live is None \
        else live.view(S, -1).double().sum(1, keepdim=True)
    mean = _exact_shares(c, x, live).view(S, -1, E).sum(1) / n.clamp(min=1.0)
    load = count.double() / count.double().sum(1, keepdim=True).clamp(min=1.0) * E
    return mean, (mean * load).sum(1)


def _exact_values(q, scales, K):
    low, high = (q & 15).long(), (q >> 4).long()
    code = torch.stack([low, high], -1).flatten(-2)
    v = torch.tensor(MAGNITUDES, dtype=torch.float64, device=q.device)[code & 7]
    v = torch.where(code > 7, -v, v)
    n = scales[..., :K // BLOCK].int() - 127
    return v * torch.ldexp(torch.ones(n.shape, dtype=torch.float64, device=q.device),
                           n).repeat_interleave(BLOCK, -1)


def _exact_rounded(x):
    """Values of bf16-like rows x (in 64 bits) after their quantisation, by the nearest
    magnitude."""
    b = x.view(x.shape[0], -1, BLOCK)
    a = b.abs().amax(2, keepdim=True)
    unit = torch.exp2(torch.ceil(torch.log2(a.clamp(min=2.0 ** -120) / 7)).clamp(min=-127))
    unit = torch.where(a >= 7 * unit, 2 * unit, unit)     # 7 itself goes to the next
    m = (b / unit).abs().unsqueeze(-1)
    grid = torch.tensor(MAGNITUDES, dtype=torch.float64, device=x.device)
    # of two equally near the one of even place
    far = (m - grid).abs() + torch.tensor([0, 1e-9] * 4, dtype=torch.float64, device=x.device)
    return (grid[far.argmin(-1)] * unit).view_as(x) * torch.where(x < 0, -1.0, 1.0)


def _exact_layer(c, s):
    h = s["x"].double() + s["residual"].double()
    y = torch.zeros_like(h)
    x = h * torch.rsqrt(h.pow(2).mean(1, keepdim=True) + EPS) * s["weight"].double()
    x = x.bfloat16().double()
    x = torch.cat([_exact_rounded(x[i:i + 256]) for i in range(0, c["T"], 256)])
    z = s["logits"].double()
    if s["live"] is not None:
        z = z.masked_fill(s["live"][:, None] == 0, -math.inf)
    v, idx = torch.sort(z, dim=1, descending=True, stable=True)
    v, idx = v[:, :c["k"]], idx[:, :c["k"]]
    w = torch.nan_to_num(torch.softmax(v, 1), nan=0.0)
    idx = idx.masked_fill(v == -math.inf, -1)
    for e in range(c["E"]):
        tok, slot = torch.nonzero(idx == e, as_tuple=True)
        if not len(tok):
            continue
        g, u = (x[tok] @ _exact_values(s["w13"][e], s["s13"][e], c["H"]).T).chunk(2, 1)
        act = (g * torch.sigmoid(g) * u).bfloat16().double()
        act = torch.cat([_exact_rounded(act[i:i + 1024]) for i in range(0, len(tok), 1024)])
        rows = act @ _exact_values(s["w2"][e], s["s2"][e], c["I"]).T
        y.index_add_(0, tok, rows * w[tok, slot][:, None])
    return {"sum": h, "idx": None, "w": w, "y": y}


def exact(case, seed):
    c, kind = case, case["kind"]
    s = prepare(case, seed)
    if kind == "balance":
        E, S = c["E"], c["T"] // c["seq"]
        live = torch.ones(c["T"], device="cuda") if s["live"] is None else s["live"]
        idx = s["idx"].long().masked_fill(live[:, None] == 0, -1).view(S, -1)
        count = torch.zeros(S, E + 1, dtype=torch.float64, device="cuda")
        count.scatter_add_(1, torch.where(idx < 0, E, idx), torch.ones_like(idx, dtype=torch.float64))
        mean, loss = _exact_losses(c, s, s["logits"].double(), count[:, :E])
        return {"count": None, "tokens": None, "mean": mean, "loss": loss}
    if kind == "balance_grad":              # by automatic differentiation
        x = s["logits"].double().requires_grad_()
        _, loss = _exact_losses(c, s, x, s["count"])
        (d,) = torch.autograd.grad((loss * s["grad_loss"].double()).sum(), x)
        d = d.masked_fill(x.detach() == -math.inf, 0.0)
        return {"grad": d if s["sum"] is None else d + s["sum"].double()}
    if kind == "quantize":
        x = s["x"].double()
        v = torch.cat([_exact_rounded(x[i:i + 256]) for i in range(0, c["rows"], 256)])
        if s["src"] is not None:
            v = v.masked_fill(s["src"][:, None] < 0, 0.0)
        return {"q": None, "scales": None, "values": v}
    if kind == "matmul":
        y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
        for e, (o, n) in enumerate(zip(s["offset"].tolist(), s["count"].tolist())):
            if not n:
                continue
            v = _exact_values(s["a"][o:o + n], s["a_scales"][o:o + n], c["K"]) \
                @ _exact_values(s["wt"][e], s["wt_scales"][e], c["K"]).T
            if c["swiglu"]:
                g, u = v.chunk(2, -1)
                v = g * torch.sigmoid(g) * u
            y[o:o + n] = v
        return {"y": y}
    return _exact_layer(c, s)
