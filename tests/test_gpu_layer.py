"""The MoE layer as a whole: against its definition in 64 bits, on a stream of its
own, and replayed from a graph."""
import math

import pytest

torch = pytest.importorskip("torch")

import layer_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _inputs(T, H, E, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    x, r = (torch.randn(T, H, generator=g).bfloat16() for _ in range(2))
    return x.cuda(), r.cuda(), torch.randn(T, E, generator=g).cuda()


def _int8(v):
    s = ref.amax_scales(v, False)
    return torch.round(v / s) * s


def _want(layer, x, r, logits):
    """The layer in 64 bits with the experts that it chose."""
    c = [t.cpu().double() for t in (x, r, layer.norm_weight, logits)]
    h, _, y = ref.rmsnorm(c[0], c[1], c[2], layer.eps)
    idx = layer.topk_idx.cpu()
    w = ref.weights(c[3], idx, layer.options["score"] == 1, layer.options["renorm"],
                    layer.options["scale"])
    a, out = _int8(y), torch.zeros_like(y)
    size = torch.zeros_like(y)
    for e in range(layer.E):
        tok, slot = torch.nonzero(idx == e, as_tuple=True)
        if not len(tok):
            continue
        v = a[tok] @ layer.w13[e].cpu().double().T * layer.w13_scale[e].cpu().double()
        g, u = v[:, :layer.I], v[:, layer.I:]
        act = _int8(g * torch.sigmoid(g) * u)
        row = act @ layer.w2[e].cpu().double().T * layer.w2_scale[e].cpu().double()
        out.index_add_(0, tok, row * w[tok, slot][:, None])
        size.index_add_(0, tok, (row * w[tok, slot][:, None]).abs())
    return h, out, size


@pytest.mark.parametrize("T,H,I,E,k", [(1, 256, 64, 4, 2), (33, 384, 208, 8, 3), (300, 512, 256, 16, 4),
                                       (700, 1024, 144, 4, 2)])
@pytest.mark.parametrize("score", [0, 1])
def test_layer(T, H, I, E, k, score):
    """A bf16 rounding (2^-8) before the second quantisation moves a code by
    one step (1/254 of the row's largest value) here and there, the experts' rows
    and the result are rounded to bf16: over a token's row the difference stays
    under 3% of its norm."""
    from paper_2607_26444_amd.layer import random_layer
    layer = random_layer(T, H, I, E, k, seed=T, score=score, scale=1.5)
    x, r, logits = _inputs(T, H, E, seed=1)
    y = layer.forward(x, r, logits)
    torch.cuda.synchronize()
    h, want, size = _want(layer, x, r, logits)
    assert torch.all((layer.sum.cpu().double() - h).abs() <= 2.0 ** -8 * 1.001 * h.abs())
    off = (y.cpu().double() - want).norm(dim=1)
    assert torch.all(off <= 0.03 * want.norm(dim=1)), float((off / want.norm(dim=1)).max())
    assert int(layer.layout.status) == 0


def test_padding_tokens_and_masked_experts():
    from paper_2607_26444_amd.layer import random_layer
    layer = random_layer(64, 256, 64, 8, 4, bias=torch.zeros(8, device="cuda"), score=1)
    x, r, logits = _inputs(64, 256, 8, seed=2)
    logits[5] = -math.inf
    logits[6, 2:] = -math.inf
    mask = torch.ones(64, dtype=torch.uint8, device="cuda")
    mask[60:] = 0
    y = layer.forward(x, r, logits, token_mask=mask)
    torch.cuda.synchronize()
    assert torch.all(layer.topk_idx[60:] == -1) and torch.all(layer.topk_idx[5] == -1)
    assert torch.all(y[60:] == 0) and torch.all(y[5] == 0) and torch.all(layer.topk_idx[6, 2:] == -1)
    _, want, _ = _want(layer, x, r, logits.masked_fill(mask[:, None] == 0, -math.inf))
    off = (y.cpu().double() - want).norm(dim=1)
    assert torch.all(off <= 0.03 * want.norm(dim=1) + 1e-12)


def test_gate_as_a_function():
    from paper_2607_26444_amd.layer import random_layer
    layer = random_layer(40, 256, 64, 8, 2)
    x, r, _ = _inputs(40, 256, 8, seed=3)
    gate = torch.randn(256, 8, device="cuda").bfloat16() / 16
    seen = []

    def logits(normed):
        seen.append(normed @ gate)
        return seen[-1]
    y = layer.forward(x, r, logits)
    again = layer.forward(x, r, seen[0]).clone()
    assert torch.equal(y, again)


def test_graph_replays():
    """Captured once, replayed with new inputs, eager work in between: every
    replay equals the eager result."""
    from paper_2607_26444_amd.layer import random_layer
    T, H, E = 48, 512, 8
    layer = random_layer(T, H, 128, E, 2)
    eager = random_layer(T, H, 128, E, 2)
    x, r, logits = (t.clone() for t in _inputs(T, H, E, seed=0))
    layer.forward(x, r, logits)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(x, r, logits)
    for seed in range(1, 5):
        for t, new in zip((x, r, logits), _inputs(T, H, E, seed)):
            t.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        want = eager.forward(x, r, logits)
        torch.cuda.synchronize()
        assert torch.equal(layer.y, want) and torch.equal(layer.sum, eager.sum)


def test_stream_of_its_own():
    from paper_2607_26444_amd.layer import random_layer
    layer = random_layer(100, 256, 64, 8, 2)
    x, r, logits = _inputs(100, 256, 8, seed=4)
    want = layer.forward(x, r, logits).clone()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    y = layer.forward(x, r, logits, stream=s)
    s.synchronize()
    assert torch.equal(y, want)


def test_refused_arguments():
    from paper_2607_26444_amd import layer as mod
    from paper_2607_26444_amd.layer import random_layer
    with pytest.raises(ValueError, match="multiple"):
        random_layer(8, 200, 64, 4, 2)
    layer = random_layer(8, 256, 64, 4, 2)
    x, r, logits = _inputs(8, 256, 4, seed=5)
    for bad in ((x.float(), r, logits), (x[:4], r, logits), (x, r.float(), logits),
                (x, r, logits[:, :3]), (x, r, logits.half())):
        with pytest.raises(ValueError):
            layer.forward(*bad)
    with pytest.raises(ValueError):
        layer.forward(x, r, logits, token_mask=torch.ones(8, device="cuda"))
    with pytest.raises(ValueError):
        mod.MoeLayer(8, 256, 64, 4, 2, layer.norm_weight, layer.w13, layer.w13_scale,
                     layer.w2[:2], layer.w2_scale)


def test_gate_as_a_function_on_a_stream_of_its_own():
    """Behind work that takes milliseconds: a gate that ran beside the stream would read
    the rows of the batch before, and its logits' memory would be given to the tensors
    that the current stream fills meanwhile."""
    from paper_2607_26444_amd.layer import random_layer
    T, H, E = 200, 512, 8
    layer = random_layer(T, H, 128, E, 2)
    gate = torch.randn(H, E, device="cuda").bfloat16() / 16
    x, r, _ = _inputs(T, H, E, seed=6)
    want = layer.forward(x, r, lambda normed: normed @ gate).clone()
    chosen = layer.topk_idx.clone()
    layer.forward(*_inputs(T, H, E, seed=7)[:2], lambda normed: normed @ gate)
    layer.topk_idx.fill_(-1)
    slow = torch.randn(8192, 8192, device="cuda").bfloat16()
    s = torch.cuda.Stream()
    out = torch.empty_like(slow)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(10):
            torch.mm(slow, slow, out=out)
    y = layer.forward(x, r, lambda normed: normed @ gate, stream=s)
    assert torch.cuda.current_stream() != s
    junk = [torch.full((T, E), 50.0 + n, dtype=torch.bfloat16, device="cuda") for n in range(64)]
    s.synchronize()
    assert torch.equal(layer.topk_idx, chosen) and torch.equal(y, want)
    assert len(junk) == 64


def test_logits_strides():
    """Rows with a pitch, a transposed single row, a transposed single column."""
    from paper_2607_26444_amd.layer import random_layer
    for T, E, k in ((1, 8, 2), (50, 8, 2), (50, 1, 1)):
        layer = random_layer(T, 256, 64, E, k, seed=T)
        x, r, logits = _inputs(T, 256, E, seed=8)
        want = layer.forward(x, r, logits).clone()
        wide = torch.full((T, E + 5), 9.0, device="cuda")
        wide[:, 2:2 + E] = logits
        views = [wide[:, 2:2 + E]] + ([logits.t().contiguous().t()] if T == 1 or E == 1 else [])
        for view in views:
            assert torch.equal(layer.forward(x, r, view), want), (T, E, view.stride())
    with pytest.raises(ValueError, match="logits"):
        layer.forward(x, r, torch.zeros(1, device="cuda").expand(50, 1))


def test_token_mask_strides():
    from paper_2607_26444_amd.layer import random_layer
    layer = random_layer(20, 256, 64, 8, 2)
    x, r, logits = _inputs(20, 256, 8, seed=9)
    table = (torch.arange(60, device="cuda").view(20, 3) % 4 != 0).to(torch.uint8)
    for bad in (table[:, 1], table[0, :1].expand(20)):
        with pytest.raises(ValueError, match="token_mask"):
            layer.forward(x, r, logits, token_mask=bad)
    layer.forward(x, r, logits, token_mask=table[:, 1].contiguous())
    assert torch.equal((layer.topk_idx[:, 0] >= 0).to(torch.uint8), table[:, 1])


def test_no_tokens():
    from paper_2607_26444_amd.layer import random_layer
    layer = random_layer(0, 256, 64, 8, 2)
    x, r, logits = _inputs(0, 256, 8, seed=0)
    for given in (logits, lambda normed: normed.float() @ torch.ones(256, 8, device="cuda")):
        assert layer.forward(x, r, given).shape == (0, 256)
    torch.cuda.synchronize()
    assert int(layer.layout.status) == 0 and torch.all(layer.layout.expert_count == 0)


def test_gate_on_a_stream_of_another_library():
    """A stream that is known by its address alone."""
    from paper_2607_26444_amd.layer import random_layer
    T, H, E = 64, 256, 8
    layer = random_layer(T, H, 64, E, 2)
    gate = torch.randn(H, E, device="cuda").bfloat16() / 16
    x, r, _ = _inputs(T, H, E, seed=10)
    want = layer.forward(x, r, lambda normed: normed @ gate).clone()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()

    class Foreign:
        cuda_stream = s.cuda_stream
    seen = []

    def logits(normed):
        seen.append(torch.cuda.current_stream().cuda_stream)
        return normed @ gate
    y = layer.forward(x, r, logits, stream=Foreign())
    s.synchronize()
    assert seen == [s.cuda_stream] and torch.equal(y, want)
