"""Routing and its gradient against their definitions in 64 bits.

Choice: where the key is the logit the order is exact, ties by the index.  Where
it is a score (+ bias) in float32, keys nearer than KEY_TOL may swap: a score is
off by at most 2^-22 of itself (exp, a sum over a tree of at most ten levels,
a division: fewer than 16 roundings of 2^-24 ... of values up to 1), a sum of
two keys by twice that.
Weights: exp of a rounded difference d is off by (|d| + 2) 2^-24 of itself, a sum
of up to 32 and a division add 34 roundings; |d| <= 24 here: 2^-18.
"""
import math

import pytest

torch = pytest.importorskip("torch")

import layer_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu

KEY_TOL = 2.0 ** -20
W_TOL = 2.0 ** -18


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _moe():
    from paper_2607_26444_amd import moe
    return moe


def _draw(T, E, f32, seed, spread=2.0):
    g = torch.Generator()
    g.manual_seed(seed)
    x = torch.randn(T, E, generator=g) * spread
    return x if f32 else x.bfloat16()


def _route(x, k, bias=None, mask=None, pitch=0, **opt):
    moe = _moe()
    T, E = x.shape
    idx = torch.full((T, k), -9, dtype=torch.int32, device="cuda")
    w = torch.full((T, k), -9.0, device="cuda")
    xd = x if x.is_cuda else x.cuda()
    moe.moe_route(xd, moe.MOE_DTYPE_F32 if x.dtype == torch.float32 else moe.MOE_DTYPE_BF16, E,
                  None if bias is None else bias.cuda(), None if mask is None else mask.cuda(),
                  idx, w, logits_pitch=pitch, **opt)
    torch.cuda.synchronize()
    return idx.cpu(), w.cpu()


def _check(x, idx, w, k, bias=None, mask=None, score=0, groups=1, top_groups=1, group_top=1,
           renorm=True, scale=1.0):
    xd = x.double()
    if mask is not None:
        xd = xd.masked_fill(mask[:, None] == 0, -math.inf)
    key = ref.keys(xd, score == 1, bias, groups, group_top)
    by_score = bias is not None or (groups > 1 and group_top > 1)
    tol = KEY_TOL * (1 + (0 if bias is None else float(bias.abs().max()))) if by_score else 0.0
    size = x.shape[1] // groups
    for t in range(x.shape[0]):
        row = key[t].tolist()
        got = idx[t].tolist()
        allowed = range(len(row))
        if groups > 1:
            keep, margin = ref.kept_groups(row, groups, top_groups, group_top)
            if margin <= 4 * tol and by_score:
                continue                       # either group may be taken
            allowed = [e for g in keep for e in range(g * size, (g + 1) * size)]
        live = sorted((e for e in allowed if row[e] > -math.inf), key=lambda e: (-row[e], e))
        n = min(k, len(live))
        assert got[n:] == [-1] * (k - n), (t, got)
        if by_score:
            assert len(set(got[:n])) == n and set(got[:n]) <= set(live), (t, got)
            for j in range(n):                 # j-th key within tol of the j-th best
                assert abs(row[got[j]] - row[live[j]]) <= tol, (t, j, got, live[:n])
        else:
            assert got[:n] == live[:n], (t, got, live[:n])
    want = ref.weights(xd, idx, score == 1, renorm, scale)
    assert torch.all((w.double() - want).abs() <= W_TOL * want.abs() + 1e-37)
    assert torch.all(w[idx < 0] == 0)


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 2, 1), (3, 8, 8), (128, 16, 2), (65, 17, 5),
                                   (50, 33, 16), (70, 60, 6), (40, 96, 17), (130, 128, 8),
                                   (33, 160, 4), (64, 256, 8), (17, 256, 32), (20, 384, 8),
                                   (9, 1000, 10), (5, 1024, 32)])
@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("score,bias,renorm", [(0, False, True), (0, False, False),
                                               (0, True, False), (1, False, True), (1, True, True),
                                               (1, False, False)])
def test_route(T, E, k, f32, score, bias, renorm):
    x = _draw(T, E, f32, seed=T * 1000 + E)
    b = _draw(1, E, True, seed=E + 1, spread=0.05)[0] if bias else None
    opt = dict(score=score, renorm=renorm, scale=2.5 if bias else 1.0)
    idx, w = _route(x, k, bias=b, **opt)
    _check(x, idx, w, k, bias=b, **opt)


@pytest.mark.parametrize("T,E,k,groups,top", [(33, 256, 8, 8, 4), (20, 64, 4, 4, 1), (21, 60, 6, 4, 2),
                                              (19, 12, 2, 12, 5), (9, 512, 10, 64, 7),
                                              (40, 160, 6, 8, 3), (11, 96, 3, 32, 32)])
@pytest.mark.parametrize("score,bias,two", [(0, False, 1), (1, True, 2), (0, True, 2),
                                            (1, False, 2), (1, True, 1)])
def test_route_groups(T, E, k, groups, top, score, bias, two):
    x = _draw(T, E, True, seed=E + groups)
    b = _draw(1, E, True, seed=3, spread=0.1)[0] if bias else None
    opt = dict(score=score, groups=groups, top_groups=top, group_top=two)
    idx, w = _route(x, k, bias=b, **opt)
    _check(x, idx, w, k, bias=b, **opt)


@pytest.mark.parametrize("T,E,k,groups,top", [(13, 512, 8, 4, 2), (10, 384, 8, 8, 4), (9, 1000, 20, 8, 3),
                                              (7, 1024, 8, 32, 8), (8, 300, 6, 3, 2), (6, 340, 4, 17, 5),
                                              (5, 20, 20, 2, 2), (9, 264, 5, 24, 4)])
@pytest.mark.parametrize("score,bias,two", [(0, False, 1), (1, True, 2), (0, True, 2)])
def test_groups_of_a_whole_wavefront(T, E, k, groups, top, score, bias, two):
    """More than 256 experts or 16 slots: several lanes look over a group; some groups
    and experts masked."""
    x = _draw(T, E, True, seed=E + groups)
    x[0, : E // groups] = -math.inf
    x[1, ::3] = -math.inf
    x[2] = -math.inf
    x[2, E - 1] = 0.5
    b = _draw(1, E, True, seed=3, spread=0.1)[0] if bias else None
    opt = dict(score=score, groups=groups, top_groups=top, group_top=two)
    idx, w = _route(x, k, bias=b, **opt)
    _check(x, idx, w, k, bias=b, **opt)
    assert idx[2].tolist() == [E - 1] + [-1] * (k - 1)


@pytest.mark.parametrize("E,k", [(16, 4), (100, 8), (256, 8), (700, 20)])
@pytest.mark.parametrize("score,renorm", [(0, True), (0, False), (1, True), (1, False)])
@pytest.mark.parametrize("groups", [1, 4])
def test_masked_experts_and_rows_left_empty(E, k, score, renorm, groups):
    """-inf, NaN and the type's lowest value in masked places; rows with fewer
    eligible experts than slots, and with none."""
    x = _draw(24, E, True, seed=E)
    g = torch.Generator()
    g.manual_seed(1)
    x[torch.rand(24, E, generator=g) < 0.5] = -math.inf
    x[3] = -math.inf
    x[4] = math.nan
    x[5, 1:] = -math.inf                       # one expert left
    x[6] = torch.finfo(torch.float32).min      # all equal and eligible
    x[7, 2:] = torch.finfo(torch.float32).min
    x[8, : E // 2] = math.nan
    opt = dict(score=score, renorm=renorm, groups=groups, top_groups=2 if groups > 1 else 1)
    k = min(k, 2 * (E // groups) if groups > 1 else E)
    idx, w = _route(x, k, **opt)
    _check(x, idx, w, k, **opt)
    assert torch.all(idx[3] == -1) and torch.all(idx[4] == -1) and torch.all(w[3:5] == 0)
    b = _draw(1, E, True, seed=2, spread=0.1)[0]
    b[0] = -math.inf                           # a bias that rules an expert out
    idx, w = _route(x, k, bias=b, **opt)
    _check(x, idx, w, k, bias=b, **opt)
    assert not torch.any(idx == 0)


@pytest.mark.parametrize("score", [0, 1])
def test_infinite_logit_wins(score):
    x = _draw(6, 40, True, seed=4)
    x[:, 7] = math.inf
    x[2, 30] = math.inf
    for renorm in (True, False):
        idx, w = _route(x, 3, score=score, renorm=renorm)
        _check(x, idx, w, 3, score=score, renorm=renorm)
        assert torch.all(idx[:, 0] == 7) and idx[2, 1] == 30 and torch.all(torch.isfinite(w))


def test_equal_keys_take_the_lowest_index():
    x = torch.zeros(5, 256)
    x[1, ::2] = -0.0                            # the sign of zero does not order
    x[2, 200:] = 1.0
    idx, w = _route(x, 8)
    assert idx[0].tolist() == list(range(8)) == idx[1].tolist()
    assert idx[2].tolist() == list(range(200, 208))
    assert torch.all(w == 0.125)


@pytest.mark.parametrize("E,groups,top", [(256, 8, 4), (128, 4, 2), (256, 16, 3), (64, 2, 1), (60, 6, 2),
                                          (160, 8, 3)])
@pytest.mark.parametrize("two", [1, 2])
def test_equal_groups_take_the_lowest_index(E, groups, top, two):
    x = torch.zeros(6, E)
    x[1, E // groups:] = 1.0                    # all groups but the first
    x[2, E - 1] = 1.0                           # the last one stands out
    x[3, : E // groups] = -math.inf
    opt = dict(groups=groups, top_groups=top, group_top=two, score=1)
    idx, w = _route(x, 6, **opt)
    _check(x, idx, w, 6, **opt)
    size = E // groups
    assert idx[0].tolist() == list(range(6))
    assert idx[1].tolist() == list(range(size, size + 6))
    assert idx[2, 0] == E - 1 and (top == 1 or idx[2, 1] == 0)
    assert idx[3].tolist() == list(range(size, size + 6))


def test_token_mask_pitch_and_offset_bases():
    wide = _draw(40, 300, True, seed=9).cuda()
    mask = (torch.arange(40) % 3 != 0).to(torch.uint8)
    for start, E in ((0, 256), (1, 256), (4, 128), (3, 17)):
        x = wide[:, start:start + E]
        idx, w = _route(x, 4, mask=mask, pitch=300)
        _check(x.cpu(), idx, w, 4, mask=mask)
        h = wide.bfloat16()[:, start:start + E]
        idx, w = _route(h, 4, pitch=300)
        _check(h.cpu(), idx, w, 4)


def test_no_tokens():
    idx, w = _route(torch.empty(0, 16), 2)
    assert idx.shape == (0, 2)


def test_replicas_agree_to_the_bit():
    """A softmax key's sum is the same whatever the launch: the same tokens in
    another batch size, and next to others, give the same bits."""
    x = _draw(300, 256, True, seed=11)
    b = _draw(1, 256, True, seed=12, spread=0.01)[0]
    whole = _route(x, 8, bias=b, renorm=False)
    part = _route(x[100:107], 8, bias=b, renorm=False)
    assert torch.equal(whole[0][100:107], part[0]) and torch.equal(whole[1][100:107], part[1])
    wide = torch.full((300, 600), -math.inf)    # other widths of launch, the same experts
    wide[:, :256] = x
    b2 = torch.zeros(600)
    b2[:256] = b
    other = _route(wide, 8, bias=b2, renorm=False)
    assert torch.equal(whole[0], other[0]) and torch.equal(whole[1], other[1])


def test_routing_drives_the_exchange():
    """Rows of the layout follow what moe_route wrote, unused slots included."""
    moe = _moe()
    x = _draw(500, 64, True, seed=13)
    x[::5] = -math.inf
    x[1::5, 3:] = -math.inf
    idx, _ = _route(x, 6)
    lay = moe.Layout(500, 6, 64, 4)
    lay.run(idx.cuda())
    torch.cuda.synchronize()
    assert int(lay.status) == 0
    assert torch.equal(lay.expert_count.cpu(),
                       torch.bincount(idx[idx >= 0].long(), minlength=64).int())


# ------------------------------------------------------------------ gradient
def _grad(x, idx, gw, score, renorm, scale):
    moe = _moe()
    T, E = x.shape
    out = torch.full_like(x, 7.0).cuda()
    moe.moe_route_backward(x.cuda(), moe.MOE_DTYPE_F32 if x.dtype == torch.float32
                           else moe.MOE_DTYPE_BF16, E, idx.cuda(), gw.cuda(), out, score=score,
                           renorm=renorm, scale=scale)
    torch.cuda.synchronize()
    return out.cpu()


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (3, 8, 3), (130, 16, 2), (50, 33, 16), (70, 60, 6),
                                   (40, 96, 17), (130, 128, 8), (64, 256, 8), (20, 512, 10),
                                   (5, 1024, 32)])
@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("score,renorm", [(0, True), (0, False), (1, True), (1, False)])
def test_route_gradient(T, E, k, f32, score, renorm):
    """Against automatic differentiation in 64 bits.  A value is a difference of
    terms bounded by scale * max|g|; each has a relative error of at most
    2^-18 (see the weights), a bf16 result half a step more."""
    x = _draw(T, E, f32, seed=T + E)
    if T > 4:
        x[1] = -math.inf
        x[2, : E // 2] = -math.inf
    idx, _ = _route(x, k, score=score, renorm=renorm)
    g = torch.Generator()
    g.manual_seed(5)
    gw = torch.randn(T, k, generator=g)
    got = _grad(x, idx, gw, score, renorm, 2.5).double()
    want = ref.route_grad(x.double(), idx, gw.double(), score == 1, renorm, 2.5)
    bound = W_TOL * 2.5 * gw.abs().amax(1, keepdim=True).double() * (1 + k ** 0.5)
    if not f32:
        bound = bound + 2.0 ** -8 * want.abs()
    assert torch.all((got - want).abs() <= bound)
    if T > 4:
        assert torch.all(got[1] == 0)


@pytest.mark.parametrize("score,renorm", [(0, True), (0, False), (1, True), (1, False)])
def test_route_gradient_against_differences(score, renorm):
    """Central differences of moe_route's own weights, the choice unchanged:
    third derivatives of at most 2 times (1/64)^2 / 6, and weights rounded at
    2^-18 over 1/32: 2e-4 in all for |g| of about 1."""
    T, E, k, step = 6, 24, 4, 1.0 / 64
    x = _draw(T, E, True, seed=21)
    for t in range(T):                          # winners stand clear of the others
        x[t, torch.randperm(E, generator=torch.Generator().manual_seed(t))[:k]] += 8.0
        x[t] += 0.1 * torch.arange(E) % 0.7
    idx, _ = _route(x, k, score=score, renorm=renorm)
    gw = torch.randn(T, k, generator=torch.Generator().manual_seed(6))
    got = _grad(x, idx, gw, score, renorm, 1.0)

    def loss(v):
        i, w = _route(v, k, score=score, renorm=renorm)
        dense = torch.zeros(T, E, dtype=torch.float64).scatter_(1, i.long(), w.double())
        return (dense.gather(1, idx.long()) * gw.double()).sum(1)
    for e in range(E):
        up, down = x.clone(), x.clone()
        up[:, e] += step
        down[:, e] -= step
        diff = (loss(up) - loss(down)) / (2 * step)
        assert torch.all((got[:, e].double() - diff).abs() <= 1e-3), e


def test_gradient_of_unused_and_foreign_slots():
    x = _draw(8, 32, True, seed=1)
    idx = torch.full((8, 3), -1, dtype=torch.int32)
    idx[2] = torch.tensor([5, -1, 40])          # 40 is no expert
    idx[3] = torch.tensor([0, 1, 2])
    gw = torch.ones(8, 3)
    for score, renorm in ((0, True), (0, False), (1, True), (1, False)):
        got = _grad(x, idx, gw, score, renorm, 1.0).double()
        clean = torch.where(idx >= 32, torch.full_like(idx, -1), idx)
        want = ref.route_grad(x.double(), clean, torch.where(clean < 0, 0.0, gw).double(),
                              score == 1, renorm, 1.0)
        assert torch.all((got - want).abs() <= 8 * W_TOL)
        assert torch.all(got[0] == 0)


@pytest.mark.parametrize("E,groups", [(16, 4), (64, 8), (60, 6), (256, 16), (160, 8), (512, 8), (300, 3)])
@pytest.mark.parametrize("score", [0, 1])
def test_group_of_experts_at_the_lowest_value(E, groups, score):
    """A bias of the type's lowest value leaves an expert eligible, and so its group,
    though the sum of two such keys is below every float32: it comes behind all
    others, before groups that have no eligible expert.  The keys are equal there (a
    score is far below the bias's last bit), so the index decides."""
    size, lowest = E // groups, torch.finfo(torch.float32).min
    x = _draw(9, E, True, seed=E)
    b = torch.full((E,), lowest)
    b[:size] = -math.inf                       # the first group is ruled out
    opt = dict(score=score, groups=groups, group_top=2)
    idx, w = _route(x, 2, bias=b, top_groups=1, **opt)
    assert torch.equal(idx, torch.tensor([[size, size + 1]] * 9, dtype=torch.int32))
    _check(x, idx, w, 2, bias=b, top_groups=1, **opt)
    b[-size:] = 0.0                            # the last one stands above
    idx, w = _route(x, 3, bias=b, top_groups=2, **opt)
    live = idx >= E - size
    assert torch.all(live[:, :min(3, size)])
    b[-size + 1:] = lowest                     # ... by one expert
    idx, w = _route(x, 3, bias=b, top_groups=1, **opt)
    assert torch.all(idx[:, 0] == E - size) and torch.all(idx[:, 1] == E - size + 1)
    b[:] = -math.inf
    idx, w = _route(x, 3, bias=b, top_groups=2, **opt)
    assert torch.all(idx == -1) and torch.all(w == 0)


@pytest.mark.parametrize("renorm", [False, True])
def test_sigmoid_gradient_of_large_logits(renorm):
    """1 - s is sigmoid(-x), small beside s where x is large: the gradient keeps its
    relative accuracy (W_TOL of its terms) there, also where s rounds to 1."""
    T, E, k = 40, 48, 6
    x = _draw(T, E, True, seed=31) + torch.linspace(-20, 60, T)[:, None]
    idx, _ = _route(x, k, score=1, renorm=renorm)
    gw = torch.randn(T, k, generator=torch.Generator().manual_seed(8))
    got = _grad(x, idx, gw, 1, renorm, 1.5).double().gather(1, idx.long())
    xw, g = x.double().gather(1, idx.long()), gw.double()
    s, rest = torch.sigmoid(xw), torch.sigmoid(-xw)
    q = s / s.sum(1, keepdim=True) if renorm else s
    dot = (g * q).sum(1, keepdim=True) if renorm else torch.zeros(T, 1).double()
    size = (g * q).abs().sum(1, keepdim=True) if renorm else dot
    want = 1.5 * q * rest * (g - dot)
    assert torch.all((got - want).abs() <= W_TOL * 1.5 * q * rest * (g.abs() + size))
    assert torch.all(want[T // 2:].abs() < 1e-4)      # the rows of large logits are there


@pytest.mark.parametrize("start,E", [(0, 256), (1, 256), (4, 128), (3, 17), (2, 60), (5, 300)])
@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("score,renorm", [(0, True), (0, False), (1, True), (1, False)])
def test_route_gradient_of_pitches_and_offset_bases(start, E, f32, score, renorm):
    """Rows of a wider table, from a base that vectors would not be aligned at; the
    gradient's base likewise.  The bits are those of packed rows."""
    moe = _moe()
    T, k, pitch = 37, 4, 307
    wide = _draw(T, pitch, f32, seed=17)
    x = wide[:, start:start + E]
    idx, _ = _route(x.contiguous(), k, score=score, renorm=renorm)
    gw = torch.randn(T, k, generator=torch.Generator().manual_seed(9))
    want = _grad(x.contiguous(), idx, gw, score, renorm, 2.0)
    out = torch.full((T * E + 9,), 7.0, dtype=x.dtype, device="cuda")
    view = out[start:start + T * E].view(T, E)
    moe.moe_route_backward(wide.cuda()[:, start:start + E], moe.MOE_DTYPE_F32 if f32
                           else moe.MOE_DTYPE_BF16, E, idx.cuda(), gw.cuda(), view, score=score,
                           renorm=renorm, scale=2.0, logits_pitch=pitch)
    torch.cuda.synchronize()
    assert torch.equal(view.cpu(), want)
    assert torch.all(out[:start] == 7) and torch.all(out[start + T * E:] == 7)
    exact = ref.route_grad(x.double(), idx, gw.double(), score == 1, renorm, 2.0)
    bound = W_TOL * 2.0 * gw.abs().amax(1, keepdim=True).double() * (1 + k ** 0.5)
    bound = bound + (0 if f32 else 2.0 ** -8 * exact.abs())
    assert torch.all((want.double() - exact).abs() <= bound)


@pytest.mark.parametrize("E,k,opt", [(8, 2, {}), (16, 4, dict(groups=4, top_groups=2, group_top=2)),
                                     (4, 1, dict(renorm=False)), (72, 4, {})])
@pytest.mark.parametrize("score", [0, 1])
def test_more_tokens_than_one_grid(E, k, opt, score):
    """Workgroups go round again from 2^24 tokens on: the last ones route, and have gradients,
    as in a call of their own (with 72 experts past 2^32 bytes)."""
    moe = _moe()
    T, tail = (1 << 24) + 1237, 5000
    g = torch.Generator(device="cuda")
    g.manual_seed(E)
    x = torch.randn(T, E, generator=g, device="cuda", dtype=torch.float32)
    idx = torch.full((T, k), -9, dtype=torch.int32, device="cuda")
    w = torch.full((T, k), -9.0, device="cuda")
    moe.moe_route(x, moe.MOE_DTYPE_F32, E, None, None, idx, w, score=score, **opt)
    part_idx, part_w = torch.empty_like(idx[-tail:]), torch.empty_like(w[-tail:])
    moe.moe_route(x[-tail:], moe.MOE_DTYPE_F32, E, None, None, part_idx, part_w, score=score, **opt)
    assert torch.equal(idx[-tail:], part_idx) and torch.equal(w[-tail:], part_w)
    assert bool(((idx >= 0) & (idx < E)).all()) and bool((w > 0).all())
    _check(x[-50:].cpu(), idx[-50:].cpu(), w[-50:].cpu(), k, score=score, **opt)
    gw = torch.randn(T, k, generator=g, device="cuda")
    grad, part = torch.full_like(x, 7.0), torch.empty_like(x[-tail:])
    back = dict(score=score, renorm=opt.get("renorm", True))
    moe.moe_route_backward(x, moe.MOE_DTYPE_F32, E, idx, gw, grad, **back)
    moe.moe_route_backward(x[-tail:], moe.MOE_DTYPE_F32, E, part_idx, gw[-tail:], part, **back)
    assert torch.equal(grad[-tail:], part) and not bool((grad == 7.0).any())
