"""RMS norm with 8-bit output, row quantisation and the norm's gradients against
their definitions in 64 bits.

A float32 value of the row is off by a few roundings (the sum of H squares is a
tree of at most 16 serial terms and 12 levels, its error halves in the root):
2^-20 of itself.  bf16 adds half a step (2^-8 of the value at most), E4M3 half a
step (2^-4, or 2^-10 scales below the normal range), int8 half a scale.
"""
import math

import pytest

torch = pytest.importorskip("torch")

import layer_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu

F32 = 2.0 ** -20
BF16 = 2.0 ** -8 * 1.001


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _moe():
    from paper_2607_26444_amd import moe
    return moe


def _dt(t):
    moe = _moe()
    return moe.MOE_DTYPE_F32 if t is not None and t.dtype == torch.float32 else moe.MOE_DTYPE_BF16


def _draw(T, H, seed, dtype=torch.bfloat16):
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.randn(T, H, generator=g) * torch.exp(torch.randn(T, 1, generator=g))).to(dtype)


def _codes(q, scales, fp8):
    """Values that codes and scales stand for, in double."""
    v = q.view(torch.float8_e4m3fn).float().double() if fp8 else q.double()
    s = scales.double()
    if fp8:
        s = s.repeat_interleave(128, dim=1)
    else:
        s = s[:, :1]
    return v * s


def _close_codes(q, scales, v, fp8):
    s = ref.amax_scales(v, fp8)
    got_s = scales.double().repeat_interleave(128, dim=1) if fp8 else scales.double()[:, :1]
    assert torch.all((got_s - s).abs() <= F32 * s)
    step = 2.0 ** -4 * v.abs() + 2.0 ** -10 * s if fp8 else 0.5 * s
    assert torch.all((_codes(q, scales, fp8) - v).abs() <= step * (1 + 1e-3) + F32 * v.abs())


def _run(x, residual, weight, eps, q_dtype=None, cols=0, want_y=True, want_sum=True, **kw):
    moe = _moe()
    T, H = x.shape
    dev = dict(device="cuda")
    out = dict(rstd=torch.full((T,), -1.0, **dev))
    out["sum"] = torch.empty(T, H, dtype=residual.dtype, **dev) \
        if residual is not None and want_sum else None
    out["y"] = torch.full((T, H), 9.0, dtype=torch.bfloat16, **dev) if want_y else None
    if q_dtype is not None:
        out["q"] = torch.full((T, H), 77, dtype=torch.int8, **dev)
        n = cols or (H // 128 if q_dtype == moe.MOE_DTYPE_FP8_E4M3 else 1)
        out["scales"] = torch.full((T, n), -3.0, **dev)
    moe.moe_rmsnorm(x.cuda(), None if residual is None else residual.cuda(), _dt(residual),
                    weight.cuda(), _dt(weight), eps, T, H, out["sum"], out["y"],
                    0 if q_dtype is None else q_dtype, out.get("q"), out.get("scales"),
                    out["rstd"], cols, **kw)
    torch.cuda.synchronize()
    return {k: None if v is None else v.cpu() for k, v in out.items()}


SHAPES = [(1, 8), (5, 16), (3, 128), (9, 512), (6, 520), (130, 1024), (7, 1032), (17, 2056),
          (33, 4096), (20, 7168), (3, 8208), (2, 16384)]


@pytest.mark.parametrize("T,H", SHAPES)
@pytest.mark.parametrize("res", [None, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("wf32", [False, True])
def test_norm(T, H, res, wf32):
    x = _draw(T, H, seed=H)
    r = None if res is None else _draw(T, H, seed=H + 1, dtype=res)
    w = _draw(1, H, seed=H + 2, dtype=torch.float32 if wf32 else torch.bfloat16)[0]
    out = _run(x, r, w, 1e-6)
    h, rstd, y = ref.rmsnorm(x.double(), None if r is None else r.double(), w.double(), 1e-6)
    assert torch.all((out["rstd"].double() - rstd).abs() <= F32 * rstd)
    assert torch.all((out["y"].double() - y).abs() <= (BF16 + F32) * y.abs())
    if r is not None:
        tol = 2.0 ** -24 if res == torch.float32 else BF16
        assert torch.all((out["sum"].double() - h).abs() <= tol * h.abs() * 1.001)


@pytest.mark.parametrize("T,H", [(1, 128), (5, 512), (130, 1024), (9, 1152), (20, 7168), (2, 16384)])
@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("res", [None, torch.bfloat16, torch.float32])
def test_norm_codes(T, H, fp8, res):
    moe = _moe()
    x = _draw(T, H, seed=H)
    r = None if res is None else _draw(T, H, seed=H + 1, dtype=res)
    w = _draw(1, H, seed=H + 2)[0]
    d = moe.MOE_DTYPE_FP8_E4M3 if fp8 else moe.MOE_DTYPE_INT8
    out = _run(x, r, w, 1e-5, d)
    _, _, y = ref.rmsnorm(x.double(), None if r is None else r.double(), w.double(), 1e-5)
    _close_codes(out["q"], out["scales"], y, fp8)
    assert torch.all((out["y"].double() - y).abs() <= (BF16 + F32) * y.abs())
    if not fp8:                                    # scale rows as dispatch carries them
        wide = _run(x, r, w, 1e-5, d, cols=H // 128, want_y=False)
        assert torch.equal(wide["q"], out["q"])
        assert torch.equal(wide["scales"], out["scales"].expand(T, H // 128))


@pytest.mark.parametrize("H", [16, 48, 1040, 2064])
def test_norm_int8_odd_widths(H):
    moe = _moe()
    x, w = _draw(11, H, seed=H), _draw(1, H, seed=1)[0]
    out = _run(x, None, w, 0.0, moe.MOE_DTYPE_INT8)
    _, _, y = ref.rmsnorm(x.double(), None, w.double(), 0.0)
    _close_codes(out["q"], out["scales"], y, False)


def test_norm_pitches_and_in_place_sum():
    moe = _moe()
    T, H = 37, 1024
    wide, wres = _draw(T, H + 64, seed=1).cuda(), _draw(T, H + 32, seed=2, dtype=torch.float32).cuda()
    w = _draw(1, H, seed=3)[0].cuda()
    x, r = wide[:, 8:8 + H], wres[:, 4:4 + H]
    y = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    moe.moe_rmsnorm(x, r, moe.MOE_DTYPE_F32, w, moe.MOE_DTYPE_BF16, 1e-6, T, H, None, y, 0, None,
                    None, None, x_pitch=H + 64, residual_pitch=H + 32)
    _, _, want = ref.rmsnorm(x.cpu().double(), r.cpu().double(), w.cpu().double(), 1e-6)
    assert torch.all((y.cpu().double() - want).abs() <= (BF16 + F32) * want.abs())
    packed = r.contiguous()
    before = packed.cpu().double()
    moe.moe_rmsnorm(x, packed, moe.MOE_DTYPE_F32, w, moe.MOE_DTYPE_BF16, 1e-6, T, H, packed, y, 0,
                    None, None, None, x_pitch=H + 64)
    h = x.cpu().double() + before
    assert torch.all((packed.cpu().double() - h).abs() <= 2.0 ** -23 * h.abs())
    assert torch.all((y.cpu().double() - want).abs() <= (BF16 + F32) * want.abs())


@pytest.mark.parametrize("fp8", [True, False])
def test_zero_tiny_and_non_finite_rows(fp8):
    moe = _moe()
    H = 1024
    x = torch.randn(6, H, generator=torch.Generator().manual_seed(0)).bfloat16()
    x[0] = 0
    x[1] = 0
    x[1, 5] = 1e-38                                # far below 2^-100: some scale, no NaN
    x[3, 700] = math.inf
    x[4, 700] = math.nan
    q = torch.empty(6, H, dtype=torch.int8, device="cuda")
    s = torch.empty(6, H // 128 if fp8 else 1, device="cuda")
    moe.moe_quantize(x.cuda(), 6, H, moe.MOE_DTYPE_FP8_E4M3 if fp8 else moe.MOE_DTYPE_INT8, q, s)
    q, s = q.cpu(), s.cpu()
    assert torch.all(s[0] == 1) and torch.all(q[0] == 0)
    v = _codes(q, s, fp8)
    assert torch.all(torch.isfinite(v[:3])) and torch.all(torch.isfinite(v[5]))
    assert torch.all((v[1] - x[1].double()).abs() <= 2e-31)
    _close_codes(q[[2, 5]], s[[2, 5]], x[[2, 5]].double(), fp8)
    block = slice(640, 768) if fp8 else slice(0, H)
    for row in (3, 4):                             # the block shows it, the others are whole
        assert not torch.any(torch.isfinite(v[row, block]))
    if fp8:
        _close_codes(q[3:5, :640], s[3:5, :5], x[3:5, :640].double(), True)
    # the norm: a row of zeros stays zero, a NaN spreads over its row
    out = _run(x[[0, 4, 5]], None, torch.ones(H).bfloat16(), 1e-6,
               moe.MOE_DTYPE_FP8_E4M3 if fp8 else moe.MOE_DTYPE_INT8)
    assert torch.all(out["y"][0] == 0) and torch.all(out["q"][0] == 0)
    assert torch.all(torch.isnan(out["y"][1].float())) and torch.all(torch.isnan(out["scales"][1]))
    assert torch.all(torch.isfinite(out["scales"][2]))


@pytest.mark.parametrize("rows,H", [(1, 16), (300, 256), (64, 2048), (9, 1424), (5, 16384)])
@pytest.mark.parametrize("skip", [False, True])
def test_quantize_rows(rows, H, skip):
    moe = _moe()
    x = _draw(rows, H, seed=rows)
    src = torch.arange(rows, dtype=torch.int32)
    if skip:
        src[1::3] = -1
    for fp8 in (False, True):
        if fp8 and H % 128:
            continue
        q = torch.full((rows, H), 77, dtype=torch.int8, device="cuda")
        s = torch.full((rows, H // 128 if fp8 else 1), -3.0, device="cuda")
        moe.moe_quantize(x.cuda(), rows, H, moe.MOE_DTYPE_FP8_E4M3 if fp8 else moe.MOE_DTYPE_INT8,
                         q, s, row_src=src.cuda() if skip else None)
        q, s = q.cpu(), s.cpu()
        live = src >= 0
        _close_codes(q[live], s[live], x[live].double(), fp8)
        assert torch.all(q[~live] == 77) and torch.all(s[~live] == -3.0)


def test_norm_feeds_the_fp8_dispatch():
    """Codes and scales go to moe_dispatch as they are: every routed row of the
    region is its token's row."""
    moe = _moe()
    T, H, E, k = 70, 1024, 16, 4
    x, w = _draw(T, H, seed=5), _draw(1, H, seed=6)[0]
    for d, cols in ((moe.MOE_DTYPE_FP8_E4M3, 0), (moe.MOE_DTYPE_INT8, H // 128)):
        out = _run(x, None, w, 1e-6, d, cols=cols, want_y=False)
        idx = torch.stack([torch.randperm(E, generator=torch.Generator().manual_seed(t))[:k]
                           for t in range(T)]).int().cuda()
        lay = moe.Layout(T, k, E, 1)
        lay.run(idx)
        rows, srows = moe.Regions([T * k], H), moe.Regions([T * k], H // 128 * 4)
        moe.moe_dispatch(out["q"].cuda(), out["scales"].cuda(), moe.MOE_DTYPE_FP8_E4M3, H, E, 1, idx,
                         lay.pos, lay.rank_offset, rows.table, srows.table, rows.cap, lay.workspace,
                         lay.status)
        torch.cuda.synchronize()
        tok = lay.row_src[:T * k].cpu().long() // k
        assert torch.equal(rows.region(0).cpu().view(torch.int8), out["q"][tok])
        assert torch.equal(srows.region(0).cpu().contiguous().view(torch.float32),
                           out["scales"][tok])


def test_no_rows():
    out = _run(torch.empty(0, 128).bfloat16(), None, torch.ones(128), 1e-6)
    assert out["y"].shape == (0, 128)


# ----------------------------------------------------------------- gradients
def _back(gy, h, rstd, w, gs, weight_grad=True):
    moe = _moe()
    T, H = h.shape
    gx = torch.full_like(h, 5.0).cuda()
    gw = torch.full((H,), 5.0, device="cuda") if weight_grad else None
    n = moe.moe_rmsnorm_backward_workspace_bytes(T, H)
    ws = torch.full((max(1, n),), 0xFF, dtype=torch.uint8, device="cuda") if weight_grad else None
    moe.moe_rmsnorm_backward(gy.cuda(), h.cuda(), _dt(h), rstd.cuda(), w.cuda(), _dt(w),
                             None if gs is None else gs.cuda(), T, H, gx, gw, ws)
    torch.cuda.synchronize()
    return gx.cpu(), None if gw is None else gw.cpu()


@pytest.mark.parametrize("T,H", SHAPES + [(5000, 256), (3000, 2048)])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("with_sum", [False, True])
def test_norm_gradients(T, H, f32, with_sum):
    """Every sum is a chain of at most 64 serial float32 additions and a tree of
    a dozen: 80 roundings of 2^-24 of the sum of magnitudes."""
    dtype = torch.float32 if f32 else torch.bfloat16
    h, gy = _draw(T, H, seed=H, dtype=dtype), _draw(T, H, seed=H + 1)
    w = _draw(1, H, seed=H + 2, dtype=dtype)[0]
    gs = _draw(T, H, seed=H + 3, dtype=dtype) if with_sum else None
    rstd = (1 / (h.double().square().mean(1) + 1e-6).sqrt()).float()
    gx, gw = _back(gy, h, rstd, w, gs)
    d = [v.double() for v in (gy, h, rstd, w)]
    want, want_w = ref.rmsnorm_grad(*d, None if gs is None else gs.double())
    u, r = d[0] * d[3], d[2][:, None]
    size = r * u.abs() + d[1].abs() * r ** 3 * (u * d[1]).abs().mean(1, keepdim=True)
    tol = 80 * 2.0 ** -24 * (size + (0 if gs is None else gs.double().abs()))
    if not f32:
        tol = tol + BF16 * want.abs()
    assert torch.all((gx.double() - want).abs() <= tol)
    mag = (d[0] * d[1] * r).abs().sum(0)
    assert torch.all((gw.double() - want_w).abs() <= 80 * 2.0 ** -24 * mag)
    only, none = _back(gy, h, rstd, w, gs, weight_grad=False)
    assert none is None and torch.equal(only, gx)
    again, again_w = _back(gy, h, rstd, w, gs)
    assert torch.equal(again, gx) and torch.equal(again_w, gw)     # equal calls, equal bits


def test_norm_gradient_against_differences():
    """The gradient along random directions against central differences of the
    definition in 64 bits (step 1e-5: 1e-8 from the third derivative and the
    rounding), float32 inputs: 1e-4 of the gradient's norm."""
    T, H = 4, 1032
    h, gy = _draw(T, H, seed=1, dtype=torch.float32), _draw(T, H, seed=2)
    w = _draw(1, H, seed=3, dtype=torch.float32)[0]
    rstd = (1 / (h.double().square().mean(1) + 1e-6).sqrt()).float()
    gx, gw = _back(gy, h, rstd, w, None)

    def loss(hh, ww):
        return (ref.rmsnorm(hh, None, ww, 1e-6)[2] * gy.double()).sum()
    for n in range(5):
        g = torch.Generator().manual_seed(n)
        dh, dw = torch.randn(T, H, generator=g).double(), torch.randn(H, generator=g).double()
        a = (loss(h.double() + 1e-5 * dh, w.double()) - loss(h.double() - 1e-5 * dh, w.double())) / 2e-5
        assert abs(float((gx.double() * dh).sum() - a)) <= 1e-4 * float(gx.double().norm() * dh.norm())
        b = (loss(h.double(), w.double() + 1e-5 * dw) - loss(h.double(), w.double() - 1e-5 * dw)) / 2e-5
        assert abs(float((gw.double() * dw).sum() - b)) <= 1e-4 * float(gw.double().norm() * dw.norm())


def test_gradient_may_overwrite_grad_sum():
    moe = _moe()
    T, H = 300, 2048
    h, gy, gs = _draw(T, H, 1).cuda(), _draw(T, H, 2).cuda(), _draw(T, H, 3).cuda()
    w = _draw(1, H, 4)[0].cuda()
    rstd = (1 / (h.float().square().mean(1) + 1e-6).sqrt())
    a = torch.empty_like(h)
    for gx, s in ((a, gs), (gs, gs)):
        moe.moe_rmsnorm_backward(gy, h, moe.MOE_DTYPE_BF16, rstd, w, moe.MOE_DTYPE_BF16, s, T, H,
                                 gx, None, None)
    assert torch.equal(a, gs)


def test_weight_gradient_of_no_tokens_is_zero():
    z = torch.empty(0, 256).bfloat16()
    gx, gw = _back(z, z, torch.empty(0), torch.ones(256), None)
    assert torch.all(gw == 0)


@pytest.mark.parametrize("T,H", [(5, 128), (6, 1024), (3, 4096), (4, 16384), (1100, 7168)])
@pytest.mark.parametrize("exponents", [(40, 100), (-50, -90)])
def test_products_of_row_and_weight_beyond_float32(T, H, exponents):
    """v = (h rstd) weight lies within float32 where h weight does not, or is below the
    normal range.  Every second row is an ordinary one (with 1100 rows a workgroup takes both
    kinds), every fifth is zero."""
    moe = _moe()
    up_x, up_w = exponents
    g = torch.Generator().manual_seed(H)
    x = torch.randn(T, H, generator=g)
    x[::2] *= 2.0 ** up_x
    x[::5] = 0
    x = x.bfloat16()
    w = (1 + 0.1 * torch.randn(H, generator=g)) * 2.0 ** up_w
    h, rstd, v = ref.rmsnorm(x.double(), None, w.double(), 1e-37)
    for d in (None, moe.MOE_DTYPE_FP8_E4M3, moe.MOE_DTYPE_INT8):
        out = _run(x, None, w, 1e-37, d)
        assert torch.all((out["rstd"].double() - rstd).abs() <= F32 * rstd)
        assert torch.all((out["y"].double() - v).abs() <= (BF16 + F32) * v.abs())
        if d is not None:
            _close_codes(out["q"], out["scales"], v, d == moe.MOE_DTYPE_FP8_E4M3)


@pytest.mark.parametrize("T,H", [(7, 256), (5, 4096), (900, 2048)])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("exponents", [(40, 100), (-50, -90)])
def test_gradients_of_products_beyond_float32(T, H, f32, exponents):
    """The gradients lie within float32 where grad_y weight h does not, or is below the
    normal range; bounds as for ordinary rows."""
    up_h, up_w = exponents
    dtype = torch.float32 if f32 else torch.bfloat16
    h = (_draw(T, H, seed=H, dtype=torch.float32) * 2.0 ** up_h).to(dtype)
    gy = _draw(T, H, seed=H + 1)
    w = ((1 + 0.1 * _draw(1, H, seed=H + 2, dtype=torch.float32)[0]) * 2.0 ** up_w).to(dtype)
    rstd = (1 / (h.double().square().mean(1) + 1e-37).sqrt()).float()
    gx, gw = _back(gy, h, rstd, w, None)
    d = [v.double() for v in (gy, h, rstd, w)]
    want, want_w = ref.rmsnorm_grad(*d, None)
    u, r = d[0] * d[3], d[2][:, None]
    size = r * u.abs() + d[1].abs() * r ** 3 * (u * d[1]).abs().mean(1, keepdim=True)
    tol = 80 * 2.0 ** -24 * size + (0 if f32 else BF16 * want.abs())
    assert torch.all((gx.double() - want).abs() <= tol)
    mag = (d[0] * d[1] * r).abs().sum(0)
    assert torch.all((gw.double() - want_w).abs() <= 80 * 2.0 ** -24 * mag)


@pytest.mark.parametrize("fp8", [True, False])
def test_quantize_no_rows(fp8):
    moe = _moe()
    x = torch.empty(0, 256, dtype=torch.bfloat16, device="cuda")
    moe.moe_quantize(x, 0, 256, moe.MOE_DTYPE_FP8_E4M3 if fp8 else moe.MOE_DTYPE_INT8,
                     torch.empty(0, 256, dtype=torch.int8, device="cuda"),
                     torch.empty(0, 2, device="cuda"), scale_cols=2)
    torch.cuda.synchronize()


# More rows than stay on the GPU at once (4096 of 128, 1024 of 2064, 512 of 7168, 256 of 16384):
# workgroups take a third row, some of them not, and ask for the next one early.
@pytest.mark.parametrize("T,H", [(9001, 128), (2900, 2064), (1200, 7168), (600, 16384)])
@pytest.mark.parametrize("kind", ["bf16", "fp8", "int8"])
@pytest.mark.parametrize("res", [None, torch.bfloat16, torch.float32])
def test_norm_of_many_rows(T, H, kind, res):
    moe = _moe()
    if kind == "fp8" and H % 128:
        H = H // 128 * 128
    x = _draw(T, H, seed=T)
    r = None if res is None else _draw(T, H, seed=T + 1, dtype=res)
    w = _draw(1, H, seed=T + 2, dtype=torch.float32 if res == torch.float32 else torch.bfloat16)[0]
    d = dict(bf16=None, fp8=moe.MOE_DTYPE_FP8_E4M3, int8=moe.MOE_DTYPE_INT8)[kind]
    out = _run(x, r, w, 1e-6, d, want_y=kind != "fp8")
    h, rstd, y = ref.rmsnorm(x.double(), None if r is None else r.double(), w.double(), 1e-6)
    assert torch.all((out["rstd"].double() - rstd).abs() <= F32 * rstd)
    if out["y"] is not None:
        assert torch.all((out["y"].double() - y).abs() <= (BF16 + F32) * y.abs())
    if d is not None:
        _close_codes(out["q"], out["scales"], y, kind == "fp8")
    if r is not None:
        tol = 2.0 ** -24 if res == torch.float32 else BF16
        assert torch.all((out["sum"].double() - h).abs() <= tol * h.abs() * 1.001)


@pytest.mark.parametrize("T,H", [(9001, 128), (1200, 7168)])
@pytest.mark.parametrize("res", [torch.bfloat16, torch.float32])
def test_sum_over_the_residual_of_many_rows(T, H, res):
    """Written in place while later rows' residuals are asked for: the same bits as beside it."""
    moe = _moe()
    x, r = _draw(T, H, seed=1).cuda(), _draw(T, H, seed=2, dtype=res).cuda()
    w = _draw(1, H, seed=3)[0].cuda()
    apart = [torch.empty(T, H, dtype=res, device="cuda"),
             torch.empty(T, H, dtype=torch.bfloat16, device="cuda")]
    moe.moe_rmsnorm(x, r, _dt(r), w, moe.MOE_DTYPE_BF16, 1e-6, T, H, *apart, 0, None, None, None)
    y = torch.empty_like(apart[1])
    moe.moe_rmsnorm(x, r, _dt(r), w, moe.MOE_DTYPE_BF16, 1e-6, T, H, r, y, 0, None, None, None)
    assert torch.equal(r, apart[0]) and torch.equal(y, apart[1])
    assert torch.equal(r[T - 1].cpu().double(),
                       (x[T - 1].cpu().double() + _draw(T, H, seed=2, dtype=res)[T - 1].double())
                       .to(torch.float32).to(res).double())


@pytest.mark.parametrize("rows,H", [((1 << 22) + 99, 128), ((1 << 20) + 77, 1152)])
@pytest.mark.parametrize("fp8", [True, False])
def test_quantize_more_rows_than_one_grid(rows, H, fp8):
    """Workgroups go round again, over rows that are skipped and rows that are not: the last
    rows as in a call of their own, and as the definition has them."""
    moe = _moe()
    d = moe.MOE_DTYPE_FP8_E4M3 if fp8 else moe.MOE_DTYPE_INT8
    cols, tail = H // 128 if fp8 else 1, 3000
    g = torch.Generator(device="cuda")
    g.manual_seed(H)
    x = torch.randn(rows, H, generator=g, device="cuda", dtype=torch.bfloat16)
    src = torch.arange(rows, dtype=torch.int32, device="cuda")
    src[1::3] = -1
    q = torch.full((rows, H), 77, dtype=torch.int8, device="cuda")
    s = torch.full((rows, cols), -3.0, device="cuda")
    moe.moe_quantize(x, rows, H, d, q, s, row_src=src)
    part_q = torch.full((tail, H), 77, dtype=torch.int8, device="cuda")
    part_s = torch.full((tail, cols), -3.0, device="cuda")
    moe.moe_quantize(x[-tail:], tail, H, d, part_q, part_s, row_src=src[-tail:])
    assert torch.equal(q[-tail:], part_q) and torch.equal(s[-tail:], part_s)
    live = (src[-200:] >= 0).cpu()
    _close_codes(q[-200:].cpu()[live], s[-200:].cpu()[live], x[-200:].cpu()[live].double(), fp8)
    assert bool((q[src < 0] == 77).all()) and bool((s[src < 0] == -3.0).all())
    assert bool((s[src >= 0] > 0).all())
