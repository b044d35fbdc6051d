"""The experts' int8 products against 64 bits.

The integer sums are exact; their conversion to float32 and two products round
three times (2^-24 each), the result once to bf16 (2^-8 at most): BF16 below.
SwiGLU: exp(-g) is off by (|g| + 2) 2^-24 of itself, |g| <= 64 wherever the output
is not vanishingly small.
"""
import math

import pytest

torch = pytest.importorskip("torch")

import layer_ref as ref  # noqa: E402
import matmul_rule  # noqa: E402

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8 * 1.01


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _moe():
    from paper_2607_26444_amd import moe
    return moe


def _inputs(rows, E, N, K, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    a = torch.randint(-128, 128, (rows, K), generator=g, dtype=torch.int8)
    w = torch.randint(-128, 128, (E, N, K), generator=g, dtype=torch.int8)
    sa = (0.5 + torch.rand(rows, generator=g)) / 73
    sw = (0.5 + torch.rand(E, N, generator=g)) / (73 * math.sqrt(K))
    return a, sa, w, sw


def _run(a, sa, w, sw, offset, count, swiglu, pitch=0, rows=None):
    moe = _moe()
    E, N, K = w.shape
    out = N // 2 if swiglu else N
    y = torch.full((max(1, a.shape[0]), out), math.nan, dtype=torch.bfloat16, device="cuda")
    dev = [None if t is None else torch.tensor(t, dtype=torch.int32, device="cuda")
           for t in (offset, count)]
    moe.moe_expert_matmul(a.cuda(), sa.cuda(), a.shape[0] if rows is None else rows, w.cuda(),
                          sw.cuda(), E, N, K, *dev,
                          moe.MOE_ACT_SWIGLU if swiglu else moe.MOE_ACT_NONE, y,
                          a_scale_pitch=pitch)
    torch.cuda.synchronize()
    return y.cpu()[:a.shape[0]]


def _check(y, a, sa, w, sw, windows, swiglu):
    want = ref.expert_matmul(a, sa, w, sw, windows, swiglu)
    y = y.double()
    assert torch.equal(torch.isnan(y), torch.isnan(want))     # rows of no window are untouched
    at = ~torch.isnan(want)
    assert torch.all((y[at] - want[at]).abs() <= BF16 * want[at].abs() + 1e-30)


def _packed(counts):
    offset = [0]
    for n in counts:
        offset.append(offset[-1] + n)
    return offset, list(zip(offset, counts))


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 33, 64, 100, 129, 257, 300])
@pytest.mark.parametrize("N,K", [(8, 16), (16, 64), (72, 48), (64, 128), (200, 144), (264, 1040)])
def test_plain_product(rows, N, K):
    t = _inputs(rows, 1, N, K, seed=rows + N + K)
    _check(_run(*t, None, None, False), *t, [(0, rows)], False)


@pytest.mark.parametrize("N,K", [(16, 16), (32, 64), (80, 272), (256, 128), (528, 400)])
@pytest.mark.parametrize("rows", [1, 31, 140, 270])
def test_swiglu(rows, N, K):
    t = _inputs(rows, 1, N, K, seed=rows * N)
    _check(_run(*t, None, None, True), *t, [(0, rows)], True)


@pytest.mark.parametrize("counts", [[0, 0, 0], [0, 5, 0, 0, 1], [1] * 70, [40, 0, 300, 17, 0, 1, 64],
                                    [0] * 63 + [3, 0, 9], [256, 512, 128], [2] * 130])
@pytest.mark.parametrize("swiglu", [False, True])
def test_packed_windows(counts, swiglu):
    E, N, K = len(counts), 96, 208
    offset, windows = _packed(counts)
    t = _inputs(offset[-1], E, N, K, seed=E)
    for count in (counts, None):
        if offset[-1] == 0 and count is None:
            continue
        _check(_run(*t, offset, count, swiglu), *t, windows, swiglu)


@pytest.mark.parametrize("cap", [8, 40, 300])
def test_fixed_windows_of_a_rank(cap):
    """Windows of equal capacity filled in part, rows relative to the first
    window: the local experts of a rank with their own region."""
    counts = [3, 0, cap, 7, 1]
    base = 12345
    offset = [base + e * cap for e in range(6)]
    t = _inputs(5 * cap, 5, 88, 160, seed=cap)
    _check(_run(*t, offset, counts, False), *t, [(e * cap, n) for e, n in enumerate(counts)], False)


def test_windows_are_clipped_to_the_rows():
    t = _inputs(50, 3, 16, 32, seed=1)
    y = _run(*t, [0, 30, 70, 90], [30, 40, 20], False)        # the region holds 50 rows
    _check(y, *t, [(0, 30), (30, 20), (50, 0)], False)
    y = _run(*t, [5, 0, 60, 70], [-4, 9, 9], False)           # no window lies in the rows
    assert torch.all(torch.isnan(y.float()))


@pytest.mark.parametrize("rows,N,K,E", [(700, 1416, 2064, 3), (1500, 512, 1024, 2), (90, 4096, 512, 4),
                                        (2100, 264, 272, 1), (600, 1024, 4112, 2)])
@pytest.mark.parametrize("swiglu", [False, True])
def test_large_tiles(rows, N, K, E, swiglu):
    N = N // 16 * 16 if swiglu else N
    counts = [rows // E + (7 * e) % 50 - 20 for e in range(E - 1)]
    counts.append(rows - sum(counts))
    offset, windows = _packed(counts)
    t = _inputs(rows, E, N, K, seed=rows)
    _check(_run(*t, offset, counts, swiglu), *t, windows, swiglu)

# Sizes whose products fill the GPU with 256 x 256 tiles: windows that end after
# 1, 4, 65, 76 .. rows of a tile, outputs that end inside a tile, a depth that ends inside a
# stage and one that is shorter than a stage.
@pytest.mark.parametrize("counts,N,K", [([4100], 4112, 1040), ([8193], 2064, 16),
                                        ([0, 1024, 700, 2300, 65], 4112, 400),
                                        ([1000, 1], 16400, 272),
                                        ([65, 190, 3, 250] * 32 + [0, 700], 2064, 144)])
@pytest.mark.parametrize("swiglu", [False, True])
def test_many_tiles(counts, N, K, swiglu):
    E, rows = len(counts), sum(counts)
    N -= 0 if swiglu else 8                                   # an odd number of eights
    offset, windows = _packed(counts)
    t = _inputs(rows, E, N, K, seed=rows)
    y = _run(*t, offset, counts, swiglu) if E > 1 else _run(*t, None, None, swiglu)
    _check(y, *t, windows, swiglu)
    if E > 1:
        assert torch.equal(_run(*t, offset, None, swiglu), y)

# Sizes in between, each of which another kernel or size of tile takes: 128 rows,
# 64 rows x 128 channels, 64 x 64 with two stages, 64 x 32.
@pytest.mark.parametrize("counts,N,K", [([4161], 1040, 2064),
                                        ([129, 0, 64, 1, 127, 128, 65, 190] * 5, 1056, 528),
                                        ([1000], 4112, 528),
                                        ([63, 64, 65, 1, 0, 129] * 4, 2064, 1040),
                                        ([30] * 50, 2064, 400),
                                        ([230, 400, 70], 1424, 2064), ([512], 4112, 1552),
                                        ([139, 1], 1040, 2064), ([65, 17, 98], 1040, 2064)])
@pytest.mark.parametrize("swiglu", [False, True])
def test_tiles_in_between(counts, N, K, swiglu):
    E, rows = len(counts), sum(counts)
    N -= 0 if swiglu else 8
    offset, windows = _packed(counts)
    t = _inputs(rows, E, N, K, seed=rows)
    _check(_run(*t, offset, counts, swiglu), *t, windows, swiglu)


@pytest.mark.parametrize("swiglu", [False, True])
def test_many_tiles_fixed_windows(swiglu):
    """Equal capacities of which some are empty, full or hold a few rows; then all empty."""
    E, cap, N, K = 12, 800, 2064, 272
    counts = [0, 800, 1, 130, 257, 0, 799, 70, 512, 0, 0, 5]
    base = 4321
    offset = [base + e * cap for e in range(E + 1)]
    t = _inputs(E * cap, E, N, K, seed=12)
    windows = [(e * cap, n) for e, n in enumerate(counts)]
    _check(_run(*t, offset, counts, swiglu), *t, windows, swiglu)
    assert torch.all(torch.isnan(_run(*t, offset, [0] * E, swiglu).float()))


def test_many_tiles_against_few():
    """The same rows in one call and in calls of 40 rows, which another kernel takes."""
    a, sa, w, sw = _inputs(4100, 1, 4112, 1040, seed=5)
    y = _run(a, sa, w, sw, None, None, True)
    for r in (0, 1000, 2048, 4060):
        assert torch.equal(_run(a[r:r + 40], sa[r:r + 40], w, sw, None, None, True), y[r:r + 40])


def test_scale_pitch():
    a, sa, w, sw = _inputs(40, 1, 64, 128, seed=2)
    wide = sa[:, None].expand(40, 5).contiguous()
    _check(_run(a, wide, w, sw, None, None, False, pitch=5), a, sa, w, sw, [(0, 40)], False)


@pytest.mark.parametrize("rows,N", [(1, 8), (300, 264)])
def test_deepest_sum_of_extremes(rows, N):
    """All -128 at the deepest product: the sum is one rounding off 2^31."""
    K = _moe().MOE_MAX_DEPTH
    a = torch.full((rows, K), -128, dtype=torch.int8)
    w = torch.full((1, N, K), -128, dtype=torch.int8)
    w[0, 1] = 127
    y = _run(a, torch.ones(rows), w, torch.full((1, N), 2.0 ** -31), None, None, False).double()
    want = torch.full((N,), 128 * 128 * K * 2.0 ** -31).double()
    want[1] = -128 * 127 * K * 2.0 ** -31
    assert torch.all((y - want).abs() <= BF16 * want.abs())


def test_non_finite_scales_show():
    a, sa, w, sw = _inputs(20, 1, 32, 64, seed=3)
    sa[4] = math.nan
    sa[5] = math.inf
    y = _run(a, sa, w, sw, None, None, False).float()
    assert torch.all(torch.isnan(y[4])) and not torch.any(torch.isfinite(y[5]))
    assert torch.all(torch.isfinite(y[[3, 6]]))


@pytest.mark.parametrize("n", [3, 200])
def test_offsets_past_32_bits(n):
    """Rows, weights and outputs whose byte offsets pass 2^32: the last window of many."""
    moe = _moe()
    E, N, K, cap = 34, 2048, 65536, 2000
    rows = E * cap                              # 4.5 GB of rows, 4.6 GB of weights
    a = torch.zeros(rows, K, dtype=torch.int8, device="cuda")
    w = torch.zeros(E, N, K, dtype=torch.int8, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    start = (E - 1) * cap + cap - n
    a[start:] = torch.randint(-128, 128, (n, K), generator=g, device="cuda", dtype=torch.int8)
    w[-1, -8:] = torch.randint(-128, 128, (8, K), generator=g, device="cuda", dtype=torch.int8)
    offset = torch.arange(E + 1, dtype=torch.int32, device="cuda") * cap
    offset[E - 1] = start
    count = torch.zeros(E, dtype=torch.int32, device="cuda")
    count[-1] = n
    sa = torch.full((rows,), 1 / 73, device="cuda")
    sw = torch.full((E, N), 1 / (73 * 256.0), device="cuda")
    y = torch.zeros(rows, N, dtype=torch.bfloat16, device="cuda")
    moe.moe_expert_matmul(a, sa, rows, w, sw, E, N, K, offset, count, moe.MOE_ACT_NONE, y)
    want = (a[start:].double() @ w[-1, -8:].double().T) / (73 * 73 * 256.0)
    got = y[start:, -8:].double()
    assert torch.all((got - want).abs() <= BF16 * want.abs() + 1e-9)
    assert not torch.any(y[:start]) and not torch.any(y[start:, :-8])


def test_no_rows():
    moe = _moe()
    w = torch.zeros(1, 8, 16, dtype=torch.int8, device="cuda")
    moe.moe_expert_matmul(None, None, 0, w, torch.ones(8, device="cuda"), 1, 8, 16, None, None,
                          moe.MOE_ACT_NONE, None)


def test_other_streams():
    """Calls on a stream of their own, inputs made there."""
    a, sa, w, sw = _inputs(130, 1, 256, 512, seed=4)
    s = torch.cuda.Stream()
    moe = _moe()
    with torch.cuda.stream(s):
        dev = [t.cuda(non_blocking=True) for t in (a, sa, w, sw)]
        y = torch.empty(130, 256, dtype=torch.bfloat16, device="cuda")
        moe.moe_expert_matmul(dev[0], dev[1], 130, dev[2], dev[3], 1, 256, 512, None, None,
                              moe.MOE_ACT_NONE, y)
    s.synchronize()
    _check(y.cpu(), a, sa, w, sw, [(0, 130)], False)


def test_more_rows_than_one_launch_has_workgroups():
    """600 million rows of a narrow product: tiles of 64 rows would need more workgroups than
    a launch has.  Sums of 16 products are exact in float32; checked in pieces on the GPU,
    the rounding to bf16 as for the others."""
    moe = _moe()
    rows, N, K = 600_000_000, 8, 16
    if torch.cuda.mem_get_info()[0] < 40e9:
        pytest.skip("not enough memory free")
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    a = torch.empty(rows, K, dtype=torch.int8, device="cuda")
    step = 50_000_000
    for i in range(0, rows, step):
        a[i:i + step] = torch.randint(-128, 128, (step, K), generator=g, device="cuda",
                                      dtype=torch.int8)
    w = torch.randint(-128, 128, (1, N, K), generator=g, device="cuda", dtype=torch.int8)
    sa = torch.rand(rows, generator=g, device="cuda") + 0.5
    sw = torch.rand(1, N, generator=g, device="cuda") + 0.5
    y = torch.empty(rows, N, dtype=torch.bfloat16, device="cuda")
    moe.moe_expert_matmul(a, sa, rows, w, sw, 1, N, K, None, None, moe.MOE_ACT_NONE, y)
    for i in range(0, rows, step):
        want = (a[i:i + step].float() @ w[0].float().T.contiguous()) * sa[i:i + step, None] * sw
        assert bool(((y[i:i + step].float() - want).abs() <= BF16 * want.abs()).all()), i


@pytest.mark.parametrize("case", matmul_rule.CASES, ids=lambda c: f"{c[0]}-{len(c[1])}-{c[3]}-{c[4]}")
@pytest.mark.parametrize("swiglu", [False, True])
def test_every_way(case, swiglu):
    """Each kernel and size of tile on packed or fixed windows."""
    _, counts, cap, _, _ = case
    rows, E, N, K, _, _ = matmul_rule.call_of(case, swiglu)
    if cap:
        offset, windows = [777 + e * cap for e in range(E + 1)], \
            [(e * cap, n) for e, n in enumerate(counts)]
    else:
        offset, windows = _packed(counts)
    t = _inputs(rows, E, N, K, seed=rows + N)
    y = _run(*t, offset, counts, swiglu)
    _check(y, *t, windows, swiglu)
    if not cap and E > 1:
        assert torch.equal(_run(*t, offset, None, swiglu), y)


@pytest.mark.parametrize("way,rows,E,N,K", matmul_rule.PAST_32_BITS)
def test_every_kernel_past_32_bits(way, rows, E, N, K):
    """Weights, rows or outputs whose byte offsets pass 2^32: the last rows, and channels of
    the last expert."""
    moe = _moe()
    n = min(rows, max(3, rows // E))
    start = rows - n
    g = torch.Generator(device="cuda")
    g.manual_seed(1)

    def int8(*shape):
        return torch.randint(-128, 128, shape, generator=g, device="cuda", dtype=torch.int8)
    a = torch.zeros(rows, K, dtype=torch.int8, device="cuda")
    w = torch.zeros(E, N, K, dtype=torch.int8, device="cuda")
    a[start:], w[-1, -8:] = int8(n, K), int8(8, K)
    offset = torch.full((E + 1,), start, dtype=torch.int32, device="cuda")
    offset[0], offset[E] = 0, rows
    count = torch.zeros(E, dtype=torch.int32, device="cuda")
    count[-1] = n
    sa = torch.full((rows,), 1 / 73, device="cuda")
    sw = torch.full((E, N), 1 / (73 * 256.0), device="cuda")
    y = torch.zeros(rows, N, dtype=torch.bfloat16, device="cuda")
    moe.moe_expert_matmul(a, sa, rows, w, sw, E, N, K, offset, count, moe.MOE_ACT_NONE, y)
    want = (a[start:].double() @ w[-1, -8:].double().T.contiguous()) / (73 * 73 * 256.0)
    got = y[start:, -8:].double()
    assert torch.all((got - want).abs() <= BF16 * want.abs() + 1e-9)
    assert not torch.any(y[:start]) and not torch.any(y[start:, :-8])
