"""The experts' products on 4-bit floats where every sum is exact: as deep as a call may be, with
weights that are read past the caches, and past 2^32 bytes.  Plain outputs have to be equal."""
import math

import pytest

torch = pytest.importorskip("torch")

import mx_exact  # noqa: E402
import mx_rule  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def _run(a, w, offset, count, swiglu, K):
    from paper_2607_26444_amd import moe
    E, N, _ = w[0].shape
    y = torch.full((a[0].shape[0], N // 2 if swiglu else N), math.nan, dtype=torch.bfloat16, device="cuda")
    dev = [torch.tensor(t, dtype=torch.int32, device="cuda") for t in (offset, count)]
    moe.moe_expert_matmul_mx(a[0], a[1], a[0].shape[0], *w, E, N, K, *dev,
                             moe.MOE_ACT_SWIGLU if swiglu else moe.MOE_ACT_NONE, y)
    torch.cuda.synchronize()
    return y


def _ids(c):
    return f"{c[0]}-{sum(c[1])}-{len(c[1])}-{c[2]}-{c[3]}"


@pytest.mark.parametrize("case", mx_exact.DEEP + mx_exact.READ_ONCE, ids=_ids)
@pytest.mark.parametrize("swiglu", [False, True])
def test_exact_sums(case, swiglu):
    _, counts, N, K = case
    offset, windows = mx_exact.packed(counts)
    a, w = mx_exact.inputs(offset[-1], len(counts), N, K, sum(counts) + K, swiglu)
    y = _run(a, w, offset, counts, swiglu, K)
    mx_exact.check(y, a, w, windows, swiglu, K)
    assert torch.equal(_run(a, w, offset, counts, swiglu, K), y)


@pytest.mark.parametrize("rows,E,N,K", [b[:4] for b in mx_exact.BORDERS])
def test_on_either_side_of_the_rule_for_weights_read_once(rows, E, N, K):
    counts = mx_exact._ragged(E, rows, min(70, rows)) if E > 1 else [rows]
    offset, windows = mx_exact.packed(counts)
    a, w = mx_exact.inputs(rows, E, N, K, rows + N, False)
    mx_exact.check(_run(a, w, offset, counts, False, K), a, w, windows, False, K)


@pytest.mark.parametrize("way,rows,E,N,K", mx_rule.PAST_32_BITS)
def test_exact_sums_past_32_bits(way, rows, E, N, K):
    """Weights, rows, outputs or scales whose byte offsets pass 2^32: the last rows, with every channel
    of the last expert.  Codes and scales of a row lie in one, as dispatch carries them."""
    from paper_2607_26444_amd import moe
    n = min(rows, max(3, rows // E))
    start, half, cols = rows - n, K // 2, mx_exact.scale_cols(K)
    pitch = -(-(half + cols) // 16) * 16
    (aq, asc), (wq, wsc) = mx_exact.inputs(n, 1, N, K, rows, False)
    a = torch.zeros(rows, pitch, dtype=torch.uint8, device="cuda")
    w = torch.zeros(E, N, half, dtype=torch.uint8, device="cuda")
    ws = torch.full((E, N, cols), 127, dtype=torch.uint8, device="cuda")
    a[start:, :half], a[start:, half:half + cols] = aq, asc
    w[-1], ws[-1] = wq[0], wsc[0]
    offset = torch.full((E + 1,), start, dtype=torch.int32, device="cuda")
    offset[0], offset[E] = 0, rows
    count = torch.zeros(E, dtype=torch.int32, device="cuda")
    count[-1] = n
    y = torch.zeros(rows, N, dtype=torch.bfloat16, device="cuda")
    moe.moe_expert_matmul_mx(a, a[:, half:], rows, w, ws, E, N, K, offset, count, moe.MOE_ACT_NONE,
                             y, a_pitch=pitch, a_scale_pitch=pitch)
    mx_exact.check(y[start:], (aq, asc), (wq, wsc), [(0, n)], False, K)
    assert not torch.any(y[:start])


@pytest.mark.parametrize("spread", [0, 12, 24, 40])
@pytest.mark.parametrize("keep", [0.03, 0.3, 1.0])
def test_what_an_instruction_loses(spread, keep):
    """Two instructions (and the sum of two wavefronts or none) over blocks of scales up to 2^40 apart,
    two blocks of which cancel: 2^-20 of the sum of magnitudes each, and the rounding to bf16."""
    K, rows, N = 256, 300, 264
    g = torch.Generator(device="cuda")
    g.manual_seed(spread)
    byte = dict(dtype=torch.uint8, device="cuda")
    q = torch.randint(0, 256, (rows, K // 2), generator=g, **byte)
    q[torch.rand(q.shape, generator=g, device="cuda") >= keep] = 0
    wq = torch.randint(0, 256, (1, N, K // 2), generator=g, **byte)
    s = 127 - torch.randint(0, spread + 1, (rows, 8), generator=g, **byte)
    ws = torch.full((1, N, 8), 127, **byte)
    q[:, 32:64], wq[..., 32:64], s[:, :4] = q[:, :32], wq[..., :32] ^ 0x88, 127
    y = _run((q, s), (wq, ws), [0, rows], [rows], False, K).double()
    a, w = mx_exact.decode(q, s, K), mx_exact.decode(wq[0], ws[0], K)
    want = a @ w.T.contiguous()
    off = 2 * 2.0 ** -20 * (a.abs() @ w.abs().T.contiguous())
    assert torch.all((y - want).abs() <= 2.0 ** -8 * (want.abs() + off) + off)
    if not spread:
        assert torch.equal(y, want.float().bfloat16().double())
