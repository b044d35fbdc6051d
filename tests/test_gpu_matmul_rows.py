"""The 8-bit products of as many rows as a call may have."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("windows", [False, True])
def test_as_many_rows_as_there_can_be(windows):
    """Row tiles whose count and last row come near 2^31; the rows' ends and some between.  Sums of
    16 products are exact, scales are powers of two: only the rounding to bf16 is left."""
    from paper_2607_26444_amd import moe
    rows, N, K, some = 2 ** 31 - 1, 8, 16, 300
    if torch.cuda.mem_get_info()[0] < 120e9:
        pytest.skip("not enough memory free")
    g = torch.Generator()
    g.manual_seed(11)
    aq = torch.randint(-127, 128, (some, K), generator=g, dtype=torch.int8)
    wq = torch.randint(-127, 128, (1, N, K), generator=g, dtype=torch.int8)
    ws = torch.full((1, N), 2.0 ** -7, device="cuda")
    a = torch.zeros(rows, K, dtype=torch.int8, device="cuda")
    s = torch.full((rows,), 0.5, device="cuda")
    y = torch.full((rows, N), 7.0, dtype=torch.bfloat16, device="cuda")
    starts = (0, 2 ** 30 - 100, rows - some)
    for at in starts:
        a[at:at + some] = aq.cuda()
    offset = count = None
    if windows:
        offset = torch.tensor([5, 5 + rows], dtype=torch.int64).int().cuda()   # a rank's own: from 5
        count = torch.tensor([rows], dtype=torch.int32, device="cuda")
    moe.moe_expert_matmul(a, s, rows, wq.cuda(), ws, 1, N, K, offset, count, moe.MOE_ACT_NONE, y)
    want = ((aq.double() @ wq[0].double().T) * 2.0 ** -8).bfloat16()           # 22 bits: exact before
    for at in starts:
        assert torch.equal(y[at:at + some].cpu(), want)
    for start, end in ((some, 2 ** 30 - 100), (2 ** 30 + 200, rows - some)):
        for i in range(start, end, 1 << 26):
            assert not torch.any(y[i:min(end, i + (1 << 26))])
