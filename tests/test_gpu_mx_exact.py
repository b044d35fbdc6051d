"""The experts' products on 4-bit floats where every sum is exact, with weights that are
read past the caches.  Plain outputs have to be equal."""
import math

import pytest

torch = pytest.importorskip("torch")

import mx_exact  # noqa: E402

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


@pytest.mark.parametrize("case", mx_exact.READ_ONCE, ids=_ids)
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
