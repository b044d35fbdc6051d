"""The balance loss on either side of where a sequence is cut, against 64 bits, with the bounds of
test_gpu_balance."""
import pytest

torch = pytest.importorskip("torch")

import test_gpu_balance as base  # noqa: E402
from test_balance_parts import test_short_sequences_have_one_workgroup as _sizes  # noqa: E402

pytestmark = pytest.mark.gpu

SIZES = _sizes.pytestmark[0].args[1]          # experts, rounds of tokens that one workgroup takes


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("E,rounds", [s for s in SIZES if s[0] > 1])
@pytest.mark.parametrize("more", [0, 1, 7])
@pytest.mark.parametrize("S,sigmoid,pad", [(1, False, 0.0), (3, True, 0.3)])
def test_where_sequences_are_cut(E, rounds, more, S, sigmoid, pad):
    seq = rounds * (64 if E <= 256 else 16) + more
    x, idx, mask = base._inputs(S * seq, E, min(2, E), E + more, pad=pad)
    got = base._forward(x, idx, mask, sigmoid, seq)
    base._check_forward(got, x, idx, mask, sigmoid, seq)
    again = base._forward(x, idx, mask, sigmoid, seq)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
