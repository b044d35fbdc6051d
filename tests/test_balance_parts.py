"""Parts of the balance loss's sequences, on the CPU, from the workspace that they need."""
import pytest

pytest.importorskip("torch")

from paper_2607_26444_amd import moe  # noqa: E402


@pytest.mark.parametrize("E", [1, 16, 31, 32])
def test_up_to_32_experts_one_workgroup_joins(E):
    """8192 sums of 32 experts at most, which one workgroup joins: the kernel of several never
    has a single one.  A part has two rows of 32 words and its live tokens, a sequence a ticket
    and two words of its loss."""
    sizes = sorted({n + d for b in range(31) for n in (2 ** b,) for d in (-1, 0, 1)} - {-1, 0})
    for T in sizes:
        bytes_ = moe.moe_balance_workspace_bytes(T, E)
        parts = (bytes_ - 12) // 260 if bytes_ else 1
        assert bytes_ in (0, parts * 260 + 12) and parts * 32 <= 8192
        if T > 2 ** 20:
            assert parts > 128
