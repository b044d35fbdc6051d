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


@pytest.mark.parametrize("E,rounds", [(1, 12), (16, 12), (17, 9), (32, 9), (60, 6), (128, 3), (129, 2),
                                      (256, 2), (257, 3), (512, 3), (513, 2), (1024, 2)])
def test_short_sequences_have_one_workgroup(E, rounds):
    """Rounds of 64 tokens up to 256 experts, of 16 beyond; no workspace where one workgroup has the
    whole sequence.  A longer one is cut, unless there are more than 128 of them."""
    step = 64 if E <= 256 else 16
    assert moe.moe_balance_workspace_bytes(rounds * step, E) == 0
    assert moe.moe_balance_workspace_bytes(rounds * step + 1, E) > 0
    for S in (2, 128):
        assert moe.moe_balance_workspace_bytes(S * rounds * step, E, rounds * step) == 0
        assert moe.moe_balance_workspace_bytes(S * (rounds + 1) * step, E, (rounds + 1) * step) > 0
    assert moe.moe_balance_workspace_bytes(129 * 4096, E, 4096) == 0
