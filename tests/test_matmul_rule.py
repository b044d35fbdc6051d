"""The launch rule of the experts' products, on the CPU: the way that it chooses can be
launched."""
import itertools

import pytest

pytest.importorskip("torch")

import matmul_rule  # noqa: E402


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    return matmul_rule.build_rule(tmp_path_factory.mktemp("rule"))


def _tiles(way, rows, E, N, K, swiglu, windows):
    """Tiles that the windows can have: each may add one that is not full."""
    height, channels = matmul_rule.TILE[way]
    out, per = (N // 2, channels // 2) if swiglu else (N, channels)
    row_tiles = rows // height + min(rows, E) if windows else -(-rows // height)
    return row_tiles * -(-out // per)


def test_every_call_gets_a_way_that_can_be_launched(choose):
    """One workgroup of 512 threads for each tile of a streaming way, at most 2^32 threads in
    all; the tile kernels stay resident and number their tiles in 32 bits.  Rows,
    weights and outputs together stay within the memory of one GPU."""
    calls = []
    for rows, E, N, K, swiglu in itertools.product(
            (1, 300, 70_000, 4_000_000, 540_000_000, 600_000_000, 2 ** 31 - 1), (1, 2, 64, 1024),
            (8, 16, 64, 256, 1024, 8192), (16, 128, 2048), (0, 1)):
        if swiglu and N % 16:
            continue
        out = N // 2 if swiglu else N
        if rows * (K + 4 + 2 * out) + E * N * (K + 4) > 288e9:
            continue
        calls.append((rows, E, N, K, swiglu, 1))
        if E == 1:
            calls.append((rows, E, N, K, swiglu, 0))
    calls += [(540_000_000, 1, 64, 128, 0, 0), (600_000_000, 1, 8, 16, 0, 0)]
    for call, way in zip(calls, choose(calls)):
        tiles = _tiles(way, *call)
        if way.startswith("tile"):
            assert tiles < 2 ** 31 - 512, (way, call)
        else:
            assert -(-tiles // 256) * 256 * 512 < 2 ** 32, (way, call)


@pytest.mark.parametrize("swiglu", [0, 1])
def test_the_sizes_of_the_gpu_tests_take_every_way(choose, swiglu):
    got = choose([matmul_rule.call_of(c, swiglu) for c in matmul_rule.CASES])
    assert got == [c[0] for c in matmul_rule.CASES]
    assert set(got) == set(matmul_rule.WAYS)


def test_the_sizes_past_32_bits_take_their_ways(choose):
    calls = [(*c[1:], 0, 1) for c in matmul_rule.PAST_32_BITS]
    assert choose(calls) == [c[0] for c in matmul_rule.PAST_32_BITS]
    for rows, E, N, K, _, _ in calls:
        assert max(rows * K, E * N * K, 2 * rows * N) > 2 ** 32
