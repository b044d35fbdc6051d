"""The exact products' inputs, sizes and check, on the CPU: each way of the launch rule has deep
calls and calls that read their weights past the caches, and the check notices a mistake of one
block."""
import pytest

torch = pytest.importorskip("torch")

import mx_exact  # noqa: E402


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    return mx_exact.build_rule(tmp_path_factory.mktemp("once"))


def _calls(cases, swiglu):
    return [(sum(counts), len(counts), N, K, swiglu) for _, counts, N, K in cases]


@pytest.mark.parametrize("swiglu", [0, 1])
def test_deep_sizes_take_every_way(choose, swiglu):
    ways = [way for way, _ in choose(_calls(mx_exact.DEEP, swiglu))]
    assert ways == [c[0] for c in mx_exact.DEEP] and len(set(ways)) == 8


@pytest.mark.parametrize("swiglu", [0, 1])
def test_weights_that_are_read_once_take_every_streaming_way(choose, swiglu):
    got = choose(_calls(mx_exact.READ_ONCE, swiglu))
    assert got == [(c[0], 1) for c in mx_exact.READ_ONCE]
    assert len({way for way, _ in got}) == 6
    for _, counts, _, _ in mx_exact.READ_ONCE:
        assert 0 in counts and max(counts) > 1


def test_when_weights_are_read_once(choose):
    for swiglu in (0, 1):
        got = [once for _, once in choose([(*b[:4], swiglu) for b in mx_exact.BORDERS])]
        assert got == [b[4] for b in mx_exact.BORDERS]


def _product(a, w, K, swiglu):
    v = mx_exact.decode(*a, K) @ mx_exact.decode(w[0][0], w[1][0], K).T
    if swiglu:
        g, u = v.chunk(2, 1)
        v = g * torch.sigmoid(g) * u
    return v.float().bfloat16()


@pytest.mark.parametrize("rows,N,K", [(5, 48, 131040), (3, 16, 65536), (40, 48, 8448), (1, 16, 2048)])
@pytest.mark.parametrize("swiglu", [False, True])
def test_the_check_notices_mistakes(rows, N, K, swiglu):
    a, w = mx_exact.inputs(rows, 1, N, K, rows + K, swiglu, device="cpu")
    windows = [(0, rows)]
    good = _product(a, w, K, swiglu)
    mx_exact.check(good, a, w, windows, swiglu, K)
    size = mx_exact.decode(*a, K).abs() @ mx_exact.decode(w[0][0], w[1][0], K).abs().T
    unit = 0.25 * float(2.0 ** (w[1][..., :K // 32].min().double() - 127))
    assert float(size.max()) < 2 ** 24 * unit        # every partial sum is a float32 number

    def refused(y):
        with pytest.raises(AssertionError):
            mx_exact.check(y, a, w, windows, swiglu, K)
    refused(torch.zeros_like(good))
    for at in (0, 32 * (K // 64), K - 32):           # a block of the depth left out
        q = a[0].clone()
        q[:, at // 2:at // 2 + 16] = 0
        refused(_product((q, a[1]), w, K, swiglu))
    for at in (0, K // 512 * 256):                   # a stage, or what there is of it, added twice
        s = a[1].clone()
        s[:, at // 32:min(at // 32 + 8, K // 32)] += 1
        refused(_product((a[0], s), w, K, swiglu))
    for block in (0, K // 32 - 1):                   # one scale of each row is the next power
        s = a[1].clone()
        s[:, block] += 1
        refused(_product((a[0], s), w, K, swiglu))
    refused(_product((a[0], a[1][:, torch.arange(a[1].shape[1]) ^ 1]), w, K, swiglu))
    y = good.clone()                                 # one output of another row or channel
    y[-1, -1] = good[0, 0]
    refused(y)
