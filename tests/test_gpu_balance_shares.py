"""Shares of logits that lie far apart or far down, against 64 bits.

Logits are multiples of 1/64 below 64 in size, whose differences float32 holds.  In units u of
2^-24, relative: an exponential 3 (its argument's rounding is made good, the hardware's result 2,
one rounding), 1 + e and its reciprocal 1 each, so that a softmax's term has 3 and a sigmoid score
5; with up to 16 terms in a lane and 64 lanes their sum adds 15 + 6, the quotient 2.  So a share is
off by 3 + 3 + 21 + 2 = 29 or 5 + 5 + 21 + 2 = 33 at most; 40 leaves room for the terms of second
order.  The mean of sequences of one token is the share itself.  A gradient's terms: a share 33,
1 - s 9, loads and g / n 4, the sum of f p 33 + 24, four products: 110 of the terms' size.
"""
import math

import pytest

torch = pytest.importorskip("torch")

import mx_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SHARE, GRAD = 40 * U, 110 * U


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _balance(x, idx, sigmoid, seq):
    """Slots, live tokens and mean scores, and the gradient of ones."""
    from paper_2607_26444_amd import moe
    T, E = x.shape
    S = T // seq
    count = torch.empty(S, E, dtype=torch.int32, device="cuda")
    live = torch.empty(S, dtype=torch.int32, device="cuda")
    mean, loss = torch.empty(S, E, device="cuda"), torch.empty(S, device="cuda")
    need = moe.moe_balance_workspace_bytes(T, E, seq)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    dtype = moe.MOE_DTYPE_F32 if x.dtype == torch.float32 else moe.MOE_DTYPE_BF16
    dx = x.cuda()
    moe.moe_balance(dx, dtype, E, idx.int().cuda(), None, count, live, mean, loss, ws,
                    score=int(sigmoid), seq_len=seq)
    grad = torch.empty_like(dx)
    moe.moe_balance_backward(dx, dtype, T, E, None, count, live, torch.ones(S, device="cuda"), None,
                             grad, score=int(sigmoid), seq_len=seq)
    torch.cuda.synchronize()
    return count.cpu(), live.cpu(), mean.cpu().double(), loss.cpu().double(), grad.cpu().double()


def _logits(T, E, lo, hi, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    x = torch.randint(64 * lo, 64 * hi + 1, (T, E), generator=g).float() / 64
    return x, torch.randint(0, E, (T, min(4, E)), generator=g)


# down to where a share of float32 has its lowest normal numbers, and where 1 - s has lost s
@pytest.mark.parametrize("E", [2, 16, 60, 256, 890])
@pytest.mark.parametrize("sigmoid,lo,hi", [(False, -40, 40), (True, -40, 40), (True, -62, -2),
                                           (False, -62, 0), (True, 2, 30)])
def test_shares_of_far_logits(E, sigmoid, lo, hi):
    T = 150
    x, idx = _logits(T, E, lo, hi, E)
    _, _, mean, loss, _ = _balance(x, idx, sigmoid, 1)
    want = ref.shares(x.double(), None, sigmoid)
    assert torch.all((mean - want).abs() <= SHARE * want)
    count, live, _, wl = ref.balance(x.double(), idx, None, sigmoid, 1)
    assert torch.all((loss - wl).abs() <= (SHARE + 20 * U) * wl)


@pytest.mark.parametrize("E", [2, 60, 890])
@pytest.mark.parametrize("sigmoid,lo,hi", [(False, -40, 40), (True, -40, 40), (True, -62, -2)])
def test_gradients_of_far_logits(E, sigmoid, lo, hi):
    T, seq = 120, 4
    x, idx = _logits(T, E, lo, hi, E + 1)
    count, live, _, _, grad = _balance(x, idx, sigmoid, seq)
    # by the formula: automatic differentiation takes 1 - s from s, which loses it near 1
    rest = torch.sigmoid(-x.double()) if sigmoid else torch.ones(T, E, dtype=torch.float64)
    p = ref.shares(x.double(), None, sigmoid).view(-1, seq, E)
    f = (count.double() * E / count.sum(1, keepdim=True))[:, None]
    dot, part = (f * p).sum(2, keepdim=True), p * rest.view(p.shape) / seq
    want, size = (part * (f - dot)).view(T, E), (part * (f + dot)).view(T, E)
    assert torch.all((grad - want).abs() <= GRAD * size + 2.0 ** -126)


@pytest.mark.parametrize("E", [3, 60, 256, 890])
@pytest.mark.parametrize("lo,hi", [(-90, -90), (-100, -88), (-91, -86), (-50, -28), (-140, -60)])
def test_sigmoid_scores_that_are_very_small(E, lo, hi):
    """Scores below float32's normal range whose sum is not give shares all the same, beside tokens
    of ordinary logits; only where the sum is below as well there are none."""
    T, seq = 130, 2
    x, idx = _logits(T, E, lo, hi, E - lo)
    x[::5] = _logits(T, E, -4, 4, 1)[0][::5]
    x[7, E // 2], x[9, 0] = -math.inf, math.nan
    x[11:14] = -math.inf
    total = torch.sigmoid(x.double()).masked_fill(~(x > -math.inf), 0.0).sum(1)
    least = 2.0 ** -126
    clear = ((total - least).abs() > 1e-4 * least).view(-1, seq).all(1)   # of the border
    p = ref.shares(x.double(), None, True) * (total >= least)[:, None]
    count, live, mean, loss, grad = _balance(x, idx, True, seq)
    want = p.view(-1, seq, E).mean(1)
    # two terms and a division more; a share below 2^-100 may be lost
    tol = (SHARE + 2 * U) * want + 2.0 ** -100
    assert torch.all(((mean - want).abs() <= tol)[clear])
    f = count.double() * E / count.sum(1, keepdim=True)
    wl = (f * want).sum(1)
    assert torch.all(((loss - wl).abs() <= (SHARE + 20 * U) * wl)[clear])
    p, f = p.view(-1, seq, E), f[:, None]
    dot, part = (f * p).sum(2, keepdim=True), p * torch.sigmoid(-x.double()).nan_to_num(1.0).view(p.shape) / seq
    want, size = (part * (f - dot)), part * (f + dot)
    off = (grad.view(-1, seq, E) - want).abs() <= GRAD * size + E * 2.0 ** -100
    assert torch.all(off[clear])


@pytest.mark.parametrize("E", [3, 60, 890])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_infinite_logits(E, sigmoid):
    """Infinite ones share alike under softmax, also beside float32's largest number, and have no
    gradient under sigmoid, nor have logits whose 1 - s is no float32 number."""
    T = 6
    x, idx = _logits(T, E, -4, 4, E)
    x[0, 1], x[1, :2], x[2, 2] = math.inf, math.inf, 3.4028234663852886e38
    x[3, 1], x[3, 2] = math.inf, 3.4028234663852886e38
    x[4, 0] = 200.0
    _, _, mean, loss, grad = _balance(x, idx, sigmoid, 1)
    assert torch.all(torch.isfinite(grad)) and torch.all(torch.isfinite(loss))
    if not sigmoid:
        for t, at in ((0, [1]), (1, [0, 1]), (2, [2]), (3, [1]), (4, [0])):
            want = torch.zeros(E, dtype=torch.float64)
            want[at] = 1.0 / len(at)
            assert torch.equal(mean[t], want), t
        return
    want = ref.shares(x.double(), None, True)
    want[3] = torch.sigmoid(x[3].double()) / torch.sigmoid(x[3].double()).sum()
    ok = ~torch.isnan(want)
    assert torch.all(((mean - want).abs() <= SHARE * want)[ok])
    assert not grad[x >= 150].any()
