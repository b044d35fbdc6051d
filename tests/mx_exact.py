"""Products of 4-bit floats whose sums float32 holds however deep they are, so that the outputs have
to be equal, and the sizes at which that is asked (torch, no code of the package).

Rows have any codes, weights those of 0, 0.5 and 1 and their negatives, scales are 1 or 2: products
are multiples of a quarter and at most 24, that is 96 of them.  131040 products, the deepest that a
call may have, add up to 12.6 million quarters in size, less than 2^24, whatever their order.
"""
import math
import os
import subprocess

import torch

import matmul_rule
import mx_rule
from paper_2607_26444_amd import build

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def scale_cols(K):
    return -(-K // 128) * 4


def _codes(g, shape, K, few, one):
    """Codes [*shape, K/2] and scale bytes `one` or `one` + 1; what fills a row of scales is 255."""
    dev = g.device
    if few:
        table = torch.tensor([0, 1, 2, 8, 9, 10], dtype=torch.uint8, device=dev)
        pair = (table[:, None] | table << 4).reshape(-1)
        q = pair[torch.randint(0, 36, (*shape, K // 2), generator=g, device=dev, dtype=torch.int32)]
    else:
        q = torch.randint(0, 256, (*shape, K // 2), generator=g, device=dev, dtype=torch.uint8)
    s = torch.full((*shape, scale_cols(K)), 255, dtype=torch.uint8, device=dev)
    s[..., :K // 32] = torch.randint(one, one + 2, (*shape, K // 32), generator=g, device=dev,
                                     dtype=torch.uint8)
    return q, s


def inputs(rows, E, N, K, seed, swiglu, device="cuda"):
    """Rows and weights; with swiglu the weights' scales are smaller by a power of two that makes
    gates of about 1.5 in size."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    down = round(math.log2(4.7 * math.sqrt(K) / 1.5)) if swiglu else 0
    return _codes(g, (rows,), K, False, 127), _codes(g, (E, N), K, True, 127 - down)


def decode(q, s, K):
    """Values in double, on the codes' device."""
    one = torch.tensor(MAGNITUDES, dtype=torch.float64, device=q.device)
    one = torch.cat([one, -one])
    n = torch.arange(256, device=q.device)
    v = torch.stack([one[n & 15], one[n >> 4]], 1)[q.int()].flatten(-2)
    two = torch.exp2(s[..., :K // 32].double() - 127)
    return (v.view(*two.shape, 32) * two[..., None]).view(*q.shape[:-1], K)


def product(a, w, K):
    """Rows by channels in double, exact; in pieces, since a library's product of operands of more
    than a gigabyte has been wrong, and so have large tables been refused."""
    v = torch.zeros(a[0].shape[0], w[0].shape[0], dtype=torch.float64, device=a[0].device)
    for k in range(0, K, 4096):
        end = min(K, k + 4096)
        depth = slice(k // 2, end // 2), slice(k // 32, end // 32)
        rows = decode(a[0][:, depth[0]], a[1][:, depth[1]], end - k)
        for c in range(0, v.shape[1], 4096):
            n = slice(c, c + 4096)
            v[:, n] += rows @ decode(w[0][n, depth[0]], w[1][n, depth[1]], end - k).T.contiguous()
    return v


def check(y, a, w, windows, swiglu, K):
    """Rows y [rows,out] against the windows' products; those of no window hold NaN.

    Plain outputs are equal.  With swiglu gate and up are exact, exp and reciprocal add |g| + 3 units
    of 2^-23 and the product one, before the rounding to bf16."""
    used = torch.zeros(y.shape[0], dtype=torch.bool, device=y.device)
    out = y.shape[1]
    for e, (at, n) in enumerate(windows):
        if not n:
            continue
        used[at:at + n] = True
        v = product([t[at:at + n] for t in a], [t[e] for t in w], K)
        got = y[at:at + n]
        if not swiglu:
            assert torch.equal(got, v.float().bfloat16()), e     # v is a float32 number
            continue
        g, u = v[:, :out], v[:, out:]
        v, off = g * torch.sigmoid(g) * u, (g.abs() + 4) * 2.0 ** -23
        assert torch.all((got.double() - v).abs() <= (2.0 ** -8 + 1.01 * off) * v.abs()), e
    assert torch.all(torch.isnan(y[~used]))


def packed(counts):
    """(offsets, [(first row, rows)]) of windows one after another."""
    offset = [0]
    for n in counts:
        offset.append(offset[-1] + n)
    return offset, list(zip(offset, counts))


# (way, rows of the windows, N, K) with and without swiglu.
DEEP = [("one_row", [12], 48, 131040), ("one_row", [1], 2064, 131040),
        ("few_rows", [33, 0, 16, 60, 1, 17, 3, 50], 1040, 131040), ("narrow", [2000], 144, 131040),
        ("narrow", [100, 0, 65, 165], 1040, 8224), ("half", [1300], 2064, 131040),
        ("half", [200, 300, 0, 200], 2064, 131040), ("half_two", [129, 321, 0, 250], 2064, 65568),
        ("wide", [0, 64, 65, 128, 129, 1, 63, 250] * 2, 2064, 16416),
        ("tile128", [1400, 0, 2471, 129], 1040, 131040), ("tile256", [1500, 0, 2300, 200], 2064, 131040),
        ("tile256", [4000], 2064, 65568)]


def _ragged(E, rows, longest):
    """Windows of `rows` rows together: every third empty, one of them the longest."""
    counts = [0 if e % 3 == 1 else 1 + (7 * e) % 23 for e in range(E)]
    counts[E // 2] = longest
    counts[-1] += max(0, rows - sum(counts))
    while sum(counts) > rows:
        e = max((e for e in range(E) if e != E // 2), key=lambda e: counts[e])
        counts[e] -= min(counts[e], sum(counts) - rows)
    return counts


# Calls whose weights are read past the caches, every streaming way; windows of more than one of
# their tiles among them: (way, windows, N, K).
READ_ONCE = [("wide", _ragged(32, 512, 70), 7168, 2048), ("wide", _ragged(32, 512, 130), 4096, 7168),
             ("wide", _ragged(32, 64, 20), 4112, 2304), ("half", _ragged(32, 512, 70), 1040, 8448),
             ("half_two", _ragged(32, 512, 129), 2064, 7168), ("narrow", _ragged(48, 700, 65), 272, 33024),
             ("few_rows", _ragged(16, 200, 33), 2064, 8448), ("few_rows", _ragged(16, 40, 17), 1040, 16640),
             ("one_row", _ragged(16, 40, 17), 1040, 33024), ("one_row", _ragged(16, 5, 2), 1040, 16640)]

# On either side of the conditions: (rows, E, N, K, whether the weights are read past the caches).
BORDERS = [(512, 32, 4096, 2048, 1), (513, 32, 4096, 2048, 0), (512, 32, 4088, 2048, 0),
           (512, 32, 4112, 2080, 0), (512, 32, 4112, 2304, 1), (16, 1, 131072, 2048, 1),
           (17, 1, 131072, 2048, 0)]

PROGRAM = mx_rule.PROGRAM.replace(r'std::printf("%d %.3f\n", way, ',
                                  r'std::printf("%d %d %.3f\n", way, (int)moe::weights_read_once(a), ')
assert PROGRAM != mx_rule.PROGRAM


def build_rule(folder):
    """f([(rows, E, N, K, swiglu)] of calls with windows) -> [(way, whether weights are read once)]"""
    src, exe = os.path.join(folder, "once.hip"), os.path.join(folder, "once")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run([build.hipcc(), *build.FLAGS, src, "-o", exe], check=True)

    def choose(calls):
        lines = "".join(f"{rows} {E} {N} {K // 2} {int(swiglu)} 1\n" for rows, E, N, K, swiglu in calls)
        out = subprocess.run([exe], input=lines, check=True, capture_output=True, text=True).stdout
        got = [(matmul_rule.WAYS[int(ln.split()[0])], int(ln.split()[1])) for ln in out.splitlines()]
        assert len(got) == len(calls)
        return got
    return choose
