"""The launch rule of moe_expert_matmul (csrc/matmul_rule.h), compiled into a small
host program: which way each size takes."""
import os
import subprocess

from paper_2607_26444_amd import build

WAYS = ("tile256", "tile128", "wide", "half", "half_two", "narrow", "few_rows", "one_row")
# rows and channels of a way's tile
TILE = dict(tile256=(256, 256), tile128=(128, 256), wide=(64, 128), half=(64, 64),
            half_two=(64, 64), narrow=(64, 32), few_rows=(16, 32), one_row=(16, 16))

PROGRAM = r"""
#include <cstdio>
#include "matmul_rule.h"
int main() {
  long long rows;
  int E, N, K, swiglu, windows;
  static const int32_t offset[1] = {0};
  while (std::scanf("%lld %d %d %d %d %d", &rows, &E, &N, &K, &swiglu, &windows) == 6) {
    moe::MatmulArgs a = {};
    a.rows = rows;
    a.E = E;
    a.N = N;
    a.K = K;
    a.swiglu = swiglu;
    a.offset = windows ? offset : nullptr;
    const int way = moe::choose_way(a);
    std::printf("%d %.3f\n", way, moe::way_time(a, moe::kWay[way]));
  }
}
"""


def build_rule(folder):
    src, exe = os.path.join(folder, "rule.hip"), os.path.join(folder, "rule")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run([build.hipcc(), *build.FLAGS, src, "-o", exe], check=True)

    def choose(calls):
        """[(rows, E, N, K, swiglu, windows)] -> [way]"""
        lines = "".join(" ".join(str(int(v)) for v in c) + "\n" for c in calls)
        out = subprocess.run([exe], input=lines, check=True, capture_output=True, text=True).stdout
        ways = [WAYS[int(ln.split()[0])] for ln in out.splitlines()]
        assert len(ways) == len(calls)
        return ways
    return choose


# One size at least of every way: (way, rows of the windows, capacity or 0 for packed
# windows, N, K).  Windows of no rows, of one, of one to four row tiles of 16, of two tiles; N ends
# inside a tile and K inside a stage, or is shorter than one.  With swiglu N is the
# multiple of 16 below.
_MIXED = [0, 1, 17, 33, 49, 64, 65, 129]
_TALL = [0, 1, 64, 65, 127, 128, 129, 300]
CASES = [
    ("tile256", [257, 0, 1, 256, 1000, 65, 1120, 1400] * 2, 0, 1032, 1040),
    ("tile256", [500, 0, 129, 1000], 1000, 2072, 144),
    ("tile128", _TALL * 8, 0, 2072, 400),
    ("tile128", _TALL * 3, 0, 4120, 144),
    ("tile128", [0, 1, 65, 128, 130, 64] * 8, 130, 2072, 144),
    ("wide", _MIXED * 3, 0, 1560, 1040),
    ("wide", [3, 0, 64, 65] * 4, 0, 4120, 112),
    ("wide", [0, 1, 17, 33, 49, 64] * 4, 64, 1560, 1040),
    ("half", [0, 1, 17, 33, 49, 65], 0, 2072, 144),
    ("half", [100], 0, 4120, 400),
    ("half", [64, 0, 33], 64, 2072, 400),
    ("half_two", [40, 0, 129, 100, 65, 150] * 2, 0, 1032, 400),
    ("half_two", [64, 0, 65, 129, 80, 33, 90, 70] * 4, 0, 520, 1040),
    ("half_two", [0, 5, 100, 64] * 3, 100, 1032, 400),
    ("narrow", [1, 33, 65, 17], 0, 1032, 1040),
    ("narrow", [64, 0, 49, 1], 64, 520, 2064),
    ("few_rows", [1, 0, 15, 16, 17, 9], 0, 1032, 400),
    ("few_rows", [12, 0, 3], 12, 2072, 400),
    ("one_row", [1, 0, 16, 17], 0, 520, 1040),
    ("one_row", [1], 0, 1560, 4112),
    ("one_row", [8, 0, 3, 1], 8, 520, 1040),
]


def call_of(case, swiglu):
    """The call that a case of CASES makes, as build_rule's function takes it."""
    _, counts, cap, N, K = case
    rows = len(counts) * cap if cap else sum(counts)
    return rows, len(counts), N // 16 * 16 if swiglu else N, K, swiglu, 1


# Calls whose weights, rows or outputs pass 2^32 bytes: (way, rows, E, N, K), packed windows.
PAST_32_BITS = [("few_rows", 64, 34, 2048, 65536), ("wide", 16, 34, 2048, 65536),
                ("tile128", 3400, 34, 2048, 65536), ("narrow", 70000, 1000, 8, 65536),
                ("tile128", 70000, 1000, 264, 65536), ("wide", 70000, 1000, 32768, 64),
                ("tile256", 70000, 300, 32768, 64)]
