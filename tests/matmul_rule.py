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
