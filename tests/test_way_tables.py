"""The launch rules' tables (csrc/matmul_rule.h), compiled into a small host program: a rule asks
its own table whether a way can be launched."""
import os
import subprocess

import pytest

pytest.importorskip("torch")

from paper_2607_26444_amd import build  # noqa: E402

# A table whose third way has tiles of 16 x 16, takes no time, and for 4 million rows x 1024
# channels would be 16 million workgroups.
PROGRAM = r"""
#include <cstdio>
#include "matmul_rule.h"
int main() {
  moe::Way table[moe::kWays];
  for (int n = 0; n < moe::kWays; ++n) table[n] = moe::kMxWay[n];
  table[moe::kWide] = {16, 16, 128, 1 << 30, 0.0, 0.0, 0.0, 1e30};
  for (long long rows : {1000LL, 4000000LL}) {
    moe::MatmulMxArgs a = {};
    a.rows = rows;
    a.E = 1;
    a.N = 1024;
    a.K = 64;
    const int way = moe::quickest_way(a, table);
    const long long tiles = moe::tiles_of(a, table[way]);
    std::printf("%d %lld %lld\n", way == moe::kWide, tiles, (long long)moe::kMaxGroups);
  }
}
"""


def test_a_way_that_its_own_table_cannot_launch_is_left_out(tmp_path):
    src, exe = os.path.join(tmp_path, "table.hip"), os.path.join(tmp_path, "table")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run([build.hipcc(), *build.FLAGS, src, "-o", exe], check=True)
    out = subprocess.run([exe], check=True, capture_output=True, text=True).stdout
    few, many = [[int(v) for v in ln.split()] for ln in out.splitlines()]
    assert few[0] == 1                       # where it can be launched it is the quickest
    assert many[0] == 0 and many[1] <= 2 ** 31 - 512
