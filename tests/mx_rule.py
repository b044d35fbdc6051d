"""The launch rule of moe_expert_matmul_mx (csrc/matmul_rule.h), compiled into a small host
program: which way each size takes."""
import os
import subprocess

import matmul_rule
from paper_2607_26444_amd import build

WAYS, TILE = matmul_rule.WAYS, matmul_rule.TILE
PROGRAM = matmul_rule.PROGRAM.replace("choose_way", "choose_mx_way").replace("kWay[", "kMxWay[")


def build_rule(folder):
    src, exe = os.path.join(folder, "rule.hip"), os.path.join(folder, "rule")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run([build.hipcc(), *build.FLAGS, src, "-o", exe], check=True)

    def choose(calls):
        """[(rows, E, N, K, swiglu, windows)] -> [way]"""
        lines = "".join(f"{rows} {E} {N} {K // 2} {int(swiglu)} {int(windows)}\n"
                        for rows, E, N, K, swiglu, windows in calls)
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
    ("tile256", [257, 0, 1, 256, 1000, 65, 1120, 1400] * 2, 0, 1032, 2080),
    ("tile256", [500, 0, 129, 1000], 1000, 2072, 96),
    ("tile256", [257, 0, 1, 256, 1000, 65, 1120, 1400] * 2, 0, 1032, 160),
    ("tile128", _TALL * 8, 0, 1560, 800),
    ("tile128", _TALL * 3, 0, 2072, 96),
    ("tile128", [64, 0, 65, 129, 80, 33, 90, 70] * 4, 0, 1560, 2080),
    ("wide", _MIXED * 3, 0, 2072, 160),
    ("wide", [3, 0, 64, 65] * 4, 0, 2072, 2080),
    ("wide", [0, 1, 17, 33, 49, 64] * 4, 64, 1032, 1056),
    ("half", _MIXED * 3, 0, 264, 416),
    ("half", [100], 0, 4120, 1056),
    ("half", [64, 0, 33], 64, 2072, 2080),
    ("half_two", _MIXED * 3, 0, 1032, 800),
    ("half_two", [3, 0, 64, 65] * 4, 0, 4120, 4128),
    ("half_two", [0, 5, 100, 64] * 3, 100, 1032, 800),
    ("narrow", [40, 0, 129, 100, 65, 150] * 2, 0, 264, 2080),
    ("narrow", [64, 0, 49, 1], 64, 1032, 8224),
    ("few_rows", [1, 0, 15, 16, 17, 9], 0, 1032, 416),
    ("few_rows", [64, 0, 33], 64, 520, 160),
    ("few_rows", [12, 0, 3], 12, 4120, 4128),
    ("one_row", [1, 0, 16, 17], 0, 520, 2080),
    ("one_row", [1], 0, 2072, 8224),
    ("one_row", [8, 0, 3, 1], 8, 520, 1056),
]
call_of = matmul_rule.call_of

# Calls whose weights, rows, outputs or, in one of them, scales pass 2^32 bytes:
# (way, rows, E, N, K), packed windows.
PAST_32_BITS = [("few_rows", 64, 68, 2048, 65536), ("one_row", 16, 1000, 264, 65536),
                ("half", 2200, 68, 2048, 65536), ("half_two", 3400, 68, 2304, 65536),
                ("wide", 20000, 1000, 2200, 65536), ("narrow", 140000, 1000, 8, 65536),
                ("tile128", 70000, 1000, 264, 65536), ("tile128", 70000, 1000, 32768, 128),
                ("tile256", 140000, 16, 264, 65536), ("tile256", 70000, 300, 32768, 128)]
