"""The host's choice of a product's kernel (rapid_linear8.hip: by_dots, plan_for and what they read), compiled alone with g++, so that a
test can say which tile and how many pieces along K a size is taken in."""
import ctypes
import os
import re
import subprocess

from paper_2509_22323_amd import build

TILES = ("64x64", "128x128", "256x128", "256x160", "256x192", "256x256")


def load(folder):
    """plan(M, N, K) -> ("dots" or a tile of TILES, pieces)"""
    text = open(os.path.join(build.HERE, "csrc", "rapid_linear8.hip")).read()

    def part(pattern):
        found = re.findall(pattern, text, re.S | re.M)
        assert len(found) == 1, (pattern, len(found))
        return found[0]

    constants = [part(rf"^constexpr int {name} = [^;]*;") for name in ("STEP", "CUS", "MOST_PIECES")]
    src, out = os.path.join(str(folder), "plan.cpp"), os.path.join(str(folder), "plan.so")
    with open(src, "w") as f:
        f.write("\n".join(["#include <math.h>", *constants, part(r"^bool by_dots\([^\n]*\}$"), part(r"^enum Tile \{.*?^Plan plan_for\(.*?^\}$"),
                           'extern "C" int plan(long long M, int N, int K, int* pieces)',
                           "{ *pieces = 0; if (by_dots(M, N, K)) return -1; const Plan p = plan_for(M, N, K, MOST_PIECES);",
                           "  *pieces = p.pieces; return p.tile; }", ""]))
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-fPIC", "-shared", "-o", out, src], check=True, capture_output=True, text=True)
    lib = ctypes.CDLL(out)
    lib.plan.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_int)]

    def plan(M, N, K):
        pieces = ctypes.c_int()
        tile = lib.plan(M, N, K, ctypes.byref(pieces))
        return ("dots" if tile < 0 else TILES[tile]), pieces.value
    return plan


# B, n, K, N and what they are taken in: every tile, of one sample and straddling samples, with loops that begin at another step on every
# XCD (K a multiple of 128, eight steps or more), that end inside a step and that are short; odd widths; every number of pieces
PRODUCTS = [
    (1, 4100, 1024, 456, "128x128", 1), (7, 700, 208, 584, "128x128", 1), (1, 4100, 528, 1289, "128x128", 1),
    (1, 9000, 2048, 392, "256x128", 1), (3, 1367, 1168, 904, "256x128", 1), (3, 1367, 2048, 904, "256x128", 1),
    (1, 26500, 208, 264, "256x160", 1), (7, 1100, 208, 1033, "256x160", 1), (3, 1367, 1024, 1929, "256x160", 1),
    (1, 6000, 640, 1288, "256x192", 1), (7, 1100, 208, 1032, "256x192", 1), (3, 1367, 1024, 1928, "256x192", 1),
    (1, 4100, 640, 2953, "256x256", 1), (7, 1100, 640, 1544, "256x256", 1), (7, 1100, 1024, 1544, "256x256", 1), (7, 1100, 1168, 1545, "256x256", 1),
    (5, 13, 2432, 2752, "64x64", 2), (1, 12, 1296, 32, "64x64", 3), (1, 12, 1536, 32, "64x64", 4), (1, 12, 2048, 32, "64x64", 5), (1, 12, 2432, 32, "64x64", 6),
    (1, 12, 4096, 2056, "64x64", 7), (1, 12, 4096, 32, "64x64", 8),
    (1, 700, 4096, 1800, "128x128", 2), (1, 700, 4096, 1480, "128x128", 3), (3, 66, 4096, 2104, "128x128", 4), (1, 130, 4096, 2696, "128x128", 5),
    (1, 130, 5632, 2104, "128x128", 6), (5, 13, 4096, 2696, "128x128", 7), (5, 13, 5632, 2120, "128x128", 8),
]
