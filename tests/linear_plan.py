"""The host's choice of a product's kernel (rapid_linear.hip: by_dots, plan_for and what they read), compiled alone with g++, so that a
test can say which tile and how many pieces along K a size is taken in."""
import ctypes
import os
import re
import subprocess

from paper_2509_22323_amd import build

TILES = ("64x64", "128x128", "256x128", "256x160", "256x192", "256x256")


def source():
    text = open(os.path.join(build.HERE, "csrc", "rapid_linear.hip")).read()

    def part(pattern):
        found = re.findall(pattern, text, re.S | re.M)
        assert len(found) == 1, (pattern, len(found))
        return found[0]

    constants = [part(rf"^constexpr int {name} = [^;]*;") for name in ("STEP", "CUS", "MOST_PIECES")]
    return "\n".join(["#include <math.h>", *constants, part(r"^bool by_dots\([^\n]*\}$"), part(r"^enum Tile \{.*?^Plan plan_for\(.*?^\}$"),
                      'extern "C" int plan(long long M, int N, int K, int most, int* pieces)',
                      "{ *pieces = 0; if (by_dots(M, N, K)) return -1; const Plan p = plan_for(M, N, K, most ? most : MOST_PIECES);",
                      "  *pieces = p.pieces; return p.tile; }", ""])


def load(folder):
    """plan(M, N, K, most_pieces = all) -> ("dots" or a tile of TILES, pieces)"""
    src, out = os.path.join(str(folder), "plan.cpp"), os.path.join(str(folder), "plan.so")
    open(src, "w").write(source())
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-fPIC", "-shared", "-o", out, src], check=True, capture_output=True, text=True)
    lib = ctypes.CDLL(out)
    lib.plan.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_int)]

    def plan(M, N, K, most=0):
        pieces = ctypes.c_int()
        tile = lib.plan(M, N, K, most, ctypes.byref(pieces))
        return ("dots" if tile < 0 else TILES[tile]), pieces.value
    return plan


# B, n, K, N and what they are taken in: every tile with one sample and with tiles that straddle samples, more items than there is
# room for at a time, K loops that begin at another step on every XCD (K a multiple of 64, eight steps or more) and that end inside a
# step; every number of pieces; inputs and outputs wider than those that the plan's costs were fitted to
PRODUCTS = [
    (1, 50, 512, 64, "64x64", 1), (3, 50, 512, 64, "64x64", 1), (3, 50, 200, 64, "64x64", 1),
    (1, 1500, 640, 1544, "128x128", 1), (7, 700, 512, 3200, "128x128", 1), (1, 11000, 200, 1320, "128x128", 1),
    (1, 11000, 512, 1320, "256x128", 1), (7, 700, 576, 3200, "256x128", 1), (3, 700, 1024, 2000, "256x128", 1),
    (1, 4100, 512, 4096, "256x160", 1), (7, 1500, 512, 1544, "256x160", 1), (1, 4100, 200, 2000, "256x160", 1),
    (1, 4100, 512, 5000, "256x192", 1), (7, 700, 512, 4096, "256x192", 1), (7, 2049, 200, 1320, "256x192", 1),
    (1, 4100, 512, 6144, "256x256", 1), (7, 700, 512, 5000, "256x256", 1), (1, 11000, 200, 1000, "256x256", 1),
    (1, 512, 1536, 896, "64x64", 2), (4, 4, 576, 64, "64x64", 3), (1, 16, 768, 64, "64x64", 4), (16, 1, 1024, 64, "64x64", 5),
    (3, 100, 1536, 448, "64x64", 6), (1, 300, 1536, 320, "64x64", 7), (2, 8, 1536, 64, "64x64", 8),
    (1, 1000, 2048, 1344, "128x128", 2), (5, 200, 2048, 1088, "128x128", 3), (1, 700, 2048, 960, "128x128", 4), (7, 100, 2048, 768, "128x128", 5),
    (1, 700, 2432, 704, "128x128", 6), (7, 100, 4096, 704, "128x128", 7), (1, 700, 4096, 448, "128x128", 8),
    (1, 333, 12288, 2560, "", 0), (2, 350, 512, 15360, "", 0), (3, 100, 256, 21504, "", 0), (1, 40, 21504, 72, "", 0), (2, 1, 15360, 12288, "dots", 0),
]
