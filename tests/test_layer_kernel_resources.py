"""Host-side guard on what the compiler made of the kernels around the attention: no scratch memory, hardly a scalar register in lanes of
a vector register inside the loops of the products, and the occupancy and LDS that the products' launches count on.  No GPU needed."""
import os
import re
import subprocess

import pytest

from paper_2509_22323_amd import build

KEYS = {"VGPRs": r" VGPRs: (\d+)", "scratch": r"ScratchSize \[bytes/lane\]: (\d+)", "waves": r"Occupancy \[waves/SIMD\]: (\d+)",
        "SGPRs spilled": r"SGPRs Spill: (\d+)", "VGPRs spilled": r"VGPRs Spill: (\d+)", "LDS": r"LDS Size \[bytes/block\]: (\d+)"}
# wavefront rows and fragments of a tile, in pieces along K or not
WIDE = [(1, 2, 1), (2, 4, 1), (1, 2, 0), (2, 4, 0), (4, 4, 0), (4, 5, 0), (4, 6, 0), (4, 8, 0)]


def kernel(WR, FN, split):
    return f"linear_wide_kernelILi{WR}ELi{FN}ELb{split}E"


def source(name):
    found, = [s for s in build.SOURCES if os.path.basename(s) == name]
    return found


@pytest.fixture(scope="module")
def usage(tmp_path_factory):
    cmd = [build.HIPCC] + build.FLAGS + ["-Rpass-analysis=kernel-resource-usage", "-o", str(tmp_path_factory.mktemp("res") / "x.so"),
                                         source("rapid_linear.hip"), source("rapid_layer.hip")]
    text = subprocess.run(cmd, capture_output=True, text=True, check=True).stderr
    return {part.split()[0]: {k: int(re.search(p, part)[1]) for k, p in KEYS.items()} for part in text.split("Function Name: ")[1:]}


@pytest.fixture(scope="module")
def loops(tmp_path_factory):
    """The instructions of every kernel's innermost loop with matrix instructions: a step of a product."""
    out = tmp_path_factory.mktemp("asm") / "x.s"
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([build.HIPCC] + flags + ["--offload-device-only", "-S", "-o", str(out), source("rapid_linear.hip")], capture_output=True, check=True)
    steps, lines, at, labels = {}, [], None, {}
    for line in out.read_text().splitlines():
        name = re.match(r"(_ZN\w+):", line)
        if name:
            at, lines, labels = name[1], [], {}
        label = re.match(r"(\.LBB\w+):", line)
        if label:
            labels[label[1]] = len(lines)
        if re.match(r"\t[sv]_|\t(buffer|global|flat|ds)_", line):
            lines.append(line.strip())
            back = re.match(r"s_c?branch\w*\s+(\.LBB\w+)", lines[-1])
            if back and back[1] in labels:
                loop = lines[labels[back[1]]:]
                if any(i.startswith("v_mfma") for i in loop) and len(loop) < len(steps.get(at, lines + [0])):
                    steps[at] = loop
    return steps


def test_every_kernel_stays_in_registers(usage):
    assert len(usage) == 30, sorted(usage)
    bad = {k: u for k, u in usage.items() if u["scratch"] or u["VGPRs spilled"] or (u["SGPRs spilled"] and "linear_wide_kernel" not in k)}
    assert not bad, bad


@pytest.mark.parametrize("form", WIDE, ids=str)
def test_as_many_workgroups_of_a_product_as_a_launch_counts_on(usage, form):
    """(4 / WR of 2 WR wavefronts a CU: rapid_linear.hip, launch_wide)"""
    name, = [k for k in usage if kernel(*form) in k]
    u, WR = usage[name], form[0]
    assert u["waves"] * 4 >= 4 // WR * 2 * WR and u["LDS"] * (4 // WR) <= 160 * 1024, u


def test_every_product_is_listed(usage):
    assert sum("linear_wide_kernel" in k for k in usage) == len(WIDE)


@pytest.mark.parametrize("form", WIDE, ids=str)
def test_steps_of_a_product_keep_their_scalars(loops, form):
    """A step is 8 FN matrix instructions; no scalar register is written to a lane in it and FN + 1 at most are read back (0, 0, 0, 0,
    1, 2, 7 and 8 when this was written)."""
    loop, = [v for k, v in loops.items() if kernel(*form) in k]
    FN = form[1]
    assert sum(i.startswith("v_mfma") for i in loop) == 8 * FN
    assert sum(i.startswith("v_writelane") for i in loop) == 0 and sum(i.startswith("v_readlane") for i in loop) <= FN + 1
