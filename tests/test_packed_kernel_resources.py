"""Host-side guard on what the compiler made of the kernels over packed sequences: no scratch memory, the occupancy and LDS that their
launches count on, and hardly a scalar register in lanes of a vector register inside the loops with matrix instructions.  No GPU needed."""
import os
import re
import subprocess

import pytest

from paper_2509_22323_amd import build
from test_layer_kernel_resources import KEYS, WIDE, kernel, source

SOURCES = ("rapid_rows8.hip", "rapid_linear8.hip", "rapid_packed.hip")
PACKED = [(64, 0), (64, 1), (128, 0), (128, 1)]


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    """(what the compiler says of every kernel, the instructions of its innermost loop with matrix instructions; of the attention one with
    exponents)"""
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    usage, loops = {}, {}
    work = [(name, tmp_path_factory.mktemp("asm") / "x.s") for name in SOURCES]
    runs = [subprocess.Popen([build.HIPCC] + flags + ["--offload-device-only", "-S", "-Rpass-analysis=kernel-resource-usage", "-o", str(out), source(name)],
                             stderr=subprocess.PIPE, text=True) for name, out in work]
    for run, (name, out) in zip(runs, work):
        text = run.communicate()[1]
        assert run.returncode == 0, text
        usage.update({part.split()[0]: {k: int(re.search(p, part)[1]) for k, p in KEYS.items()} for part in text.split("Function Name: ")[1:]})
        lines, at, labels = [], None, {}
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
                    if any(i.startswith("v_mfma") for i in loop) and ("packed" not in at or sum(i.startswith("v_exp") for i in loop) >= 32) and (at not in loops or len(loop) < len(loops[at])):
                        loops[at] = loop
    return usage, loops


def one(found, fragment):
    name, = [k for k in found if fragment in k]
    return found[name]


def test_every_kernel_stays_in_registers(compiled):
    usage, _ = compiled
    bad = {k: u for k, u in usage.items() if u["scratch"] or u["VGPRs spilled"]}
    assert len(usage) >= 40 and not bad, bad


@pytest.mark.parametrize("D,cap", PACKED)
def test_attention_has_the_workgroups_that_it_counts_on(compiled, D, cap):
    u = one(compiled[0], f"packed_tiles_kernelILi{D}ELb{cap}E")
    workgroups = 3 if D == 64 else 2                   # of four wavefronts, one a SIMD; 160 KB of LDS a CU
    assert u["waves"] >= workgroups and u["LDS"] * workgroups <= 160 * 1024, u


@pytest.mark.parametrize("WR,FN,split", WIDE)
def test_products_have_the_workgroups_that_they_count_on(compiled, WR, FN, split):
    u = one(compiled[0], kernel(WR, FN, split))
    workgroups = 4 // WR
    assert u["waves"] * 4 >= workgroups * 2 * WR and u["LDS"] * workgroups <= 160 * 1024, u


@pytest.mark.parametrize("D,cap", PACKED)
def test_the_attention_loop_keeps_scalars_in_scalar_registers(compiled, D, cap):
    loop = one(compiled[1], f"packed_tiles_kernelILi{D}ELb{cap}E")
    assert sum(i.startswith("v_mfma") for i in loop) % (D // 2) == 0           # a tile or two
    assert not [i for i in loop if i.startswith(("v_writelane", "scratch"))] and len([i for i in loop if i.startswith("v_readlane")]) <= 20


@pytest.mark.parametrize("WR,FN,split", WIDE)
def test_steps_of_whole_numbers_keep_scalars_in_scalar_registers(compiled, WR, FN, split):
    """(The loop of 128 x 128 without pieces is one with the way to the next item, which takes and leaves such lanes once an item.)"""
    loop = one(compiled[1], kernel(WR, FN, split))
    most = (4, 34) if (WR, FN, split) == (2, 4, 0) else (0, 1)
    assert len([i for i in loop if i.startswith("v_writelane")]) <= most[0] and len([i for i in loop if i.startswith("v_readlane")]) <= most[1]
