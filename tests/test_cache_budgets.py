"""Registers and shared memory of the operators around the pass against their launches, and the
layout of a page, without a GPU (ptxas's resource report of an sm_103a compile)."""
import os
import re
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

from paper_2608_27128_gb300 import build as B   # noqa: E402
from test_build_budgets import _one, _report    # noqa: E402

SRCS = ["twk_rope.cu", "twk_cache.cu", "twk_attend.cu"]
QUARTER_REGS, BLOCK_SMEM = 16384, 227 * 1024


@pytest.fixture(scope="module")
def reports():
    with ThreadPoolExecutor(len(SRCS)) as ex:
        return dict(zip(SRCS, ex.map(_report, SRCS)))


def _source(name):
    with open(os.path.join(B.CSRC, name)) as f:
        return f.read()


WARPS = {(64, 4): 16, (64, 8): 16, (64, 16): 8, (128, 4): 12, (128, 8): 12, (128, 16): 8}


def test_warps_are_the_sources():
    """The kernel's own expression, by the compiler."""
    expr = re.search(r"static constexpr int kWarps = ([^;]+);", _source("twk_attend.cu")).group(1)
    code = f"constexpr int w(int D, int R) {{ return {expr}; }}\n" + "".join(
        f"static_assert(w({d}, {r}) == {n}, \"\");\n" for (d, r), n in WARPS.items())
    p = subprocess.run(["g++", "-std=c++17", "-fsyntax-only", "-x", "c++", "-"], input=code,
                       capture_output=True, text=True)
    assert p.returncode == 0, p.stderr


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("r", [4, 8, 16])
def test_attention_block_fits_an_sm(reports, d, r):
    regs, spill, smem = _one(reports["twk_attend.cu"], rf"attend_kernelILi{d}ELi{r}E")
    warps = WARPS[d, r]
    assert warps % 4 == 0                                 # as many on every quarter
    assert (regs * 32 + 255) // 256 * 256 * (warps // 4) <= QUARTER_REGS
    assert spill <= 64
    half = 64 * (d // 2) + 64 * (d // 64) * 4
    ring = 221184 // (2 * half * warps) * 2 * half
    assert ring >= 2 * 2 * half                           # two pages ahead
    assert smem + warps * ring + 4 * 2049 <= BLOCK_SMEM
    assert ring >= 4 * r * (d + 2)                        # the warp's part fits its ring


@pytest.mark.parametrize("kernel", ["pack_kernelI[tf]Li64", "pack_kernelItLi128", "compact_kernelILi64",
                                    "compact_kernelILi128", "read_kernelILi64", "read_kernelILi128",
                                    "append_kernelItLi128", "index_kernel"])
def test_moves_do_not_spill(reports, kernel):
    hits = {k: v for k, v in reports["twk_cache.cu"].items() if re.search(kernel, k)}
    assert hits and all(spill == 0 for _, spill, _ in hits.values())
    assert all(smem <= 48 * 1024 for _, _, smem in hits.values())


@pytest.mark.parametrize("d", [64, 128])
def test_pack_blocks_of_an_sm(reports, d):
    regs, _, smem = _one(reports["twk_cache.cu"], rf"pack_kernelItLi{d}E")
    assert 5 * 8 * ((regs * 32 + 255) // 256 * 256) <= 65536
    assert 5 * (smem + 1024) <= 228 * 1024


def test_rope_does_not_spill(reports):
    hits = {k: v for k, v in reports["twk_rope.cu"].items() if "rope_kernel" in k}
    assert len(hits) == 4 and all(spill == 0 for _, spill, _ in hits.values())
