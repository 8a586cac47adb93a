"""Registers and shared memory of the operators that make a retained set against their launches,
without a GPU (ptxas's resource report of an sm_103a compile)."""
import os
import re
import sys
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

from paper_2608_27128_gb300 import build as B   # noqa: E402
from test_build_budgets import _one, _report    # noqa: E402

SRCS = ["twk_prompt.cu", "twk_weights.cu", "twk_cache_weights.cu", "twk_weight_policy.cu"]
SM_REGS, SM_SMEM, BLOCK_SMEM = 65536, 228 * 1024, 227 * 1024


@pytest.fixture(scope="module")
def reports():
    with ThreadPoolExecutor(len(SRCS)) as ex:
        return dict(zip(SRCS, ex.map(_report, SRCS)))


def _source(name):
    with open(os.path.join(B.CSRC, name)) as f:
        return f.read()


def _value(src, name):
    """An integer of a line of constants of the source."""
    return int(re.search(rf"\b{name} = (\d+)", _source(src)).group(1))


def _registers(regs, threads):
    """Registers of a block: a warp's are allotted in steps of 256."""
    return (regs * 32 + 255) // 256 * 256 * (threads // 32)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("src,kernel,others,share", [
    ("twk_prompt.cu", "prompt_attend_kernel", 8, "kSoftmaxRegs"),
    ("twk_weights.cu", "prompt_weights_kernel", 16, "kSumRegs")])
def test_warpgroups_trade_what_the_launch_has(reports, d, src, kernel, others, share):
    """The shares after setmaxnreg add up to the launch's: with fewer the second would never come."""
    regs, spill, _ = _one(reports[src], rf"\d{kernel}ILi{d}E")
    launch = _value(src, "kLaunchRegs")
    threads = 32 * (others + 4)
    assert regs == launch and spill <= 16
    assert _registers(regs, threads) <= SM_REGS
    assert 4 * _value(src, "kHelperRegs") + others * _value(src, share) <= launch * (others + 4)
    assert all(x % 8 == 0 for x in (launch, _value(src, "kHelperRegs"), _value(src, share)))


@pytest.mark.parametrize("src", ["twk_prompt.cu", "twk_weights.cu"])
def test_merges_do_not_spill(reports, src):
    hits = {k: v for k, v in reports[src].items() if re.search(r"\dmerge_", k)}
    assert hits and all(spill == 0 for _, spill, _ in hits.values())
    for regs, _, smem in hits.values():               # two blocks an SM at least, rows in passing
        assert 2 * _registers(regs, 256) <= SM_REGS and 2 * (smem + 1024) <= SM_SMEM


@pytest.mark.parametrize("d", [64, 128])
def test_cache_weights_blocks(reports, d):
    for e in (1, 2):
        regs, spill, smem = _one(reports["twk_cache_weights.cu"],
                                 rf"cache_weights_few_kernelILi{d}ELi{e}E")
        warps = _value("twk_cache_weights.cu", "kFewWarps")
        keys = 64 * (d // 2) + 64 * (d // 64) * 4
        rings = 221184 // (warps * keys) * warps * keys
        assert spill == 0 and _registers(regs, 32 * warps) <= SM_REGS
        assert smem + rings + 2049 * 4 <= BLOCK_SMEM
    regs, spill, smem = _one(reports["twk_cache_weights.cu"], rf"cache_weights_kernelILi{d}E")
    assert spill <= 16 and 4 * _registers(regs, 128) <= SM_REGS and 4 * (smem + 1024) <= SM_SMEM


@pytest.mark.parametrize("v,threads,blocks", [(8, 512, 3), (16, 512, 3), (32, 512, 2), (32, 1024, 1)])
def test_policy_blocks(reports, v, threads, blocks):
    """As many blocks as the launch counts on share an SM."""
    regs, spill, smem = _one(reports["twk_weight_policy.cu"],
                             rf"weight_policy_kernelILi{v}ELi{threads}ELi{blocks}E")
    assert spill <= 16 and blocks * _registers(regs, threads) <= SM_REGS
    assert smem + 4 * v * threads <= BLOCK_SMEM
    assert blocks * (smem + 4 * v * threads + 1024) <= SM_SMEM
