"""Scales whose product with log2(e) no float32 holds are refused by the operators that make a retained
set: found on the host, no GPU is needed."""
import numpy as np
import pytest

from paper_2608_27128_gb300 import twinkv as tk
from test_prompt_abi import BIG, FAKE, lib, prompt, seqs  # noqa: F401


def call(lib, what, scale):  # noqa: F811
    # without a workspace: what passes the checks of the arguments stops there
    if what == "attend":
        return lib.twinkv_prompt_attend(FAKE, FAKE, FAKE, prompt(), seqs(), scale, 0, 0, 2 * FAKE, FAKE,
                                        FAKE, None, 0, None)
    if what == "weights":
        return lib.twinkv_prompt_weights(FAKE, FAKE, FAKE, prompt(), seqs(), scale, 0, 0, 0, FAKE, FAKE,
                                         FAKE, None, 0, None)
    return lib.twinkv_cache_weights(FAKE, FAKE, tk.Queries(1, 2, 8, 1, 1024, 1024, 128), scale, 5, 0,
                                    tk.Pool(FAKE, 10, 128), FAKE, 4, FAKE, FAKE, FAKE, 256, None, None, 0,
                                    None)


@pytest.mark.parametrize("what", ["attend", "weights", "cache"])
def test_scales(lib, what):  # noqa: F811
    most = float(np.nextafter(np.float32(2.0 ** 127), np.float32(0)))
    assert np.isfinite(np.float32(most) * np.float32(1.4426950408889634))
    for scale in (2.0 ** 127, 2.5e38, 3.4e38):
        assert call(lib, what, scale) == tk.ERR_INVALID_ARG, scale
    for scale in (most, 1.0, 1e-38, 1e-45):
        assert call(lib, what, scale) == tk.ERR_WORKSPACE, scale
