"""Where the selection of dma_cache4_decode takes its sample: csrc/cache4_sample.h, compiled for the host."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2508_02124_b200", "csrc")


@pytest.fixture(scope="module")
def places(tmp_path_factory):
    at = tmp_path_factory.mktemp("sample")
    (at / "s.cpp").write_text('#include <cstdint>\n#include "cache4_sample.h"\n'
                              'extern "C" void places(uint32_t n, uint32_t groups, uint32_t* out) { for (uint32_t i = 0; i < groups; ++i) out[i] = dma::sample_quad(i, n / 4, groups); }\n')
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", str(at / "s.so"), str(at / "s.cpp")])
    f = ctypes.CDLL(str(at / "s.so")).places

    def run(n, groups):
        out = np.zeros(groups, np.uint32)
        f(ctypes.c_uint32(n), ctypes.c_uint32(groups), out.ctypes.data_as(ctypes.c_void_p))
        return out.astype(np.int64)
    return run


@pytest.mark.parametrize("groups", [512, 1024])
@pytest.mark.parametrize("n", [4097, 5000, 16384, 70001, 1 << 20, (1 << 27) - 1, 1 << 27, (1 << 28) + 5, 1 << 29, 1 << 30])
def test_the_sample_is_spread_over_the_row(places, n, groups):
    """A row's quads (four neighbouring keys) are cut into as many strata as the sample has groups, and each stratum has one, anywhere in it: rows of every length alike."""
    quads = n // 4
    at, first = places(n, groups), np.arange(groups) * quads // groups
    step = quads // groups
    off = at - first
    assert (off >= 0).all() and (off < max(step, 1)).all() and at.max() < quads
    if step >= 64:                                                         # every eighth of the strata has its share of the places: 64 or 128 of them, 6 standard deviations
        share = np.bincount(off * 8 // step, minlength=8)
        assert (np.abs(share - groups / 8) <= 6 * np.sqrt(groups * 7 / 64)).all()
