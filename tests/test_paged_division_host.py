"""The library's own multiplier and shift for a division (fast_div of csrc/dit_paged.h, compiled here for the host), at the quotients' edges."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2601_20655_amd import build

HIPCC = build.HIPCC


@pytest.fixture(scope="module")
def fast_div(tmp_path_factory):
    if shutil.which(HIPCC) is None:
        pytest.skip("hipcc not found")
    d = tmp_path_factory.mktemp("division")
    src = d / "division.hip"
    src.write_text('#include "dit_paged.h"\nextern "C" void division(uint32_t d, uint32_t* out) {\n'
                   "  const dit::FastDiv f = dit::fast_div(d);\n  out[0] = f.d, out[1] = f.mul, out[2] = (uint32_t)f.shift;\n}\n")
    so = d / "division.so"
    subprocess.check_call([HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", build.CSRC,
                           str(src), "-o", str(so)])
    f = ctypes.CDLL(str(so)).division

    def call(n):
        out = (ctypes.c_uint32 * 3)()
        f(ctypes.c_uint32(n), out)
        return list(out)

    return call


@pytest.mark.parametrize("d", [1, 2, 3, 5, 7, 48, 60, 64, 100, 641, 1560, 65537, 2 ** 30 - 1, 2 ** 30, 2 ** 30 + 1, 2 ** 31 - 1])
def test_quotients(fast_div, d):
    """n / d by the high half of 2 n times the multiplier (a product of 32 bits each), as div_by has it."""
    of, mul, shift = fast_div(d)
    assert of == d and shift < 32
    rng = np.random.default_rng(d)
    top = (2 ** 31 - 1) // d
    edges = np.concatenate([[0, 1, top], rng.integers(0, top + 1, size=4000)]).astype(np.uint64) * np.uint64(d)
    n = np.concatenate([edges, edges[edges > 0] - np.uint64(1), np.uint64([2 ** 31 - 1, 2 ** 31 - 2]), rng.integers(0, 2 ** 31, size=4000).astype(np.uint64)])
    n = n[n < 2 ** 31]
    # (the product is below 2^64: 2 n and the multiplier are below 2^32)
    got = ((np.uint64(2) * n * np.uint64(mul)) >> np.uint64(32)) >> np.uint64(shift)
    assert np.array_equal(got, n // np.uint64(d))
