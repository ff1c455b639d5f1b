"""The bins that logits are counted in (csrc/bins.h), compiled for the CPU: a bin's number is one, however little a row's logits differ, and no logit lies below the edge of its bin."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_03983_amd", "csrc")
SOURCE = """
#include "bins.h"
extern "C" float scale_of(int bins, float span) { return bin_scale(bins, span); }
extern "C" void places(const float *v, int n, float top, float scale, float *out) { for (int i = 0; i < n; ++i) out[i] = (top - v[i]) * scale; }
extern "C" float edge_of(int b, float top, float scale) { return bin_edge(b, top, scale); }
"""


@pytest.fixture(scope="module")
def bins(tmp_path_factory):
    at = tmp_path_factory.mktemp("bins")
    (at / "bins.cpp").write_text(SOURCE)
    (at / "hip").mkdir()
    (at / "hip" / "hip_runtime.h").write_text("#define __host__\n#define __device__\n#define __forceinline__ inline\n")      # all that the header needs of it
    subprocess.run(["g++", "-O1", "-ffp-contract=off", "-shared", "-fPIC", "-I" + str(at), "-I" + CSRC, str(at / "bins.cpp"), "-o", str(at / "bins.so")], check=True)
    lib = ctypes.CDLL(str(at / "bins.so"))
    lib.scale_of.argtypes, lib.scale_of.restype = [ctypes.c_int, ctypes.c_float], ctypes.c_float
    lib.edge_of.argtypes, lib.edge_of.restype = [ctypes.c_int, ctypes.c_float, ctypes.c_float], ctypes.c_float
    lib.places.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_float, ctypes.c_void_p]
    return lib


@pytest.mark.parametrize("n", [256, 1024])
def test_every_logit_has_a_bin(bins, n):
    """Spans from the smallest step of fp32 to half its range, around 0, above it, below it and far from it."""
    rng = np.random.default_rng(1)
    tiny, most = np.float32(2.0 ** -149), np.finfo(np.float32).max
    spans = np.concatenate([np.float32([tiny, 2 * tiny, 1e-40, 1e-38, 1.1754944e-38, 1e-37, 7.4e-37, 7.5e-37, 3e-36, 3.1e-36, 1.0, 3e38]),
                            (2.0 ** rng.uniform(-148, 126, 300)).astype(np.float32)])
    for span in spans:
        scale = bins.scale_of(n, span)
        assert 0 < scale <= most, (span, scale)
        for top in np.float32([0.0, span, span / 2, -span, 1e-37, 1.0, -5.0, 1e30]):
            with np.errstate(over="ignore"):
                v = top - span * np.concatenate([np.float32([0, 1]), rng.random(60, dtype=np.float32)])
            low, v = v[1], v[np.isfinite(v)]
            if not (np.isfinite(low) and np.float32(top - low) > 0):
                continue
            scale = bins.scale_of(n, np.float32(top - low))             # as a row's is formed: from the largest and the smallest
            v = np.clip(v, low, top)
            at = np.empty_like(v)
            bins.places(v.ctypes.data, len(v), top, scale, at.ctypes.data)
            assert (at >= 0).all() and (at < n).all(), (span, top, scale, at.min(), at.max())
            for b in sorted(set(at.astype(int))):
                edge = bins.edge_of(int(b), top, scale)
                assert not (v[at.astype(int) <= b] < edge).any(), (span, top, b, edge)


def test_logits_that_are_all_the_same(bins):
    assert bins.scale_of(256, 0.0) == 0.0 and bins.edge_of(0, 3.5, 0.0) == 3.5
