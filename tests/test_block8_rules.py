"""Host arithmetic of the 8-bit products: the rule for the tile (csrc/matmul8_rules.h), compiled on its own, and the activations of 8-bit results, with the coefficients
read out of the kernel source.  No GPU needed."""
import ctypes
import math
import os
import re
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def takes_large(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules8")
    (d / "r.cpp").write_text('#include "paper_2206_03382_amd/csrc/matmul8_rules.h"\n'
                             'extern "C" int large(int64_t E, double rows, int64_t K, int64_t N) { return moe::matmul8_takes_large_tile(E, rows, K, N); }\n')
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", ROOT, str(d / "r.cpp"), "-o", str(d / "r.so")], check=True)
    lib = ctypes.CDLL(str(d / "r.so"))
    lib.large.restype, lib.large.argtypes = ctypes.c_int, [ctypes.c_int64, ctypes.c_double, ctypes.c_int64, ctypes.c_int64]
    return lambda E, rows, K, N: bool(lib.large(E, float(rows), K, N))


def test_tile_rule_follows_the_measurements(takes_large):
    """Sides that differ by more than a tenth where both were measured."""
    small = [(8, 256, 2048, 2048), (8, 512, 2048, 2048), (1, 1024, 4096, 4096), (1, 2048, 4096, 4096)]
    large = [(8, 1024, 2048, 2048), (8, 2048, 2048, 2048), (64, 256, 1024, 1024), (64, 1024, 1024, 1024), (1, 4096, 4096, 4096)]
    assert not any(takes_large(*c) for c in small) and all(takes_large(*c) for c in large)


def test_gpu_cases_reach_both_tiles(takes_large):
    from test_block8_gpu import MATMULS
    assert {takes_large(*c) for c in MATMULS} == {True, False}
    assert {takes_large(*c) for c in MATMULS if c[2] > 8192} == {True, False}


def test_tile_rule_at_the_ends(takes_large):
    assert not takes_large(1, 1, 1, 8) and not takes_large(512, 1, 128, 128)
    assert takes_large(1, 1 << 17, 4096, 4096) and takes_large(512, 8192, 8192, 8192)


def coefficients():
    text = open(os.path.join(ROOT, "paper_2206_03382_amd", "csrc", "block8.h")).read()
    return [np.float32(re.search(r"kPhi8C%d = ([-+0-9.e]+)f" % i, text).group(1)) for i in range(1, 8)]


def test_gelu_of_8bit_results():
    """Within 3e-5 of Phi itself where it is fitted, of 1e-14 beyond, plus fp32 roundings; half a step of the format is 6e-2."""
    v = np.concatenate([np.linspace(-8, 8, 320001), [-0.0, 0.0, 1e-30, -1e-30, 30.0, -30.0, 1e4, -1e4, 1e30, -1e30]]).astype(np.float32)
    y = np.abs(v)
    c = coefficients()
    s = np.full_like(y, c[6])
    with np.errstate(over="ignore", under="ignore"):
        for a in c[5::-1]:
            s = (s * y + a).astype(np.float32)
        tail = (np.float32(0.5) * np.exp2(-(s * y).astype(np.float32).astype(np.float64))).astype(np.float32)
        got = (v * np.where(v < 0, tail, np.float32(1) - tail)).astype(np.float64)
        ref = v.astype(np.float64) * np.array([0.5 * math.erfc(-float(a) / math.sqrt(2.0)) for a in v])      # 1 + erf loses what is left of it below -5
    inside = y <= 8
    # relative: the exponent's fit of 4.5e-5, and its fp32 roundings, of numbers below 64, times ln 2
    assert np.all(np.abs(got - ref)[inside] <= (4.5e-5 + 64 * 2.0 ** -22) * np.log(2) * np.abs(ref)[inside] + 1e-30)
    assert np.all(np.abs(got - ref)[~inside] <= 2.0 ** -22 * np.abs(ref)[~inside] + 1e-12)
