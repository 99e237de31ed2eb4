"""The generator of dropout (csrc/philox.h), compiled for the host: its numbers, and that nothing reads a seed where nothing is dropped and there need be none.  No GPU needed."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

from oracle import rows_oracle as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2206_03382_amd", "csrc")
SOURCE = r"""
#include "paper_2206_03382_amd/csrc/philox.h"
template <bool DROP> static void numbers(const uint64_t* seed, uint64_t g, uint32_t* out) {
  const moe::Philox rng = DROP ? moe::Philox(seed) : moe::Philox();
  uint32_t w[4];
  rng.bits(g, w);
  for (int i = 0; i < 4; ++i) out[i] = w[i];
}
extern "C" void dropped(const uint64_t* seed, uint64_t g, uint32_t* out) { numbers<true>(seed, g, out); }
extern "C" void kept(const uint64_t* seed, uint64_t g, uint32_t* out) { numbers<false>(seed, g, out); }
"""


@pytest.fixture(scope="module")
def generator(tmp_path_factory):
    d = tmp_path_factory.mktemp("philox")
    (d / "philox.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O0", "-shared", "-fPIC", "-I", ROOT, str(d / "philox.cpp"), "-o", str(d / "philox.so")], check=True)
    lib = ctypes.CDLL(str(d / "philox.so"))
    lib.dropped.argtypes = lib.kept.argtypes = [ctypes.c_void_p, ctypes.c_uint64, ctypes.c_void_p]
    return lib


def test_numbers(generator):
    rng = np.random.default_rng(0)
    out = (ctypes.c_uint32 * 4)()
    for seed, offset, g in [(0, 0, 0), (2 ** 64 - 1, 2 ** 64 - 1, 2 ** 64 - 1)] + [tuple(int(x) for x in rng.integers(0, 2 ** 63, 3)) for _ in range(50)]:
        pair = (ctypes.c_uint64 * 2)(seed, offset)
        generator.dropped(pair, g, out)
        word = 0xFFFFFFFF
        assert list(out) == O.philox((seed & word, seed >> 32), (g & word, g >> 32, offset & word, offset >> 32))


def test_no_seed_is_read_where_nothing_is_dropped(generator):
    out = (ctypes.c_uint32 * 4)()
    generator.kept(None, 5, out)                                    # would end the process
    text = open(os.path.join(CSRC, "rows.hip")).read()
    made = re.findall(r"const Philox rng = ([^;]*);", text)
    assert made and set(made) == {"DROP ? Philox(seed) : Philox()"}
