"""Host arithmetic of the few-token layer (csrc/few_rules.h), compiled on its own.  No GPU needed."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("few_rules")
    (d / "r.cpp").write_text('#include "paper_2206_03382_amd/csrc/few_rules.h"\nextern "C" {\n'
                             "int columns(int64_t T, int64_t units, int64_t width, int bf16) { return moe::few_columns(T, units, width, bf16); }\n"
                             "int planned(int64_t T, int64_t H, int64_t E, int k, int bf16) { return moe::few_planned(T, H, E, k, bf16); }\n}\n")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", ROOT, str(d / "r.cpp"), "-o", str(d / "r.so")], check=True)
    lib = ctypes.CDLL(str(d / "r.so"))
    lib.columns.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int]
    lib.planned.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int] * 2
    return lib


def test_the_plan_is_worked_out_once_where_blocks_do_not_all_run_at_once(rules):
    """By the blocks that are launched, 32 columns wide ones too."""
    for T in (1, 2, 7, 16, 17, 40, 64):
        for E in (1, 2, 8, 32, 64, 128, 512):
            for k in (1, 2, 8):
                if k > E:
                    continue
                for H in (8, 64, 264, 640, 1024, 1152, 2048, 2560, 4096, 16384):
                    for bf16 in (0, 1):
                        units = min(E, T * k)
                        width = rules.columns(T, units, H, bf16)
                        blocks = -(-H // width) * units
                        assert width in (32, 64) and not (bf16 and width == 32)
                        assert bool(rules.planned(T, H, E, k, bf16)) == (blocks > (512 if T <= 16 else 256)), (T, E, k, H, bf16)


def test_narrow_blocks_fill_places_only(rules):
    assert rules.columns(16, 8, 2048, 0) == 32 and rules.columns(16, 32, 1024, 0) == 64 and rules.columns(24, 4, 512, 0) == 32 and rules.columns(64, 16, 4096, 0) == 64
    assert rules.planned(1, 2560, 128, 8, 0) and not rules.planned(1, 2560, 128, 8, 1) and not rules.planned(16, 2048, 8, 2, 0)
