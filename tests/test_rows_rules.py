"""Which kernel the products of experts' rows take (csrc/rows_rules.h, compiled on its own: no GPU needed), and that the cases of the GPU's tests reach every one of them in every layout."""
import ctypes
import os
import subprocess

import pytest

import test_dropless_large_gpu as layers
import test_rows_gpu as small
import test_rows_large_gpu as large

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "paper_2206_03382_amd/csrc/rows_rules.h"
using namespace moe;
static int put(const RowsPlan& p, int* at) { at[0] = (int)p.kernel; at[1] = (int)p.tile; at[2] = p.ri; at[3] = p.parts; return 0; }
extern "C" {
int product(int half, int experts, int64_t E, int64_t R, int64_t K, int64_t N, int64_t gather_rows, int act, int joined, int* at) {
  return put(product_plan(half, experts, E, R, K, N, gather_rows, act, joined), at);
}
int product_nt(int half, int64_t E, int64_t R, int64_t K, int64_t N, int grad, int* at) { return put(product_nt_plan(half, E, R, K, N, grad), at); }
int weight_grad(int half, int64_t E, int64_t R, int64_t K, int64_t N, int64_t gather_rows, int* at) { return put(weight_grad_plan(half, E, R, K, N, gather_rows), at); }
}
"""
KERNELS = ["tile", "thin", "short", "outer", "parts", "fp32", "fp32 split"]
TILES = ["256x256", "128x128", "64x128", "64x64", "64x128 streamed", "64x64 streamed"]


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rows_rules")
    (d / "rules.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", ROOT, str(d / "rules.cpp"), "-o", str(d / "rules.so")], check=True)
    lib = ctypes.CDLL(str(d / "rules.so"))
    i64, i32 = ctypes.c_int64, ctypes.c_int
    lib.product.argtypes = [i32, i32] + [i64] * 5 + [i32, i32, ctypes.c_void_p]
    lib.product_nt.argtypes = [i32] + [i64] * 4 + [i32, ctypes.c_void_p]
    lib.weight_grad.argtypes = [i32] + [i64] * 5 + [ctypes.c_void_p]

    def ask(name, *args):
        at = (i32 * 4)()
        getattr(lib, name)(*[int(a) for a in args], at)
        kernel = KERNELS[at[0]]
        if kernel == "tile":
            return TILES[at[1]]
        return f"thin {at[2]}, {'shared' if at[3] > 1 else 'alone'}" if kernel == "thin" else kernel
    return ask


FORWARD = {"256x256", "128x128", "64x128", "64x64", "64x128 streamed", "64x64 streamed", "thin 1, alone", "thin 1, shared", "thin 2, alone", "thin 2, shared", "thin 4, shared", "short"}
BACK = {"256x256", "128x128", "64x128", "64x64", "64x128 streamed", "64x64 streamed", "short"}
WEIGHTS = {"256x256", "128x128", "outer", "parts"}


def test_cases_reach_every_kernel(rules):
    """Forward: plain and gathered, with what is joined to the sums.  dx: plain and times the derivative.  dW: in place and gathered."""
    seen = {}

    def saw(form, kernel):
        seen.setdefault(form, set()).add(kernel)

    for half in (1, 0):
        for R, E, K, N, _, _ in small.PRODUCTS:
            tokens = max(1, R // 2) if R % 2 else 0
            act = (R + E) % 4 != 0
            saw(("forward", half), rules("product", half, 1, E, R, K, N, tokens, act, act))
            saw(("back", half), rules("product_nt", half, E, R, K, N, 0))
            saw(("weights", half), rules("weight_grad", half, E, R, K, N, tokens))
        for T, K, N in small.LINEAR:
            saw(("forward", half), rules("product", half, 0, 1, T, K, N, 0, (T + K // 8) % 4 != 0, 1))
            saw(("back", half), rules("product_nt", half, 1, T, K, N, 0))
            saw(("weights", half), rules("weight_grad", half, 1, T, K, N, 0))
    for form, got in {**{("forward", c): rules("product", 1, 1, c.E, c.R, c.K, c.N, c.tokens, c.act != "none", c.act != "none") for c in large.FORWARD},
                      **{("dense", c): rules("product", 1, 0, 1, c.R, c.K, c.N, 0, c.act != "none", 1) for c in large.DENSE},
                      **{("back", c): rules("product_nt", 1, c.E, c.R, c.K, c.N, c.act != "none") for c in large.BACK},
                      **{("weights", c): rules("weight_grad", 1, c.E, c.R, c.K, c.N, c.tokens) for c in large.WEIGHTS}}.items():
        c = form[1]
        assert got == c.kernel, (form, got)
        saw(("forward" if form[0] == "dense" else form[0], 1), got)
    assert seen["forward", 1] == FORWARD and seen["back", 1] == BACK and seen["weights", 1] == WEIGHTS
    assert seen["forward", 0] == seen["back", 0] == {"fp32", "fp32 split"} and seen["weights", 0] == {"fp32", "parts"}


def test_large_tile_in_every_form():
    """The 256 x 256 tile has code of its own for every activation, with and without kept values, residual and derivative, in place and gathered."""
    acts = {"none", "relu", "gelu", "silu"}
    of = lambda cases: [c for c in cases if c.kernel == "256x256"]   # noqa: E731
    assert {c.act for c in of(large.FORWARD) if c.tokens} == {c.act for c in of(large.FORWARD) if not c.tokens} == {c.act for c in of(large.DENSE)} == {c.act for c in of(large.BACK)} == acts
    assert {bool(c.tokens) for c in of(large.WEIGHTS)} == {True, False}


def test_a_layer_on_the_large_tile(rules):
    for T, E, k, M, H in layers.LAYERS:
        R = T * k
        assert {rules("product", 1, 1, E, R, M, H, T, 1, 1), rules("product", 1, 1, E, R, H, M, 0, 0, 0), rules("product_nt", 1, E, R, H, M, 1), rules("product_nt", 1, E, R, M, H, 0),
                rules("weight_grad", 1, E, R, M, H, T), rules("weight_grad", 1, E, R, H, M, 0)} == {"256x256"}


def test_rows_of_a_large_token_matrix(rules):
    """32-bit offsets reach 4 GiB of gathered rows; beyond, the tiles with addresses of their own take them."""
    for gather, kernel in (((1 << 19) - 1, "256x256"), (1 << 19, "128x128")):
        assert rules("product", 1, 1, 8, 1 << 20, 4096, 4096, gather, 1, 0) == kernel
        assert rules("weight_grad", 1, 8, 1 << 20, 4096, 4096, gather) == kernel
    assert rules("product", 1, 1, 8, 1 << 20, 4096, 4096, 0, 1, 0) == "256x256"


def test_shared_reductions_are_the_same_for_gathered_rows(rules):
    """The workspace is sized without their number."""
    for E, R, K, N in ((1, 32768, 512, 512), (4, 16384, 512, 512), (8, 32768, 2048, 2048), (1, 8192, 1024, 1024), (17, 3002, 776, 1544), (128, 1024, 1024, 1024)):
        for half in (0, 1):
            got = {rules("weight_grad", half, E, R, K, N, g) == "parts" for g in (0, 1, R, 1 << 29)}
            assert len(got) == 1


def test_every_launch_fits_a_grid(ffn_rules):
    """Up to the limits that the entry points check, (ceil(R / 64) + E) * ceil(width / 64) and E * ceil(K / 64) * ceil(N / 64) below 2^23, no tiling asks for 2^24 blocks, so that a block's number is all that
    finds its tile."""
    half = 1 << 23
    for E in (1, 2, 63, 64, 65, 511, 512):
        for tiles in (1, 2, 3, 100, 1 << 10, 1 << 14):                 # 64-wide column tiles
            R = min((half // tiles - 1 - E) * 64, (1 << 30) - 1)       # the most rows
            for rows in {1, 63, R // 2, R} if R > 0 else ():
                for tile in (64, 128, 256):
                    NT = -(-tiles * 64 // tile)
                    for shorts_last in (0, 1):
                        assert 0 < ffn_rules.grid(E, rows, tile, NT, rows, shorts_last) < 1 << 24
            most = (half // E - 1) // tiles                            # the most row tiles of weight gradients
            for tile in (64, 128, 256):
                if most > 0:
                    assert ffn_rules.grid(E, most * 64, tile, -(-tiles * 64 // tile), E * most * 64, 0) < 1 << 24
