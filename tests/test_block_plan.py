"""How products of block-scaled matrices and gated blocks are cut (srq_block_plan.hpp): host arithmetic, compiled alone."""
import ctypes as C
import os
import random
import subprocess

import pytest

from block_shapes import GATED, PRODUCTS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2511_00874_amd", "csrc")
WRAP = """
#include "srq_block_plan.hpp"
using namespace srq;
extern "C" void cut(int gated, size_t P, size_t Q, size_t R, int f8, size_t* o) {
  const BlockCut c = gated ? gated_cut(P, Q, R, f8) : product_cut(P, Q, R, f8);
  const BlockForm& f = (gated ? GATED_FORMS : PRODUCT_FORMS)[c.form];
  const size_t v[] = {(size_t)c.form, c.chunk, c.whole, c.nsplit, c.per_split, c.partial_bytes, (size_t)f.bm, (size_t)f.bn, (size_t)f.per_cu};
  for (int i = 0; i < 9; ++i) o[i] = v[i];
}
"""


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    d = tmp_path_factory.mktemp("block_plan")
    (d / "plan.cpp").write_text(WRAP)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(d / "plan.cpp"), "-o", str(d / "plan.so")], check=True)
    lib = C.CDLL(str(d / "plan.so"))
    lib.cut.argtypes = [C.c_int] + [C.c_size_t] * 3 + [C.c_int, C.c_void_p]

    def f(gated, size, f8):
        o = (C.c_size_t * 9)()
        lib.cut(gated, *size, f8, o)
        return dict(zip(("form", "chunk", "whole", "slices", "per", "bytes", "bm", "bn", "per_cu"), o))
    return f


def _taken(c):
    items = c["whole"] + (c["chunk"] - c["whole"]) * c["slices"]  # of an XCD, which has 32 CUs
    return c["form"], items > 32 * c["per_cu"], c["slices"] > 1


@pytest.mark.parametrize("f8", [False, True])
def test_sizes_take_the_forms_they_are_listed_for(cut, f8):
    assert set(PRODUCTS[f8]) == {(f, w, s) for f in range(4) for w in (False, True) for s in (False, True)}
    assert {k[0] for k in GATED[f8]} == set(range(4)) and {k for k in GATED[f8] if k[0] < 2} == {k for k in PRODUCTS[f8] if k[0] < 2}
    for gated, shapes in ((0, PRODUCTS[f8]), (1, GATED[f8])):
        for want, size in shapes.items():
            assert _taken(cut(gated, size, f8)) == want, (gated, size)


def test_the_sizes_of_a_training_step(cut):
    # the products of a 2048-wide block with 5632 hidden features on 16384 tokens: large tiles, weight gradients in slices beside whole ones
    for size, f8, want in (((16384, 2048, 5632), True, (0, True, False)), ((16384, 2048, 11264), True, (0, True, False)),
                           ((11264, 2048, 16384), False, (0, True, True))):
        assert _taken(cut(0, size, f8)) == want, size
    assert _taken(cut(1, (16384, 5632, 2048), False)) == (0, True, False)


def test_a_cut_covers_the_contraction_and_its_slices_fit(cut):
    rng = random.Random(3)
    for _ in range(4000):
        gated = rng.random() < 0.5
        size = [int(2 ** rng.uniform(4.1, 14)), 128 * int(2 ** rng.uniform(0, 6)) if gated else int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 15))]
        c = cut(gated, size, rng.random() < 0.5)
        stages = -(-size[2] // 128)
        columns = 2 * size[1] if gated else size[1]
        tiles = -(-size[0] // c["bm"]) * -(-columns // c["bn"])
        assert c["chunk"] == -(-tiles // 8) and c["whole"] <= c["chunk"]
        assert (c["slices"] - 1) * c["per"] < stages <= c["slices"] * c["per"]  # every slice has a stage
        if c["slices"] == 1:
            assert c["whole"] == c["chunk"] and c["bytes"] == 0
        else:  # tiles in slices: the last of every XCD
            assert c["bytes"] == 8 * (c["chunk"] - c["whole"]) * c["slices"] * c["bm"] * c["bn"] * 4 and c["chunk"] > c["whole"]
            assert c["whole"] % (32 * c["per_cu"]) == 0


def test_few_tiles_of_a_long_contraction_ask_for_a_workspace(cut):
    from paper_2511_00874_amd import lib as L
    for flags in (0, 1):
        need = L.raw.sr_gemm_blocks_workspace_bytes(1009, 2048, 65536, flags)
        assert need == cut(0, (1009, 2048, 65536), flags)["bytes"] > 0
