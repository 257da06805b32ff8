"""Which kernels the gated linear map's sizes take (the rule is host code of its own, compiled here), and that the GPU tests'
sizes take all of them."""
import ctypes
import math
import os
import random
import subprocess

import pytest

import test_gpu_gated_linear as sizes

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2605_30409_amd", "csrc")
FWD, D, DX, DW = range(4)


@pytest.fixture(scope="module")
def variants(tmp_path_factory):
    """variants(M, C, F, bf16): {(product, bf16, BM, BN, buffers, parts?): stages of a part} of a call and its gradient."""
    lib = str(tmp_path_factory.mktemp("rule") / "rule.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", lib, os.path.join(HERE, "gated_rule.cpp")], check=True)
    lib, out = ctypes.CDLL(lib), (ctypes.c_int * 5)()

    def of(M, C, F, bf16):
        got = {}
        for kind in range(4):
            if lib.rule_tiles(kind, M, C, F, bf16):
                lib.rule_cut(kind, M, C, F, bf16, out)
                got[(kind, bf16, *out[:3], out[3] > 1)] = out[4]
        return got
    return of


def taken(variants):
    """Those that a GPU test takes for more stages than there are buffers, so that each is used again."""
    return {v for s in sizes.VARIANTS for bf16 in (0, 1) for v, stages in variants(*s, bf16).items() if stages > v[4] + 1}


def test_every_choice_is_tested(variants):
    have = taken(variants)
    r = random.Random(1)

    def log(lo, hi):
        return int(math.exp(r.uniform(math.log(lo), math.log(hi))))
    for _ in range(60000):
        M, C, F = log(1, 70 if r.random() < 0.3 else 20000), log(1, 20000), log(1, 40000)
        if r.random() < 0.5:
            C = max(8, C // 8 * 8)
        for bf16 in (0, 1):
            assert have.issuperset(variants(M, C, F, bf16)), (M, C, F, bf16)


def test_decoding_batches_through_tiles(variants):
    """64 x 64 tiles with a contraction that is not cut, and one that is: eight buffers, used again."""
    for s in ((64, 2048, 8192), (39, 1656, 6441), (57, 872, 5349), (64, 768, 4159)):
        assert variants(*s, 1)[(FWD, 1, 64, 64, 8, False)] > 9
    assert variants(9, 8272, 547, 1)[(FWD, 1, 64, 64, 8, True)] > 9


def test_nothing_is_built_that_no_size_takes(variants):
    """The tiled kernels by their names in the built library: those that the sizes above take."""
    import re

    import paper_2605_30409_amd as gdn
    with open(gdn.LIB_PATH, "rb") as f:
        names = set(re.findall(rb"gdn_gated_tile_kernelI([tf])Li(\d)ELi(\d+)ELi(\d+)ELi\dELi\dELi(\d)EEE", f.read()))
    built = {(int(kind), int(e == b"t"), int(bm), int(bn), int(depth)) for e, kind, bm, bn, depth in names}
    assert built == {v[:5] for v in taken(variants)}
