"""Which form of its kernels a product of a linear layer in 8 bits takes: the sizes that the tests on a GPU use to reach each of them."""
import ctypes as C
import os
import subprocess

import pytest

import paper_2510_09103_b200 as A
from linear8_forms import BF16, F32, FORWARD, INPUT, SIZES, WEIGHT

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def form(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("linear8") / "form.so")
    cuda = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2510_09103_b200", "csrc"),
                    "-I", cuda, "-o", path, os.path.join(ROOT, "tests", "linear8_form_host.cpp")], check=True)
    lib = C.CDLL(path)
    lib.linear8_form.restype = C.c_char_p

    def of(which, kind, tokens, out, inn):
        ld = -(-inn // 16) * 16
        d = A.linear8_desc(tokens, out, inn, x8_ld=ld, w8_ld=ld, y_dtype=kind, dx_dtype=kind, dweight_dtype=kind)
        return lib.linear8_form(C.byref(d), which).decode()

    return of


@pytest.mark.parametrize("which,kind,name,tokens,out,inn", SIZES)
def test_sizes_take_the_form_that_they_stand_for(form, which, kind, name, tokens, out, inn):
    assert form(which, kind, tokens, out, inn) == name


def test_every_form_has_its_sizes():
    have = {(s[0], s[1], s[2]) for s in SIZES}
    for which, names in ((FORWARD, ("lines", "strips", "pairs")), (INPUT, ("folded strips", "strips", "pairs", "pairs, K cut", "pairs, long sums")),
                         (WEIGHT, ("folded strips", "strips", "pairs", "pairs, K cut", "pairs, long sums"))):
        for name in names:
            assert (which, BF16, name) in have
            if which != FORWARD and name in ("folded strips", "pairs", "pairs, K cut"):
                assert (which, F32, name) in have
