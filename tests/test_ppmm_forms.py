"""Which kernel takes a product (no GPU): every form that is built is reached by some size, and every form that is reached by a GPU test."""
import itertools
import os
import re
import shutil
import subprocess

import pytest

import paper_2601_18511_amd as pkg
from tests.test_ppmv_forms_gpu import CASES, forms

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    exe = str(tmp_path_factory.mktemp("forms") / "ppmm_forms")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-O1", "-I", os.path.join(ROOT, "paper_2601_18511_amd", "csrc"), "-o", exe,
                    os.path.join(ROOT, "tests", "host", "ppmm_forms.cpp")], check=True)

    def run(calls):
        """{(kernel, waves, tokens, group, gated, offsets)}"""
        calls = list(calls)
        lines = subprocess.run([exe], input="\n".join("%d %d %d %d %d %d" % c for c in calls), capture_output=True, text=True, check=True).stdout.split("\n")
        return {(f[0], int(f[1]), int(f[2])) + tuple(c[3:]) for f, c in zip((line.split() for line in lines), calls)}

    return run


@pytest.fixture(scope="module")
def reached(choose):
    M = (1, 16, 100, 1000, 2100, 4096, 4200, 8192, 8300, 12000, 13000, 14336, 20000, 100000, 1 << 20)
    K = (1, 500, 3584, 4096, 8200, 14336, 14337)
    T = (1, 2, 4, 5, 9, 16, 17, 30, 32, 33, 45, 48, 49, 60, 64, 65, 70, 130, 300, 1000, 4000)
    return choose(call for size in itertools.product(M, K, T) for call in forms(*size))


def test_gpu_cases_reach_every_form(choose, reached):
    assert len(reached) > 100
    assert reached == choose(call for size in CASES for call in forms(*size))


def test_every_form_that_is_built_is_reached(reached):
    if shutil.which("nm") is None:
        pytest.skip("no nm")
    pkg.load_library()
    names = subprocess.run(["nm", "-C", pkg.build.LIB], capture_output=True, text=True, check=True).stdout
    built = set()
    for kernel, args in re.findall(r"::(stream|few_tokens|batch|many_tokens)_kernel<(.*?)>", names):
        *numbers, gated, offsets = [x.strip() for x in args.split(",")][1:]
        *sizes, groups = [int(x) for x in numbers]
        waves, tokens = {"stream": lambda w: (w, 0), "few_tokens": lambda w: (w, 16), "batch": lambda t, w: (w, 16 * t), "many_tokens": lambda: (4, 128)}[kernel](*sizes)
        built.add((kernel.split("_")[0], waves, tokens, 128 // groups, gated == "true", offsets == "true"))
    assert len(built) > 100
    assert built == reached
