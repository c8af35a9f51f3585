"""Strides of the clear track's arrays at their limits (no GPU: the checks are the host's)."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2601_18511_amd import pcmm, ppmm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_strides_at_their_limits_under_sanitizers(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    exe = tmp_path / "ppmm_strides_check"
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-g", "-O1",
                    "-I", os.path.join(ROOT, "paper_2601_18511_amd", "csrc"), "-o", str(exe), os.path.join(ROOT, "tests", "host", "ppmm_strides_check.cpp")], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and "all checks held" in r.stdout, r.stdout + r.stderr


def test_heads_too_far_apart_are_refused():
    lib = ppmm.load_library()
    cache, batch = ppmm._CCache(0x1000, 4, 16, 1024, 64), ppmm._CBatch(0x1000, 0x2000, 0x3000, 2, 2)
    heads = 1 << 26

    def attend(q_head=64, out_head=64):         # never runs: without rows there is nothing to do, and the checks come first
        return lib.ppkv_attention(cache, batch, 2, 0, heads, ctypes.c_void_p(0x1000), 1 << 40, q_head, ctypes.c_void_p(0x2000), 1 << 58, out_head,
                                  0.125, 1, 0, 0, None, 0, 0, None)

    assert attend() == pcmm.PCMM_OK
    assert attend(out_head=1 << 40) == pcmm.PCMM_EINVAL
    assert attend(q_head=1 << 40) == pcmm.PCMM_EINVAL
