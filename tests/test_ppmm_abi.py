"""The clear track's C ABI and binding without a GPU: symbols, argument checks, the header as plain C, the host code under
sanitizers; and the pins of its oracle."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

import paper_2601_18511_amd as pkg
from oracle import clear_oracle as oracle
from paper_2601_18511_amd import pcmm, ppmm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, EUNSUPPORTED = pcmm.PCMM_OK, pcmm.PCMM_EINVAL, pcmm.PCMM_EUNSUPPORTED
A, B, C = (ctypes.c_void_p(x) for x in (0x1000, 0x2000, 0x3000))       # never dereferenced: the checks fail first


def test_header_symbols_are_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ppmm.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(pp(?:mv|kv)_[a-z_]+)\s*\(", text)))
    lib = ppmm.load_library()
    for name in names:
        assert getattr(lib, name) is not None
        assert hasattr(pkg, name), name
    assert sorted(ppmm.EXPORTED) == names


def test_header_is_plain_c(tmp_path):
    src = tmp_path / "use_ppmm.c"
    src.write_text('#include "ppmm.h"\nint main(void) {\n    ppmv_plan *p = 0;\n    ppkv_cache c = {0, 0, 0, 0, 0};\n    ppkv_batch b = {0, 0, 0, 0, 0};\n'
                   "    if (ppmv_plan_create(&p, 0, 0, 32, PPMM_BF16, 0, 0, 0, 0, 0) != PCMM_EINVAL || p) return 1;\n"
                   "    if (ppkv_append(&c, &b, 0, PPMM_BF16, 0, 0, 0, 0, 0, 0, 0, 0) != PCMM_EINVAL) return 2;\n"
                   "    ppmv_plan_destroy(p);\n    return ppkv_pool_bytes(1, 16, 1, 64) == 16 * 80 ? 0 : 3;\n}\n")
    inc = os.path.join(ROOT, "include")
    for cc, std in (("gcc", "-std=c99"), ("g++", "-std=c++11")):
        if shutil.which(cc) is None:
            pytest.skip("no %s" % cc)
        subprocess.run([cc, std, "-Wall", "-Wextra", "-pedantic", "-Werror", "-fsyntax-only", "-I", inc] + (["-x", "c++"] if cc == "g++" else []) + [str(src)], check=True)
    exe = tmp_path / "use_ppmm"
    subprocess.run(["gcc", "-std=c99", "-I", inc, str(src), "-o", str(exe), "-L", os.path.dirname(pkg.build.LIB), "-l:libpcmm.so",
                    "-Wl,-rpath," + os.path.dirname(pkg.build.LIB)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0


def test_weight_plan_arguments():
    lib = ppmm.load_library()
    out = ctypes.c_void_p(123)

    def create(M=4, K=64, group=32, kind=0, codes=A, scales=B, device=0):
        return lib.ppmv_plan_create(ctypes.byref(out), M, K, group, kind, codes, scales, None, device, None)

    assert create(M=0) == EINVAL and out.value is None
    for bad in (dict(K=0), dict(M=(1 << 24) + 1), dict(K=(1 << 22) + 1), dict(group=16), dict(group=96), dict(kind=2), dict(kind=-1),
                dict(codes=None), dict(scales=None), dict(device=-1)):
        assert create(**bad) == EINVAL, bad
    assert create(M=1 << 24, K=1 << 22) == EUNSUPPORTED
    assert lib.ppmv_plan_create(None, 4, 64, 32, 0, A, B, None, 0, None) == EINVAL
    assert lib.ppmv_run(None, 1, A, 64, B, 4, None) == EINVAL
    assert lib.ppmv_gated_run(None, None, 1, A, 64, B, 4, None) == EINVAL
    assert lib.ppmv_plan_workspace_bytes(None) == 0
    lib.ppmv_plan_destroy(None)


def _cache(pool=0x1000, pages=4, page_size=16, kv_heads=2, head_dim=64):
    return ppmm._CCache(pool, pages, page_size, kv_heads, head_dim)


def _batch(starts=0x1000, lens=0x2000, table=0x3000, batch=2, width=2):
    return ppmm._CBatch(starts, lens, table, batch, width)


BAD_CACHES = [dict(pool=None), dict(pool=0x1008), dict(pages=0), dict(pages=1 << 31), dict(page_size=0), dict(page_size=24), dict(page_size=65552),
              dict(kv_heads=0), dict(kv_heads=1025), dict(head_dim=96), dict(head_dim=0)]
BAD_BATCHES = [dict(starts=None), dict(lens=None), dict(table=None), dict(batch=0), dict(batch=65536), dict(width=0), dict(width=1 << 27)]


def test_cache_arguments():
    lib = ppmm.load_library()

    def append(cache=_cache(), batch=_batch(), tokens=3, kind=0, k=A, strides=(128, 64), v=B, device=0):
        return lib.ppkv_append(cache, batch, tokens, kind, k, *strides, v, *strides, device, None)

    def read(cache=_cache(), batch=_batch(), tokens=3, kind=0, frac=0, k=A, strides=(128, 64), v=B, device=0):
        return lib.ppkv_read(cache, batch, tokens, kind, frac, k, *strides, v, *strides, device, None)

    def attend(cache=_cache(), batch=_batch(), tokens=3, kind=0, heads=4, q=A, strides=(256, 64), out=B, ostrides=(256, 64), max_q=2, max_len=0,
               scratch=None, size=0, device=0):
        return lib.ppkv_attention(cache, batch, tokens, kind, heads, q, *strides, out, *ostrides, 0.125, 1, max_q, max_len, scratch, size, device, None)

    for call in (append, read, attend):
        for bad in BAD_CACHES:
            assert call(cache=_cache(**bad)) == EINVAL, (call.__name__, bad)
        for bad in BAD_BATCHES:
            assert call(batch=_batch(**bad)) == EINVAL, (call.__name__, bad)
        for bad in (dict(tokens=-1), dict(tokens=1 << 31), dict(device=-1), dict(kind=7), dict(strides=(-1, 64)) if call is not read else dict(kind=3)):
            assert call(**bad) == EINVAL, (call.__name__, bad)
        assert call(tokens=0) == OK                                        # nothing to do, no device needed
    assert append(kind=2) == EINVAL and attend(kind=2) == EINVAL
    assert append(k=None) == EINVAL and append(v=None) == EINVAL
    assert read(kind=2, frac=31) == EINVAL and read(kind=2, frac=-1) == EINVAL and read(kind=0, frac=1) == EINVAL
    assert read(k=A, v=A) == EINVAL
    for strides in ((127, 64), (128, 63), (0, 64), (64, 64)):              # rows that overlap
        assert read(strides=strides) == EINVAL, strides
        assert attend(ostrides=strides) == EINVAL, strides
    assert read(k=None, v=None) == OK
    for bad in (dict(heads=0), dict(heads=3), dict(q=None), dict(out=None), dict(out=A), dict(max_q=-1), dict(max_len=-1), dict(heads=2 * 65537)):
        assert attend(**bad) == EINVAL, bad
    assert attend(max_q=0) == OK
    assert lib.ppkv_attention_scratch_bytes(_cache(pages=0), _batch(), 3, 4, 2, 0, 0) == 0


def test_pool_sizes():
    assert pkg.ppkv_pool_bytes(1, 16, 1, 64) == 16 * 80
    assert pkg.ppkv_pool_bytes(1000, 48, 8, 128) == 1000 * 48 * 8 * 160
    for args in ((0, 16, 1, 64), (1, 8, 1, 64), (1, 16, 0, 64), (1, 16, 1, 80), (1 << 31, 16, 1, 64), ((1 << 31) - 1, 65536, 1024, 128)):
        assert pkg.ppkv_pool_bytes(*args) == 0


def test_binding_refuses_what_is_not_on_a_gpu():
    import torch

    codes, scales = torch.zeros((4, 32), dtype=torch.uint8), torch.ones((4, 2), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        pkg.ppmv_plan_create(codes, scales, 64, 32)
    with pytest.raises(ValueError):
        pkg.ppkv_cache_create(0, 16, 1, 64, device="cpu")
    with pytest.raises(ValueError):
        pkg.ppkv_cache_create(2, 16, 1, 64, device="cpu")
    cache = object.__new__(pkg.PpkvCache)
    cache.kv_heads, cache.head_dim, cache.device = 1, 64, 0
    x = torch.zeros((1, 1, 64), dtype=torch.bfloat16)
    ints = torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros((1, 1), dtype=torch.int32)
    for call in (lambda: pkg.ppkv_append(cache, x, x.clone(), *ints), lambda: pkg.ppkv_read(cache, x, None, *ints),
                 lambda: pkg.ppkv_attention(cache, x, x.clone(), *ints, max_q=1)):
        with pytest.raises(ValueError):
            call()


def test_host_checks_under_sanitizers(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    exe = tmp_path / "ppmm_host_check"
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-g", "-O1",
                    "-I", os.path.join(ROOT, "paper_2601_18511_amd", "csrc"), "-o", str(exe), os.path.join(ROOT, "tests", "host", "ppmm_host_check.cpp")], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and "all checks held" in r.stdout, r.stdout + r.stderr


# ---- pins of the oracle ---------------------------------------------------------------------------------------------


def test_oracle_weights_by_hand():
    codes = np.array([[0x80, 0x0F]], np.uint8)                  # c = 0, 8, 15 (and a filler): w = s (c - 8) + o
    got = oracle.weights(codes, [[0.5]], [[0.25]], 3, 32)
    assert got.tolist() == [[-3.75, 0.25, 3.75]]


def test_oracle_format_by_hand():
    x = np.zeros((1, 32))
    x[0, 0], x[0, 1], x[0, 2] = 15.0, 0.5, 1.5                  # s = 1, b = -16: codes are the numbers themselves, ties to even
    c, s, b = oracle.quantise(x)
    assert (s.tolist(), b.tolist()) == ([[1.0]], [[-16.0]])
    assert c[0, :4].tolist() == [15, 0, 2, 0]
    assert oracle.held(x)[0, :4].tolist() == [15.0, 0.0, 2.0, 0.0]
    same = np.full((1, 32), 0.625)
    assert (oracle.held(same) == 0.625).all()                   # no range: the offset alone
    for v in (np.nan, np.inf, -np.inf):
        x[0, 3] = v
        assert np.isnan(oracle.held(x)).all()
    assert (oracle.held(np.concatenate([x, same], 1))[0, 32:] == 0.625).all()                # a bad group leaves its neighbour
    rng = np.random.default_rng(0)
    y = rng.standard_normal((50, 128))
    c, s, b = oracle.quantise(y)
    assert (np.abs(oracle.held(y) - y) <= np.repeat(s, 32, -1) * 0.5 + np.repeat(np.abs(b) + 16 * s, 32, -1) * 2.0 ** -8).all()


def test_oracle_bf16_rounding():
    import torch

    rng = np.random.default_rng(1)
    x = rng.standard_normal(1000) * 2.0 ** rng.integers(-100, 100, 1000)
    assert (oracle.round_bf16(x) == torch.from_numpy(x).float().bfloat16().double().numpy()).all()


def test_oracle_attention_by_hand():
    k = np.array([[[0.0]], [[np.log(3.0)]]])
    v = np.array([[[4.0]], [[8.0]]])
    q = np.ones((2, 1, 1))
    assert np.allclose(oracle.attention(q, k, v, 1.0, True)[:, 0, 0], [4.0, 7.0])
    assert np.allclose(oracle.attention(q, k, v, 1.0, False)[:, 0, 0], [7.0, 7.0])
    assert (oracle.attention(np.ones((3, 1, 1)), k, v, 1.0, True)[0] == 0).all()             # in front of the first token
    assert (oracle.attention(q, k[:0], v[:0], 1.0, False) == 0).all()
