"""The largest calls of the cache and of attention: what the header calls unsupported is refused before anything is launched (no GPU)."""
import ctypes

import pytest

from paper_2601_18511_amd import pcmm, ppmm

A, B = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x2000)         # never dereferenced


@pytest.mark.parametrize("tokens,kv_heads,D", [(1 << 27, 1, 128), ((1 << 27) - 1, 1, 128), (1 << 17, 1024, 128), ((1 << 31) - 1, 8, 64)])
def test_tokens_of_an_append_or_a_read(tokens, kv_heads, D):
    assert tokens * kv_heads * D > (1 << 34) - 1024
    lib = ppmm.load_library()
    cache, batch = ppmm._CCache(0x1000, 4, 16, kv_heads, D), ppmm._CBatch(0x1000, 0x2000, 0x3000, 2, 2)
    strides = (kv_heads * D, D)
    assert lib.ppkv_append(cache, batch, tokens, 0, A, *strides, B, *strides, 0, None) == pcmm.PCMM_EUNSUPPORTED
    assert lib.ppkv_read(cache, batch, tokens, 0, 0, A, *strides, B, *strides, 0, None) == pcmm.PCMM_EUNSUPPORTED


@pytest.mark.parametrize("sequences,max_q,heads,kv_heads", [(1, 1 << 25, 32, 8), (4096, 2048, 32, 8), (65535, 32, 256, 256), (1 << 14, 1, 1024, 1024)])
def test_work_groups_of_attention(sequences, max_q, heads, kv_heads):
    assert sequences * kv_heads * -(-max_q * (heads // kv_heads) // 16) >= 1 << 24
    lib = ppmm.load_library()
    cache, batch = ppmm._CCache(0x1000, 4, 16, kv_heads, 128), ppmm._CBatch(0x1000, 0x2000, 0x3000, sequences, 2)
    tokens = min(sequences * max_q, 1 << 20)
    strides = (heads * 128, 128)
    size = lib.ppkv_attention_scratch_bytes(cache, batch, tokens, heads, max_q, 0, 0)
    assert lib.ppkv_attention(cache, batch, tokens, 0, heads, A, *strides, B, *strides, 0.125, 1, max_q, 0, A, size, 0, None) == pcmm.PCMM_EUNSUPPORTED
