"""Integers that the C ABI's 32 and 64 bits do not hold are refused by the binding, not cut (no GPU: nothing is launched)."""
import pytest
import torch

import paper_2601_18511_amd as pkg
from paper_2601_18511_amd import ppmm

HUGE = ((1 << 32) + 1, (1 << 64) + 1, -(1 << 32) + 1)


def _cut(monkeypatch):
    """A cache and a batch whose tensors are never looked at, and a library that records what reaches it."""
    seen = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: seen.append(name) or 0

    monkeypatch.setattr(ppmm, "_lib", Library())
    monkeypatch.setattr(ppmm, "_batch", lambda *args: ppmm._CBatch(0x1000, 0x2000, 0x3000, 1, 1))
    monkeypatch.setattr(ppmm, "_packed", lambda cache, name, t, heads, types: (t.shape[0], 0, (0x1000, 64, 64)))
    monkeypatch.setattr(ppmm, "_handle", lambda device, stream: 0)
    cache = object.__new__(pkg.PpkvCache)
    cache.kv_heads, cache.head_dim, cache.device, cache._c = 1, 64, 0, ppmm._CCache(0x1000, 1, 16, 1, 64)
    return cache, seen


def test_pool_sizes():
    good = (1, 16, 1, 64)
    assert pkg.ppkv_pool_bytes(*good) == 16 * 80
    for at in range(4):
        for v in HUGE[:2] + ((1 << 32) + good[at], (1 << 64) + good[at]):
            assert pkg.ppkv_pool_bytes(*good[:at], v, *good[at + 1:]) == 0, (at, v)
            with pytest.raises(ValueError):
                pkg.ppkv_cache_create(*good[:at], v, *good[at + 1:], device="cpu")


@pytest.mark.parametrize("huge", HUGE)
def test_sizes_of_a_call(monkeypatch, huge):
    cache, seen = _cut(monkeypatch)
    x = torch.zeros((1, 1, 64), dtype=torch.bfloat16)
    for call in (lambda: pkg.ppkv_attention(cache, x, x, None, None, None, max_q=huge),
                 lambda: pkg.ppkv_attention_scratch_bytes(cache, 1, 1, None, None, None, max_q=huge),
                 lambda: pkg.ppkv_attention_scratch_bytes(cache, 1, huge, None, None, None, max_q=1),
                 lambda: pkg.ppkv_read(cache, x, None, None, None, None, frac_bits=huge)):
        with pytest.raises(ValueError):
            call()
    assert not seen


def test_64_bit_sizes_of_a_call(monkeypatch):
    cache, seen = _cut(monkeypatch)
    x = torch.zeros((1, 1, 64), dtype=torch.bfloat16)
    for huge in (1 << 64, -(1 << 64) + 5):
        for call in (lambda: pkg.ppkv_attention(cache, x, x, None, None, None, max_q=1, max_len=huge),
                     lambda: pkg.ppkv_attention_scratch_bytes(cache, 1, 1, None, None, None, max_q=1, max_len=huge),
                     lambda: pkg.ppkv_attention_scratch_bytes(cache, huge, 1, None, None, None, max_q=1)):
            with pytest.raises(ValueError):
                call()
    assert not seen
