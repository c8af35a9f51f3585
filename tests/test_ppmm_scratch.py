"""How much scratch attention asks for (no GPU: the sizes are the host's)."""
import itertools

import pytest

from paper_2601_18511_amd import ppmm

MOST = 1 << 27


def _scratch(batch, max_q, heads, kv_heads, D, page, width, max_len=0, tokens=None):
    cache = ppmm._CCache(0x1000, 1 << 20, page, kv_heads, D)
    where = ppmm._CBatch(0x1000, 0x2000, 0x3000, batch, width)
    tokens = batch * max_q if tokens is None else tokens
    return ppmm.load_library().ppkv_attention_scratch_bytes(cache, where, tokens, heads, max_q, max_len, 0)


@pytest.mark.parametrize("D", (64, 128))
def test_scratch_stays_below_its_bound(D):
    """Chunks of a prompt and batches of single tokens over caches of every length, with and without an expected length."""
    sizes = itertools.product((1, 7, 64, 500, 8000), (1, 3, 17, 100, 512, 2000, 2040, 2048, 30000), ((8, 8), (32, 8), (7, 1), (128, 1)),
                              (4096, 32768, 131072, 1 << 24), (False, True))
    for batch, max_q, (heads, kv_heads), capacity, expected in sizes:
        size = _scratch(batch, max_q, heads, kv_heads, D, 64, capacity // 64, capacity if expected else 0)
        assert size <= MOST, (batch, max_q, heads, kv_heads, capacity, size)
        assert size % (4 * (D + 2) * batch * max_q * heads) == 0


def test_no_cliff_between_neighbouring_chunks():
    """Where the rows fill the chip there is nothing to split, a few rows more or less."""
    for tokens in (1000, 2000, 2040, 2048, 4000):
        assert _scratch(1, tokens, 32, 8, 128, 64, 512) <= 32 << 20, tokens


def test_rows_of_no_sequence_count():
    """The scratch is laid out by row: rows behind the last sequence have a share of it, and there may be very many."""
    assert _scratch(4, 1, 32, 8, 128, 64, 2048, tokens=1 << 20) <= MOST
    assert _scratch(4, 1, 1 << 16, 1, 128, 64, 2048, tokens=(1 << 31) - 1) <= MOST
    assert 0 < _scratch(4, 1, 32, 8, 128, 64, 2048) <= MOST
