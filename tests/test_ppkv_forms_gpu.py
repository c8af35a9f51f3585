"""Every form of the attention kernel, alone and with its keys split, against the oracle in 64 bits, with the bound of the other
attention tests.  With 128 channels up to 4 rows of a K/V head take one tile of (group, query) columns and 5 to 8 rows two; with 64
channels up to 8 rows take one; more rows take columns of one query each."""
import pytest

from tests.test_ppkv_gpu import Batch, _attend

pytestmark = pytest.mark.gpu
TYPES = ("bfloat16", "float16")
ONE = [(1, 1), (1, 17), (1, 64), (1, 65), (1, 1000)]
TWO = [(2, 70), (2, 2), (1, 129), (0, 5), (2, 400)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("seqs,heads,kv_heads,D,page", [(ONE, 8, 1, 128, 16), (ONE, 14, 2, 128, 48), (ONE, 5, 1, 128, 64), (ONE, 6, 2, 128, 16),
                                                        (TWO, 8, 2, 128, 16), (TWO, 3, 1, 128, 32), (ONE, 8, 1, 64, 16), (TWO, 8, 2, 64, 48),
                                                        (ONE, 9, 1, 128, 16), (ONE, 9, 1, 64, 16)])
def test_few_rows(gpu_device, seqs, heads, kv_heads, D, page, dtype):
    for causal in (True, False):
        b = Batch(seqs, heads, kv_heads, D, page, dtype, gpu_device, seed=heads + D).fill()
        b.check_attention(_attend(b, causal), causal)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("seqs,heads,kv_heads,D", [([(1, 5000), (1, 3), (1, 2049), (1, 700)], 8, 1, 128), ([(1, 5000), (1, 3), (1, 2049), (1, 700)], 16, 2, 128),
                                                   ([(2, 3000), (1, 1500)], 8, 2, 128), ([(1, 5000), (1, 3), (1, 2049)], 4, 1, 128),
                                                   ([(1, 5000), (1, 3), (1, 2049)], 8, 1, 64), ([(70, 3000), (3, 40)], 8, 2, 128), ([(40, 2500), (9, 1100)], 8, 1, 64)])
def test_split_keys(gpu_device, seqs, heads, kv_heads, D, dtype):
    import paper_2601_18511_amd as pkg

    b = Batch(seqs, heads, kv_heads, D, 16, dtype, gpu_device, seed=heads + D).fill()
    most = max(t for t, _ in seqs)
    for max_len in (0, max(n for _, n in seqs)):
        assert pkg.ppkv_attention_scratch_bytes(b.cache, b.tokens, heads, *b.where(), max_q=most, max_len=max_len) > 0
        b.check_attention(_attend(b, max_len=max_len))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,D,n", [(8, 128, 200), (8, 128, 3000), (4, 128, 200), (8, 64, 200)])
def test_nan_values_and_keys(gpu_device, heads, D, n, dtype):
    """One token whose 32 channels hold a NaN: of the value, those channels of every row; of the key, every row; behind the row, nothing."""
    import torch

    for which in ("k", "v"):
        for at in (0, n - 1, n):
            b = Batch([(1, n)], heads, 1, D, 16, dtype, gpu_device, seed=3, spare=2)
            clean = _attend(b.fill())
            if at == n:                                 # a token that is cached, but counted by a longer sequence only
                b = Batch([(1, n + 1)], heads, 1, D, 16, dtype, gpu_device, seed=3, spare=2)
            getattr(b, which)[0][at, 0, 40] = float("nan")
            b.fill()
            b.lens.fill_(n)
            if at == n:
                longer = _attend(b).cpu()
                assert torch.isfinite(longer).all()
                continue
            out = _attend(b).cpu()
            if which == "k":
                assert torch.isnan(out).all()
            else:
                assert torch.isnan(out[..., 32:64]).all()
                keep = [c for c in range(D) if not 32 <= c < 64]
                assert torch.equal(out[..., keep], clean.cpu()[..., keep])
