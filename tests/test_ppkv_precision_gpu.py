"""How exactly attention weighs the values: results that cancel, so that the rounding of a result hides nothing.

Keys 0 and 1 are alike and hold the values v and -v; key 2 is zero in everything and has the largest score.  With s = 5 unit, a power of
two, and v = s (code - 7.5) the format is exact (b = -23.5 s), so both values are held as they are and the result is 0.  It is computed
with weights w near p s, two bf16 numbers off by 2^-16 p s at the most:  w (16 + code - 24) + w (31 - code - 24) + 2 p (b + 24 s) over
1 + 2 p.  That leaves |w - p s| <= 2^-16 p s, and the roundings of sums of at most 48 p s: eight matrix instructions, two multiply-adds and
the sum of waves, 12 2^-23 48 p s (2^-23: a matrix unit may cut instead of rounding).  With p / (1 + 2 p) <= 1/3 both are below
s (2^-17.5 + 2^-15.4); half a step of a result that small is less than 2^-8 of it or half the smallest fp16 step, 2^-25.  Together below
47 s 2^-20 = s 2^-14.4.  Weights off by 2^-16 that are not taken off again, w (16 + code) - p 23.5 s each, are off by 47 s 2^-18."""
import numpy as np
import pytest

from oracle import clear_oracle as oracle

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ("bfloat16", "float16"))
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("heads,T", ((4, 1), (8, 1), (40, 3)))
def test_values_that_cancel(gpu_device, heads, T, D, dtype):
    import torch

    import paper_2601_18511_amd as pkg

    B, t, rng = 16, getattr(torch, dtype), np.random.default_rng(heads + D)
    codes = rng.integers(0, 16, (B, D))
    codes[:, 0::32], codes[:, 1::32] = 0, 15                             # every group has its whole range
    unit = 2.0 ** rng.integers(-2, 3, (B, D // 32)).repeat(32, 1)
    v = np.zeros((B, 3, 1, D))
    v[:, 0, 0] = 5 * unit * (codes - 7.5)
    v[:, 1] = -v[:, 0]
    k = np.zeros((B, 3, 1, D))
    k[:, :2, 0, 0] = -1.0
    q = np.zeros((B * T, heads, D))
    q[:, :, 0] = rng.uniform(0.1, 1.5, (B * T, heads))
    k, v, q = (torch.from_numpy(x).to(t) for x in (k, v, q))
    cache = pkg.ppkv_cache_create(B, 16, 1, D, device=gpu_device)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=gpu_device)  # noqa: E731
    lens, table = i32([3] * B), i32(np.arange(B)[:, None])
    pkg.ppkv_append(cache, k.view(-1, 1, D).to(gpu_device), v.view(-1, 1, D).to(gpu_device), i32(3 * np.arange(B + 1)), lens, table)
    out = torch.empty((B * T, heads, D), dtype=t, device=gpu_device)
    pkg.ppkv_attention(cache, q.to(gpu_device), out, i32(T * np.arange(B + 1)), lens, table, max_q=T, causal=False, scale=1.0)
    got = out.double().cpu().numpy().reshape(B, T, heads, D)
    for b in range(B):
        held_k, held_v = oracle.held(k[b].double().numpy()), oracle.held(v[b].double().numpy())
        assert (held_v[0] + held_v[1] == 0).all()
        want = oracle.attention(q[b * T:(b + 1) * T].double().numpy(), held_k, held_v, 1.0, False)
        assert (np.abs(got[b] - want) <= 47 * 5 * unit[b] * 2.0 ** -20).all(), float((np.abs(got[b] - want) / unit[b]).max())
