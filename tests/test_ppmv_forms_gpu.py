"""Every kernel form that a product can be given to, against the oracle in 64 bits: both types, all groups, plain and gated, with and
without offsets.  Tolerances as for the products of other sizes: a sum of n terms in 32 bits is off by at most n 2^-23 times the sum of
their magnitudes, the largest |x| (s (31 + 24) + |o|); |silu'| < 1.1, exp2 and the division by a few 2^-22; then half a step of the result."""
import numpy as np
import pytest

from oracle import clear_oracle as oracle

# M, K, T; K with whole blocks of 128 and part of one, several to each wave
CASES = [(40, 2500, 1), (33, 1100, 4),                     # x in LDS, 8 waves
         (40, 14336, 1), (33, 8200, 1),                    # 16 waves (two matrices in groups of 32: 8)
         (100, 700, 7), (520, 1100, 100), (2050, 264, 16),  # 16 tokens a work-group
         (20000, 1160, 9), (4200, 1160, 9),                # x shared by two waves, 16 tokens (plain; gated)
         (2100, 1160, 30), (2100, 1160, 45), (2100, 1160, 60), (2100, 1160, 70), (2100, 2184, 130),
         (13000, 1160, 9), (13000, 1160, 30), (13000, 1160, 45), (13000, 1160, 60), (20000, 264, 70),      # by four
         (12400, 392, 300), (6300, 264, 500), (2100, 264, 4000)]        # large tiles


def forms(M, K, T):
    """All calls of a size: (M, K, T, group, gated, offsets)"""
    return [(M, K, T, group, gated, offsets) for group in (32, 64, 128) for gated in (False, True) for offsets in (False, True)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ("bfloat16", "float16"))
@pytest.mark.parametrize("group", (32, 64, 128))
@pytest.mark.parametrize("M,K,T", CASES)
def test_every_form_matches_the_oracle(gpu_device, M, K, T, group, dtype):
    import torch

    import paper_2601_18511_amd as pkg

    t, half = getattr(torch, dtype), torch.finfo(getattr(torch, dtype)).eps / 2
    g = torch.Generator().manual_seed(M + K + T + group)
    rows = np.unique(np.concatenate([np.arange(min(M, 40)), np.arange(max(0, M - 40), M), np.random.default_rng(M).integers(0, M, 100)]))
    x = torch.randn((T, K), generator=g).to(t)
    X, at = x.double().numpy(), np.arange(K) // group
    weights = []
    for _ in range(2):
        codes = torch.randint(0, 256, (M, (K + 1) // 2), dtype=torch.uint8, generator=g)
        scales = ((0.5 + torch.rand((M, at[-1] + 1), generator=g)) / 64).to(t)
        weights.append((codes, scales, (torch.randn((M, at[-1] + 1), generator=g) / 64).to(t)))
    for offsets in (False, True):
        plans, want, bound = [], [], []
        for codes, scales, off in weights:
            plans.append(pkg.ppmv_plan_create(codes.to(gpu_device), scales.to(gpu_device), K, group, offsets=off.to(gpu_device) if offsets else None))
            s, o = scales.double().numpy()[rows], off.double().numpy()[rows] if offsets else None
            want.append(X @ oracle.weights(codes.numpy()[rows], s, o, K, group).T)
            bound.append((K + 64) * 2.0 ** -23 * (np.abs(X) @ (s[:, at] * 55.0 + (np.abs(o[:, at]) if offsets else 0.0)).T))
        for gated in (False, True):
            y = torch.full((T, M), float("nan"), dtype=t, device=gpu_device)
            if gated:
                pkg.ppmv_gated_run(plans[0], plans[1], x.to(gpu_device), y)
                silu = oracle.silu(want[0])
                exact = silu * want[1]
                most = 1.1 * bound[0] * (np.abs(want[1]) + bound[1]) + np.abs(silu) * bound[1] + np.abs(exact) * (np.abs(want[0]) + 8) * 2.0 ** -22
            else:
                pkg.ppmv_run(plans[0], x.to(gpu_device), y)
                exact, most = want[0], bound[0]
            got = y.double().cpu().numpy()
            assert np.isfinite(got).all(), (gated, offsets)
            off_by = np.abs(got[:, rows] - exact)
            assert (off_by <= half * (np.abs(exact) + most) + most + 2.0 ** -24).all(), (gated, offsets, float((off_by - half * np.abs(exact) - most).max()))
