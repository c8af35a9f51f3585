"""Products with 4-bit weights on the GPU against the oracle in 64 bits.

Tolerances.  A result is sum_g s_g (sum_{k in g} x (16 + c) - 24 sum_{k in g} x) + o_g sum x at the most: every term is at most
|x| (s (31 + 24) + |o|), and a sum of n terms in 32 bits, whatever its order, is off by at most n 2^-23 times the sum of their
magnitudes (2^-23: a matrix unit may cut instead of rounding).  The result is then rounded once, by half a step of its type."""
import numpy as np
import pytest

from oracle import clear_oracle as oracle

pytestmark = pytest.mark.gpu
TYPES = ("bfloat16", "float16")


def _case(M, K, T, group, dtype, offsets, seed, dev):
    import torch

    t = getattr(torch, dtype)
    g = torch.Generator().manual_seed(seed)
    groups = -(-K // group)
    codes = torch.randint(0, 256, (M, (K + 1) // 2), dtype=torch.uint8, generator=g)
    scales = ((0.5 + torch.rand((M, groups), generator=g)) / 64).to(t)
    off = (torch.randn((M, groups), generator=g) / 64).to(t) if offsets else None
    x = torch.randn((T, K), generator=g).to(t)
    return codes, scales, off, x


def _plan(codes, scales, off, K, group, dev):
    import paper_2601_18511_amd as pkg

    return pkg.ppmv_plan_create(codes.to(dev), scales.to(dev), K, group, offsets=None if off is None else off.to(dev))


def _want(codes, scales, off, x, group):
    """(exact product, bound of the error before the result is rounded)"""
    K = x.shape[1]
    o = None if off is None else off.double().numpy()
    w = oracle.weights(codes.numpy(), scales.double().numpy(), o, K, group)
    at = np.arange(K) // group
    most = scales.double().numpy()[:, at] * 55.0 + (0.0 if o is None else np.abs(o[:, at]))
    X = x.double().numpy()
    return X @ w.T, (K + 64) * 2.0 ** -23 * (np.abs(X) @ most.T)


def _half_step(dtype):
    import torch

    return torch.finfo(getattr(torch, dtype)).eps / 2


def _near(got, want, bound, dtype):
    got = got.double().cpu().numpy()
    half = _half_step(dtype)
    off = np.abs(got - want)
    assert (off <= half * (np.abs(want) + bound) + bound + 2.0 ** -24).all(), float((off - half * np.abs(want) - bound).max())
    # in the norm a result is rounded by half a step at the most, and the sums add less than a quarter of that at these sizes
    assert np.linalg.norm(off) <= 1.25 * half * np.linalg.norm(want) + 1e-30


SHAPES = [(1, 1, 1, 32), (1, 2, 3, 128), (16, 128, 1, 128), (17, 129, 16, 128), (16, 31, 2, 32), (33, 33, 17, 32), (100, 777, 13, 32), (64, 640, 33, 64),
          (130, 1000, 64, 64), (48, 4096, 1, 128), (257, 2049, 65, 128), (300, 512, 130, 32), (129, 1536, 200, 64), (512, 1024, 300, 128),
          (7, 14336, 5, 128), (2000, 96, 1, 64)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,T,group", SHAPES)
def test_product_matches_the_oracle(gpu_device, M, K, T, group, dtype):
    import torch

    import paper_2601_18511_amd as pkg

    for offsets in (False, True):
        codes, scales, off, x = _case(M, K, T, group, dtype, offsets, M + K + T, gpu_device)
        plan = _plan(codes, scales, off, K, group, gpu_device)
        y = torch.full((T, M), float("nan"), dtype=x.dtype, device=gpu_device)
        pkg.ppmv_run(plan, x.to(gpu_device), y)
        want, bound = _want(codes, scales, off, x, group)
        _near(y, want, bound, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,T,group", SHAPES)
def test_gated_product_matches_the_oracle(gpu_device, M, K, T, group, dtype):
    import torch

    import paper_2601_18511_amd as pkg

    for offsets in (False, True):
        gate = _case(M, K, T, group, dtype, offsets, 7 * M + K + T, gpu_device)
        up = _case(M, K, T, group, dtype, offsets, 11 * M + K + T, gpu_device)[:3]
        x = gate[3]
        plans = [_plan(*w, K, group, gpu_device) for w in (gate[:3], up)]
        h = torch.full((T, M), float("nan"), dtype=x.dtype, device=gpu_device)
        pkg.ppmv_gated_run(plans[0], plans[1], x.to(gpu_device), h)
        g, bg = _want(*gate[:3], x, group)
        u, bu = _want(*up, x, group)
        want = oracle.silu(g) * u
        # |silu'| < 1.1; exp2, its argument's rounding (|g| log2(e) 2^-23, relative), the division and the two products: a few 2^-22
        bound = 1.1 * bg * (np.abs(u) + bu) + np.abs(oracle.silu(g)) * bu + np.abs(want) * (np.abs(g) + 8) * 2.0 ** -22
        _near(h, want, bound, dtype)


@pytest.mark.parametrize("M,K,T,gated", [(64, 14336, 1, True), (40, 14337, 1, True), (64, 16384, 1, True), (16, 3584, 4, True), (16, 64, 70000, False),
                                         (16, 40, 5000, True), (5000, 64, 60, False), (9000, 128, 16, True)])
def test_sizes_at_the_limits_of_each_kernel(gpu_device, M, K, T, gated):
    """The largest x that lies in LDS and the first that does not, very many tokens of few rows, many rows of a short contraction."""
    import torch

    import paper_2601_18511_amd as pkg

    codes, scales, off, x = _case(M, K, T, 32, "bfloat16", True, M + K + T, gpu_device)
    plan = _plan(codes, scales, off, K, 32, gpu_device)
    y = torch.full((T, M), float("nan"), dtype=x.dtype, device=gpu_device)
    g, b = _want(codes, scales, off, x, 32)
    if gated:
        pkg.ppmv_gated_run(plan, plan, x.to(gpu_device), y)
        _near(y, oracle.silu(g) * g, 2.2 * b * (np.abs(g) + b + 1) + np.abs(g * g) * (np.abs(g) + 8) * 2.0 ** -22, "bfloat16")
    else:
        pkg.ppmv_run(plan, x.to(gpu_device), y)
        _near(y, g, b, "bfloat16")


def test_one_plan_as_gate_and_up(gpu_device):
    import torch

    import paper_2601_18511_amd as pkg

    codes, scales, off, x = _case(40, 200, 3, 64, "bfloat16", False, 5, gpu_device)
    plan = _plan(codes, scales, off, 200, 64, gpu_device)
    h = torch.empty((3, 40), dtype=torch.bfloat16, device=gpu_device)
    pkg.ppmv_gated_run(plan, plan, x.to(gpu_device), h)
    g, b = _want(codes, scales, off, x, 64)
    _near(h, oracle.silu(g) * g, 2.2 * b * (np.abs(g) + b + 1) + np.abs(g * g) * (np.abs(g) + 8) * 2.0 ** -22, "bfloat16")


@pytest.mark.parametrize("T", (1, 5, 33, 150))
def test_strides_alignment_and_neighbours(gpu_device, T):
    """Rows longer than K and M, elements aligned to two bytes only, one row for all tokens; nothing beside the result is written."""
    import torch

    import paper_2601_18511_amd as pkg

    M, K, group = 70, 333, 64
    codes, scales, off, x = _case(M, K, T, group, "bfloat16", True, T, gpu_device)
    plan = _plan(codes, scales, off, K, group, gpu_device)
    want, bound = _want(codes, scales, off, x, group)
    for lead, ldx, ldy in ((0, K, M), (1, K + 2, M + 1), (3, K + 11, M + 90), (8, 344, 72)):
        xs = torch.full((T * ldx + 16,), float("nan"), dtype=torch.bfloat16, device=gpu_device)
        ys = torch.full((T * ldy + 16,), 77.0, dtype=torch.bfloat16, device=gpu_device)
        xv, yv = xs[lead:lead + T * ldx].view(T, ldx)[:, :K], ys[lead:lead + T * ldy].view(T, ldy)[:, :M]
        xv.copy_(x)
        pkg.ppmv_run(plan, xv, yv)
        _near(yv, want, bound, "bfloat16")
        yv.fill_(77.0)
        assert (ys == 77.0).all()
    row = x[:1].to(gpu_device).expand(T, K)
    y = torch.empty((T, M), dtype=torch.bfloat16, device=gpu_device)
    pkg.ppmv_run(plan, row, y)
    _near(y, np.repeat(want[:1], T, 0), np.repeat(bound[:1], T, 0), "bfloat16")


@pytest.mark.parametrize("T", (1, 20, 100))
def test_a_bad_token_stays_alone(gpu_device, T):
    """A token that is not finite spoils its own results and no other's; its padding (K is no multiple of anything) neither."""
    import torch

    import paper_2601_18511_amd as pkg

    M, K, group = 50, 170, 32
    for dtype in TYPES:
        codes, scales, off, x = _case(M, K, T, group, dtype, False, 3, gpu_device)
        plan = _plan(codes, scales, off, K, group, gpu_device)
        y = torch.empty((T, M), dtype=x.dtype, device=gpu_device)
        clean = torch.empty_like(y)
        pkg.ppmv_run(plan, x.to(gpu_device), clean)
        for bad in (float("nan"), float("inf")):
            x[T // 2, K - 1] = bad
            pkg.ppmv_run(plan, x.to(gpu_device), y)
            assert not torch.isfinite(y[T // 2].float()).any()
            keep = torch.arange(T, device=gpu_device) != T // 2
            assert torch.equal(y[keep], clean[keep])


def test_extreme_codes_and_sums(gpu_device):
    """All codes 0 or 15, activations that cancel: integers that every format holds, so the results are exact."""
    import torch

    import paper_2601_18511_amd as pkg

    M, K = 32, 512
    for dtype in TYPES:
        t = getattr(torch, dtype)
        for T in (1, 40, 100):
            codes = torch.full((M, K // 2), 0xF0, dtype=torch.uint8)           # even k: -8, odd k: 7
            scales = torch.full((M, K // 32), 0.5, dtype=t)
            x = torch.ones((T, K), dtype=t)
            x[:, 1::2] = -1.0
            x[:, 2::4] = 1.0
            y = torch.empty((T, M), dtype=t, device=gpu_device)
            pkg.ppmv_run(_plan(codes, scales, None, K, 32, gpu_device), x.to(gpu_device), y)
            assert (y == -0.5 * (8 + 7) * (K // 2)).all()


def test_no_tokens_and_refusals(gpu_device):
    import torch

    import paper_2601_18511_amd as pkg

    codes, scales, off, x = _case(24, 100, 4, 32, "bfloat16", False, 1, gpu_device)
    plan = _plan(codes, scales, off, 100, 32, gpu_device)
    dx, y = x.to(gpu_device), torch.empty((4, 24), dtype=torch.bfloat16, device=gpu_device)
    pkg.ppmv_run(plan, dx[:0], y[:0])
    for bad_x, bad_y in ((dx, y[:3]), (dx[:, :99], y), (dx, y[:, :23]), (dx.half(), y), (dx, y.half()), (x, y), (dx.t().contiguous().t(), y), (dx[0], y)):
        with pytest.raises(ValueError):
            pkg.ppmv_run(plan, bad_x, bad_y)
        with pytest.raises(ValueError):
            pkg.ppmv_gated_run(plan, plan, bad_x, bad_y)
    with pytest.raises(pkg.PcmmError):
        pkg.ppmv_run(plan, dx, y[:1].expand(4, 24))                        # results on top of each other
    for other in (_case(24, 100, 1, 64, "bfloat16", False, 1, gpu_device), _case(25, 100, 1, 32, "bfloat16", False, 1, gpu_device),
                  _case(24, 100, 1, 32, "float16", False, 1, gpu_device), _case(24, 100, 1, 32, "bfloat16", True, 1, gpu_device)):
        o = _plan(*other[:3], 100, 64 if other[1].shape[1] == 2 else 32, gpu_device)
        with pytest.raises(pkg.PcmmError) as e:
            pkg.ppmv_gated_run(plan, o, dx, y)
        assert e.value.status == pkg.pcmm.PCMM_EINVAL
    for bad in (lambda: pkg.ppmv_plan_create(codes.to(gpu_device), scales.to(gpu_device), 102, 32),
                lambda: pkg.ppmv_plan_create(codes.to(gpu_device), scales.to(gpu_device)[:, :3], 100, 32),
                lambda: pkg.ppmv_plan_create(codes.to(gpu_device), scales.to(gpu_device).float(), 100, 32),
                lambda: pkg.ppmv_plan_create(codes.to(gpu_device), scales.to(gpu_device), 100, 16),
                lambda: pkg.ppmv_plan_create(codes.to(gpu_device), scales.to(gpu_device), 100, 32, offsets=scales.half().to(gpu_device))):
        with pytest.raises(ValueError):
            bad()
    assert pkg.ppmv_plan_workspace_bytes(plan) > 0
    pkg.ppmv_plan_destroy(plan)
    pkg.ppmv_plan_destroy(plan)
    with pytest.raises(ValueError):
        pkg.ppmv_run(plan, dx, y)


@pytest.mark.parametrize("T", (1, 40, 200))
def test_streams_and_graphs(gpu_device, T):
    """Two runs of one plan at once on two streams, and a captured run replayed on new inputs."""
    import torch

    import paper_2601_18511_amd as pkg

    M, K, group = 300, 900, 128
    codes, scales, off, x = _case(M, K, T, group, "float16", True, 9, gpu_device)
    plan = _plan(codes, scales, off, K, group, gpu_device)
    a, b = x.to(gpu_device), (-x).to(gpu_device)
    want = [torch.empty((T, M), dtype=torch.float16, device=gpu_device) for _ in range(2)]
    pkg.ppmv_run(plan, a, want[0])
    pkg.ppmv_run(plan, b, want[1])
    torch.cuda.synchronize()
    s = [torch.cuda.Stream() for _ in range(2)]
    got = [torch.zeros_like(w) for w in want]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, src in enumerate((a, b)):
            pkg.ppmv_run(plan, src, got[i], stream=s[i])
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    src, dst, gated = a.clone(), torch.zeros_like(want[0]), torch.zeros_like(want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkg.ppmv_run(plan, src, dst)
        pkg.ppmv_gated_run(plan, plan, src, gated)
    eager = torch.empty_like(dst)
    for i, new in enumerate((a, b, a)):
        src.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        pkg.ppmv_gated_run(plan, plan, new, eager)
        assert torch.equal(dst, want[i % 2]) and torch.equal(gated, eager)


# M, K, T, group: more rows than sixteen tokens a work-group are taken for; x shared by two waves (16 to 64 tokens and more than
# one such batch) and by four, and large tiles
BATCHES = [(2100, 1000, 20, 64), (2100, 333, 40, 32), (2051, 640, 57, 128), (2100, 264, 150, 32), (13000, 200, 20, 128), (13000, 136, 40, 32),
           (13000, 328, 64, 64), (8300, 300, 9, 64), (12400, 300, 300, 64), (12400, 392, 300, 32), (12400, 264, 300, 128)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gated", (False, True))
@pytest.mark.parametrize("M,K,T,group", BATCHES)
def test_batches_of_tokens_and_many_rows(gpu_device, M, K, T, group, gated, dtype):
    """Against the oracle, with rows aligned to 16 bytes and to two only; nothing beside the result is written, and a token that is
    not finite spoils no other's results."""
    import torch

    import paper_2601_18511_amd as pkg

    for offsets in (False, True):
        codes, scales, off, x = _case(M, K, T, group, dtype, offsets, M + K + T, gpu_device)
        plan = _plan(codes, scales, off, K, group, gpu_device)
        want, bound = _want(codes, scales, off, x, group)
        if gated:
            bound = 2.2 * bound * (np.abs(want) + bound + 1) + np.abs(want * want) * (np.abs(want) + 8) * 2.0 ** -22
            want = oracle.silu(want) * want
        for lead, ldx, ldy in ((0, -(-K // 8) * 8, M), (1, K + 3, M + 5)):
            xs = torch.full((T * ldx + 16,), float("nan"), dtype=x.dtype, device=gpu_device)
            ys = torch.full((T * ldy + 16,), 77.0, dtype=x.dtype, device=gpu_device)
            xv, yv = xs[lead:lead + T * ldx].view(T, ldx)[:, :K], ys[lead:lead + T * ldy].view(T, ldy)[:, :M]
            xv.copy_(x)
            run = (lambda: pkg.ppmv_gated_run(plan, plan, xv, yv)) if gated else (lambda: pkg.ppmv_run(plan, xv, yv))
            run()
            _near(yv, want, bound, dtype)
            clean = yv.clone()
            assert (ys[:lead] == 77).all() and (ys[lead + T * ldy:] == 77).all()
            assert (ys[lead:lead + T * ldy].view(T, ldy)[:, M:] == 77).all()
            xv[T - 2, K - 1] = float("nan")
            run()
            assert torch.isnan(yv[T - 2]).all()
            assert torch.equal(yv[:T - 2], clean[:T - 2]) and torch.equal(yv[T - 1], clean[T - 1])
