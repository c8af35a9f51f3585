"""The 4-bit K/V cache and attention over it on the GPU against the oracle in 64 bits.

The cache: codes, scales and offsets are whole numbers and bf16 values by definition, so the values read back are the oracle's,
rounded once to the type they are read in; they are compared exactly.

Attention.  With n keys, V the largest |s| 31 + |b| of the values, and a score's sum of at most D terms of magnitude
|q| (31 s + |b|): a score is off by at most (D + 16) 2^-23 times that sum's magnitude times the scale, dS; the exponentials and the
two sums over the keys by n 2^-23 relative and more; the probabilities enter the second product in two halves of 8 bits each, 2^-15.
Hence |out - exact| <= V (2 dS + 2^-15 + (n + 64) 2^-22), and the rounding of the result, half a step."""
import numpy as np
import pytest

from oracle import clear_oracle as oracle

pytestmark = pytest.mark.gpu
TYPES = ("bfloat16", "float16")


class Batch:
    """Sequences of (new tokens, all tokens), their K and V, and a cache whose pages lie in random order."""

    def __init__(self, seqs, heads, kv_heads, D, page, dtype, dev, seed=0, spare=2, lead=0, tail=0):
        import torch

        import paper_2601_18511_amd as pkg

        g = torch.Generator().manual_seed(seed)
        t = getattr(torch, dtype)
        self.seqs, self.D, self.dtype, self.page = seqs, D, dtype, page
        self.lead, self.tokens = lead, lead + sum(n for n, _ in seqs) + tail
        self.k = [(torch.randn((n, kv_heads, D), generator=g) + torch.randn((kv_heads, D), generator=g)).to(t) for _, n in seqs]
        self.v = [torch.randn((n, kv_heads, D), generator=g).to(t) for _, n in seqs]
        self.q = torch.randn((self.tokens, heads, D), generator=g).to(t)
        width = max(1, max(-(-n // page) for _, n in seqs)) + spare
        pages = len(seqs) * width
        self.table = torch.randperm(pages, generator=g).to(torch.int32).view(len(seqs), width)
        self.cache = pkg.ppkv_cache_create(pages, page, kv_heads, D, device=dev)
        self.cache.pool.fill_(255)                      # whatever the pool holds before: NaN scales among it
        self.dev = dev
        starts = [lead]
        for n, _ in seqs:
            starts.append(starts[-1] + n)
        self.starts_host = starts
        self.starts = torch.tensor(starts, dtype=torch.int32, device=dev)
        self.lens = torch.tensor([n for _, n in seqs], dtype=torch.int32, device=dev)
        self.dtable = self.table.to(dev)

    def where(self):
        return self.starts, self.lens, self.dtable

    def everything(self):
        """(starts, lens, table) of all cached tokens as new ones"""
        import torch

        starts = np.concatenate([[0], np.cumsum([n for _, n in self.seqs])])
        return torch.tensor(starts, dtype=torch.int32, device=self.dev), self.lens, self.dtable

    def fill(self):
        import torch

        import paper_2601_18511_amd as pkg

        pkg.ppkv_append(self.cache, torch.cat(self.k).to(self.dev), torch.cat(self.v).to(self.dev), *self.everything())
        return self

    def check_attention(self, out, causal=True, scale=None, touched=None):
        import torch

        half = torch.finfo(getattr(torch, self.dtype)).eps / 2
        scale = self.D ** -0.5 if scale is None else scale
        got = out.double().cpu().numpy()
        for (t, n), first, k, v in zip(self.seqs, self.starts_host, self.k, self.v):
            if t == 0:
                continue
            q = self.q[first:first + t].double().numpy()
            hk, hv = oracle.held(k.double().numpy()), oracle.held(v.double().numpy())
            want = oracle.attention(q, hk, hv, scale, causal)
            off = np.abs(got[first:first + t] - want)
            if n:
                _, ks, kb = oracle.quantise(k.double().numpy())
                _, vs, vb = oracle.quantise(v.double().numpy())
                G = q.shape[1] // k.shape[1]
                reach = np.repeat(31 * ks + np.abs(kb), 32, -1).max(0).repeat(G, 0)          # [heads][D]
                dS = (self.D + 16) * 2.0 ** -23 * (np.abs(q) * reach).sum(-1) * abs(scale)
                V = (31 * vs + np.abs(vb)).max()
                bound = V * (2 * dS + 2.0 ** -15 + (n + 64) * 2.0 ** -22)[..., None]
            else:
                bound = 0.0
            assert (off <= half * np.abs(want) + bound + 2.0 ** -25).all(), (t, n, float((off - half * np.abs(want) - bound).max()))


def _attend(b, causal=True, scale=None, fill=None, max_len=0, out=None):
    import torch

    import paper_2601_18511_amd as pkg

    q = b.q.to(b.dev)
    out = torch.full_like(q, float("nan") if fill is None else fill) if out is None else out
    pkg.ppkv_attention(b.cache, q, out, *b.where(), max_q=max([t for t, _ in b.seqs] + [1]), max_len=max_len, causal=causal, scale=scale)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("page", (16, 48, 128))
def test_values_read_back_are_the_formats(gpu_device, dtype, D, page):
    """Every token of every sequence, written in two calls (a prompt, then a few tokens of some sequences), read in one."""
    import torch

    import paper_2601_18511_amd as pkg

    b = Batch([(3, 70), (0, 5), (1, 1), (16, 16), (7, 129)], 3, 3, D, page, dtype, gpu_device, seed=D + page)
    old = [n - t for t, n in b.seqs]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=gpu_device)  # noqa: E731
    pkg.ppkv_append(b.cache, torch.cat([x[:n] for x, n in zip(b.k, old)]).to(gpu_device), torch.cat([x[:n] for x, n in zip(b.v, old)]).to(gpu_device),
                    i32(np.concatenate([[0], np.cumsum(old)])), i32(old), b.dtable)
    pkg.ppkv_append(b.cache, torch.cat([x[n:] for x, n in zip(b.k, old)]).to(gpu_device), torch.cat([x[n:] for x, n in zip(b.v, old)]).to(gpu_device), *b.where())
    for out_type in (torch.bfloat16, torch.float16, torch.int16):
        k, v = (torch.zeros((sum(n for _, n in b.seqs), 3, D), dtype=out_type, device=gpu_device) for _ in range(2))
        pkg.ppkv_read(b.cache, k, v, *b.everything(), frac_bits=10 if out_type == torch.int16 else 0)
        for got, src in ((k, b.k), (v, b.v)):
            held = oracle.held(torch.cat(src).double().numpy())
            if out_type == torch.int16:
                want = torch.from_numpy(np.clip(np.rint(held.astype(np.float32).astype(np.float64) * 1024), -32768, 32639)).to(torch.int16)
            else:
                want = torch.from_numpy(held).float().to(out_type)
            assert torch.equal(got.cpu(), want)


def test_values_next_to_borders_and_extreme_groups(gpu_device):
    """Values on and next to the border between two codes, groups without a range, with tiny and huge ones, and with NaN and infinities."""
    import torch

    import paper_2601_18511_amd as pkg

    rng = np.random.default_rng(2)
    x = np.zeros((40, 1, 128))
    for i in range(40):
        for j in range(4):
            unit = 2.0 ** rng.integers(-20, 20)
            x[i, 0, 32 * j:32 * j + 32] = unit * (rng.integers(0, 31, 32) / 2.0 + rng.choice([0, 2.0 ** -6, -2.0 ** -6], 32))
            x[i, 0, 32 * j:32 * j + 2] = 0.0, 15.0 * unit
    x[0, 0, :32] = 3.25
    x[1, 0, :32] = 0.0
    x[2, 0, 5] = np.nan
    x[3, 0, 40] = np.inf
    x[4, 0, 70] = -np.inf
    x[5, 0, :32] = rng.standard_normal(32) * 2.0 ** -130
    x[6, 0, :32] = np.where(rng.random(32) < 0.5, 3e38, -3e38)
    x[7, 0, :32] = 100.0 + rng.random(32)
    for dtype in TYPES:
        t = torch.from_numpy(x).to(getattr(torch, dtype)) if dtype == "bfloat16" else torch.from_numpy(np.clip(x, -6e4, 6e4)).half()
        cache = pkg.ppkv_cache_create(3, 16, 1, 128, device=gpu_device)
        cache.pool.fill_(255)
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=gpu_device)  # noqa: E731
        where = i32([0, 40]), i32([40]), i32([[2, 0, 1]])
        pkg.ppkv_append(cache, t.to(gpu_device), t.to(gpu_device), *where)
        k, v = torch.empty((40, 1, 128), dtype=torch.bfloat16, device=gpu_device), torch.empty((40, 1, 128), dtype=torch.bfloat16, device=gpu_device)
        pkg.ppkv_read(cache, k, v, *where)
        want = torch.from_numpy(oracle.held(t.double().numpy())).float().bfloat16()
        assert torch.equal(torch.nan_to_num(k.cpu(), nan=1234.0), torch.nan_to_num(want, nan=1234.0))
        assert torch.equal(torch.nan_to_num(v.cpu(), nan=1234.0), torch.nan_to_num(want, nan=1234.0))
        fixed = torch.empty((40, 1, 128), dtype=torch.int16, device=gpu_device)
        pkg.ppkv_read(cache, fixed, None, *where, frac_bits=30)             # everything saturates or is rounded
        held = oracle.held(t.double().numpy()).astype(np.float32).astype(np.float64)
        assert torch.equal(fixed.cpu(), torch.from_numpy(np.nan_to_num(np.clip(np.rint(held * 2.0 ** 30), -32768, 32639), nan=0.0)).to(torch.int16))


SEQS = {
    "one_key": [(1, 1)],
    "tokens": [(1, 1), (1, 17), (1, 64), (1, 65), (1, 1000)],
    "ragged": [(3, 70), (0, 5), (1, 1), (16, 16), (7, 129), (0, 0), (2, 2)],
    "turns": [(40, 300), (33, 33), (1, 513)],
    "prompt": [(150, 150)],
    "more_new_than_held": [(6, 2), (4, 0), (3, 3)],
}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", sorted(SEQS))
@pytest.mark.parametrize("heads,kv_heads,D,page", [(4, 4, 64, 16), (8, 2, 128, 48), (7, 1, 64, 32), (32, 8, 128, 64), (34, 2, 128, 16)])
def test_attention_matches_the_oracle(gpu_device, name, heads, kv_heads, D, page, dtype):
    for causal in (True, False):
        if name == "more_new_than_held":        # every token is held from its own place on: the ones in front have none
            b = Batch([(t, max(n, 0)) for t, n in SEQS[name]], heads, kv_heads, D, page, dtype, gpu_device, seed=3)
        else:
            b = Batch(SEQS[name], heads, kv_heads, D, page, dtype, gpu_device, seed=len(name) + heads)
        b.fill()
        b.check_attention(_attend(b, causal), causal)


@pytest.mark.parametrize("dtype", TYPES)
def test_long_sequences(gpu_device, dtype):
    """Long enough to be divided among work-groups, with every kind of expectation of the length."""
    import torch

    b = Batch([(1, 5000), (2, 3), (1, 2049), (5, 700)], 8, 2, 128, 16, dtype, gpu_device, seed=4)
    b.fill()
    for max_len in (0, 5000, 100, 1 << 20):
        b.check_attention(_attend(b, max_len=max_len))
    assert torch.isfinite(_attend(b).float()).all()


def test_scales_and_large_scores(gpu_device):
    """Scores far apart (one key takes all), all alike (scale 0), and of the other sign."""
    b = Batch([(2, 200), (20, 90)], 4, 2, 64, 32, "bfloat16", gpu_device, seed=6).fill()
    for scale in (0.0, 30.0, -0.5, 1e-3):
        b.check_attention(_attend(b, scale=scale), scale=scale)


def test_rows_of_no_sequence_are_left(gpu_device):
    import torch

    b = Batch([(2, 40), (3, 10)], 4, 2, 64, 16, "bfloat16", gpu_device, seed=7, lead=3, tail=9).fill()
    out = _attend(b, fill=55.0)
    b.check_attention(out)
    assert (out[:3] == 55.0).all() and (out[8:] == 55.0).all()
    import paper_2601_18511_amd as pkg

    k = torch.full((17, 2, 64), 55.0, dtype=torch.bfloat16, device=gpu_device)
    pkg.ppkv_read(b.cache, k, None, *b.where())
    assert (k[:3] == 55.0).all() and (k[8:] == 55.0).all() and (k[3:8] != 55.0).any()
    # rows beyond max_q are left too
    few = torch.full_like(out, 55.0)
    pkg.ppkv_attention(b.cache, b.q.to(gpu_device), few, *b.where(), max_q=2)
    assert torch.equal(few[3:7], out[3:7]) and (few[7] == 55.0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_alignment(gpu_device, dtype):
    """Heads outside, gaps between rows, an odd first element; the same results, and nothing written between them."""
    import torch

    import paper_2601_18511_amd as pkg

    b = Batch([(3, 40), (1, 100), (20, 20)], 4, 2, 64, 16, dtype, gpu_device, seed=8)
    keys, values = torch.cat(b.k).to(gpu_device), torch.cat(b.v).to(gpu_device)
    n = keys.shape[0]
    wide = torch.full((2 * n * 70 + 1,), float("nan"), dtype=keys.dtype, device=gpu_device)
    kk = wide[1:].view(2, n, 70)[:, :, 3:67].transpose(0, 1)               # [tokens][heads][D], heads outside, two-byte alignment
    kk.copy_(keys)
    pkg.ppkv_append(b.cache, kk, values, *b.everything())
    plain = _attend(b)
    b.check_attention(plain)
    q = torch.zeros((4, b.tokens, 67), dtype=keys.dtype, device=gpu_device)[:, :, 1:65].transpose(0, 1)
    q.copy_(b.q)
    buf = torch.full((4, b.tokens, 67), 9.0, dtype=keys.dtype, device=gpu_device)
    out = buf[:, :, 3:].transpose(0, 1)
    pkg.ppkv_attention(b.cache, q, out, *b.where(), max_q=20)
    assert torch.equal(out, plain)
    out.fill_(9.0)
    assert (buf == 9.0).all()
    r = torch.full((2, n, 65), 9.0, dtype=torch.int16, device=gpu_device)
    want = torch.zeros((n, 2, 64), dtype=torch.int16, device=gpu_device)
    pkg.ppkv_read(b.cache, want, None, *b.everything(), frac_bits=8)
    pkg.ppkv_read(b.cache, None, r[:, :, :64].transpose(0, 1), *b.everything(), frac_bits=8)
    pkg.ppkv_read(b.cache, r[:, :, :64].transpose(0, 1), None, *b.everything(), frac_bits=8)
    assert torch.equal(r[:, :, :64].transpose(0, 1), want) and (r[:, :, 64] == 9).all()
    # one query row for every token and head
    one = b.q[:1, :1].to(gpu_device).expand(b.tokens, 4, 64)
    b.q = one.cpu()
    pkg.ppkv_attention(b.cache, one, out, *b.where(), max_q=20)
    b.check_attention(out)


@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_not_attended_to_has_no_part(gpu_device, dtype):
    """NaN and infinities in tokens behind a causal row, behind the sequence and in the pool's unused places do not reach a result;
    a NaN that a row attends to does."""
    import torch

    import paper_2601_18511_amd as pkg

    for t, n, bad in ((30, 30, 17), (5, 100, 97), (100, 260, 200)):
        b = Batch([(t, n)], 4, 2, 64, 16, dtype, gpu_device, seed=9)
        clean = _attend(b.fill())
        b.check_attention(clean)
        for which in ("k", "v"):
            for value in (float("nan"), float("inf"), -float("inf")):
                spoiled = Batch([(t, n)], 4, 2, 64, 16, dtype, gpu_device, seed=9)
                getattr(spoiled, which)[0][bad, 1, 40] = value              # head 1, channels 32..63
                out = _attend(spoiled.fill())
                row = bad - (n - t)                                         # the first row that attends to it
                assert torch.equal(out[:row], clean[:row])
                assert torch.equal(out[:, :2], clean[:, :2])                # the other head's queries
                hit = out[row:, 2:]
                if which == "k":
                    assert torch.isnan(hit).all()
                else:
                    assert torch.isnan(hit[..., 32:]).all() and torch.equal(hit[..., :32], clean[row:, 2:, :32])


@pytest.mark.parametrize("D", (64, 128))
def test_rows_that_attend_to_nothing_but_nan(gpu_device, D):
    """Every key that a row attends to is a NaN: the row is NaN, not the zeros of a row without keys; one token, a tile, several splits."""
    import torch

    for t, n, max_len in ((1, 1, 0), (1, 64, 0), (1, 3000, 3000), (40, 90, 0), (3, 2, 0)):
        b = Batch([(t, n)], 4, 2, D, 16, "bfloat16", gpu_device, seed=12)
        b.k[0][:, 0, 5] = float("nan")
        out = _attend(b.fill(), max_len=max_len).cpu()
        empty = max(t - n, 0)                                               # causal rows in front of the first token
        assert (out[:empty] == 0).all()
        assert torch.isnan(out[empty:, :2]).all(), (t, n)
        assert not torch.isnan(out[:, 2:]).any()


def test_bad_pages_and_lengths_stay_inside(gpu_device):
    """Page numbers outside the pool, lengths beyond the table and below zero, starts that do not ascend: nothing is written outside,
    such tokens are not attended to."""
    import torch

    import paper_2601_18511_amd as pkg

    b = Batch([(4, 64), (2, 48)], 4, 2, 64, 16, "bfloat16", gpu_device, seed=10)
    b.fill()
    pool = b.cache.pool.clone()
    table = b.dtable.clone()
    table[0, 1], table[0, 2], table[1, 0] = -1, b.cache.pages, 1 << 30
    out = torch.zeros_like(b.q, device=gpu_device)
    pkg.ppkv_attention(b.cache, b.q.to(gpu_device), out, b.starts, b.lens, table, max_q=4)
    keep = [list(range(16)) + list(range(48, 64)), list(range(16, 48))]
    for s, (t, n) in enumerate(b.seqs):
        k, v = oracle.held(b.k[s].double().numpy())[keep[s]], oracle.held(b.v[s].double().numpy())[keep[s]]
        first = b.starts_host[s]
        for i in range(t):
            last = n - t + i
            m = sum(x <= last for x in keep[s])
            want = oracle.attention(b.q[first + i:first + i + 1].double().numpy(), k[:m], v[:m], 0.125, False)
            assert np.abs(out[first + i].double().cpu().numpy() - want[0]).max() < 2.0 ** -6 * np.abs(v).max()
    bad = [(b.starts, b.lens, table), (b.starts, b.lens + 1000, b.dtable), (b.starts, b.lens - 1000, b.dtable),
           (b.starts.flip(0).contiguous(), b.lens, b.dtable), (b.starts + 100, b.lens, b.dtable), (b.starts - 100, b.lens, b.dtable),
           (b.starts, torch.full_like(b.lens, 0x7fffffff), b.dtable), (b.starts, torch.full_like(b.lens, -0x80000000), b.dtable),
           (torch.tensor([-0x80000000, 0, 0x7fffffff], dtype=torch.int32, device=gpu_device), b.lens, b.dtable)]
    x = torch.randn((6, 2, 64), dtype=torch.bfloat16, device=gpu_device)
    for where in bad:
        pkg.ppkv_attention(b.cache, b.q.to(gpu_device), out, *where, max_q=4)
        pkg.ppkv_read(b.cache, torch.empty_like(x), torch.empty_like(x), *where)
        pkg.ppkv_append(b.cache, x, x, *where)
        torch.cuda.synchronize()
        b.cache.pool.copy_(pool)
    # a token without a place reads as zeros and is not written
    r = torch.full_like(x, 3.0)
    pkg.ppkv_read(b.cache, r, None, b.starts, b.lens + 1000, b.dtable)
    assert (r == 0).all()
    pkg.ppkv_append(b.cache, x, x, b.starts, b.lens + 1000, b.dtable)
    assert torch.equal(b.cache.pool, pool)


@pytest.mark.parametrize("seqs", ([(1, 3000), (1, 20)], [(70, 200)]))
def test_streams_and_graphs(gpu_device, seqs):
    """Two calls over one cache at once, each with scratch of its own; a captured step (write, attend) replayed with eager calls between."""
    import torch

    import paper_2601_18511_amd as pkg

    b = Batch(seqs, 8, 2, 128, 16, "bfloat16", gpu_device, seed=11).fill()
    most = max(t for t, _ in seqs)
    q = [b.q.to(gpu_device), -b.q.to(gpu_device)]
    want = [torch.empty_like(x) for x in q]
    for i in range(2):
        pkg.ppkv_attention(b.cache, q[i], want[i], *b.where(), max_q=most)
    got = [torch.zeros_like(x) for x in q]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(4):
        for i in range(2):
            pkg.ppkv_attention(b.cache, q[i], got[i], *b.where(), max_q=most, stream=streams[i])
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    k, v = (torch.cat([x[n - t:] for x, (t, n) in zip(y, seqs)]).to(gpu_device) for y in (b.k, b.v))
    src, dst = q[0].clone(), torch.zeros_like(q[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkg.ppkv_append(b.cache, k, v, *b.where())
        pkg.ppkv_attention(b.cache, src, dst, *b.where(), max_q=most)
    other = torch.cuda.CUDAGraph()
    dst2 = torch.zeros_like(dst)
    with torch.cuda.graph(other):
        pkg.ppkv_attention(b.cache, q[1], dst2, *b.where(), max_q=most)
    for i in (0, 1, 0):
        src.copy_(q[i])
        graph.replay()
        other.replay()
        torch.cuda.synchronize()
        assert torch.equal(dst, want[i]) and torch.equal(dst2, want[1])
        eager = torch.empty_like(dst)
        pkg.ppkv_attention(b.cache, q[1 - i], eager, *b.where(), max_q=most)
        assert torch.equal(eager, want[1 - i])


def test_the_last_tokens_of_a_padded_batch(gpu_device):
    """Keys, values and queries as views of the last token of [batch][tokens][heads][channels] arrays: far apart rows."""
    import torch

    import paper_2601_18511_amd as pkg

    b = Batch([(1, n) for n in (5, 40, 17)], 8, 2, 128, 16, "bfloat16", gpu_device, seed=13).fill()
    want = _attend(b)
    b.check_attention(want)
    big = [torch.zeros((3, 1000, h, 128), dtype=torch.bfloat16, device=gpu_device) for h in (2, 2, 8, 8)]
    for dst, src in zip(big, (torch.stack([x[-1] for x in b.k]), torch.stack([x[-1] for x in b.v]), b.q)):
        dst[:, -1].copy_(src)
    pkg.ppkv_append(b.cache, big[0][:, -1], big[1][:, -1], *b.where())
    pkg.ppkv_attention(b.cache, big[2][:, -1], big[3][:, -1], *b.where(), max_q=1)
    assert torch.equal(big[3][:, -1], want) and (big[3][:, :-1] == 0).all()


def test_many_sequences_and_shared_pages(gpu_device):
    """More sequences than a wave has lanes, all over the same public prefix: its pages stand in every row of the table."""
    import torch

    import paper_2601_18511_amd as pkg

    n, B, page = 48, 300, 16
    b = Batch([(1, n)], 4, 2, 64, page, "float16", gpu_device, seed=14).fill()
    q = torch.randn((B, 4, 64), dtype=torch.float32).half()
    starts = torch.arange(B + 1, dtype=torch.int32, device=gpu_device)
    lens = torch.full((B,), n, dtype=torch.int32, device=gpu_device)
    table = b.dtable.expand(B, -1).contiguous()
    out = torch.empty_like(q, device=gpu_device)
    pkg.ppkv_attention(b.cache, q.to(gpu_device), out, starts, lens, table, max_q=1)
    for i in (0, 1, 63, 64, 65, 255, 299):
        b.q = q[i:i + 1]
        b.check_attention(out[i:i + 1])
    k = torch.zeros((B, 2, 64), dtype=torch.float16, device=gpu_device)
    pkg.ppkv_read(b.cache, k, None, starts, lens, table)
    want = torch.from_numpy(oracle.held(b.k[0][-1:].double().numpy())).float().half()
    assert torch.equal(k.cpu(), want.expand(B, 2, 64))


def test_refusals(gpu_device):
    import torch

    import paper_2601_18511_amd as pkg

    b = Batch([(2, 20)], 4, 2, 64, 16, "bfloat16", gpu_device, seed=12)
    k, q = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device=gpu_device), b.q.to(gpu_device)
    s, n, t = b.where()
    for bad in (k.float(), k[:, :1], k[:, :, :32], k.cpu(), k[0], k.transpose(1, 2).contiguous().transpose(1, 2), k.half()):
        with pytest.raises(ValueError):
            pkg.ppkv_append(b.cache, bad, k, s, n, t)
        with pytest.raises(ValueError):
            pkg.ppkv_read(b.cache, bad, k, s, n, t)
    for where in ((s[:1], n, t), (s.long(), n, t), (s, n, t[0]), (s, n, torch.cat((t, t))), (s.cpu(), n, t), (s, n, t[:, ::2])):
        with pytest.raises(ValueError):
            pkg.ppkv_append(b.cache, k, k, *where)
        with pytest.raises(ValueError):
            pkg.ppkv_attention(b.cache, q, torch.empty_like(q), *where, max_q=2)
    for bad_q, bad_out in ((q, q[:1]), (q[:, :3], q[:, :3].clone()), (q, q.half()), (q.cpu(), q), (q[:, :, :32], q)):
        with pytest.raises(ValueError):
            pkg.ppkv_attention(b.cache, bad_q, bad_out, s, n, t, max_q=2)
    with pytest.raises(ValueError):
        pkg.ppkv_read(b.cache, None, None, s, n, t)
    for call in (lambda: pkg.ppkv_attention(b.cache, q, q, s, n, t, max_q=2), lambda: pkg.ppkv_attention(b.cache, q, torch.empty_like(q), s, n, t, max_q=-1),
                 lambda: pkg.ppkv_read(b.cache, k[:1].expand(2, 2, 64), None, s, n, t), lambda: pkg.ppkv_read(b.cache, k, None, s, n, t, frac_bits=3)):
        with pytest.raises(pkg.PcmmError) as e:
            call()
        assert e.value.status == pkg.pcmm.PCMM_EINVAL
    pkg.ppkv_append(b.cache, k[:0], k[:0], s, n, t)
    pkg.ppkv_attention(b.cache, q[:0], q[:0].clone(), s, n, t, max_q=2)
