"""The operators of the clear track, as they are measured: products with 4-bit weights, the gated feed-forward products, the
4-bit K/V cache and attention over it.

A mixed prompt has a public prefix, which runs in the clear with the same weights as the encrypted suffix and leaves a public K/V
cache.  Kinds of cases:

  ppmv        y = x W^T with W in 4 bits and group scales
  gated       h = silu(x Wg^T) * (x Wu^T), both weights in 4 bits
  cache       K and V of new tokens quantised into the paged cache, and read back as values
  attention   softmax attention over the paged 4-bit cache

`own` false: the plain form, elementary torch operations in 32 bits.  `own` true: the library's calls.
"""
import math
import random

import torch

own = False

# Model dimensions of the layers: hidden 4096, intermediate 14336, 32 heads of 128, K/V projections of 1024 (8 heads).
HIDDEN, INTER, HEAD, KV = 4096, 14336, 128, 1024
PROMPT = 3968                       # public tokens of the long prompt
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
GROUP = 32                          # channels of a K or V vector that share a scale and an offset


def _ppmv(name, M, K, T, group, dtype, offsets=False, kind="ppmv"):
    return {"name": name, "kind": kind, "M": M, "K": K, "T": T, "group": group, "dtype": dtype, "offsets": offsets}


def _attention(name, batch, heads, kv_heads, head_dim, q_max, len_min, len_max, page, causal, dtype):
    return {"name": name, "kind": "attention", "batch": batch, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "q_max": q_max, "len_min": len_min, "len_max": len_max, "page": page, "causal": causal, "dtype": dtype}


def _cache(name, batch, kv_heads, head_dim, q_max, len_min, len_max, page, dtype):
    return {"name": name, "kind": "cache", "batch": batch, "kv_heads": kv_heads, "head_dim": head_dim,
            "q_max": q_max, "len_min": len_min, "len_max": len_max, "page": page, "dtype": dtype}


def listed():
    return [
        # K (or V) projection of one public token: the smallest product of a layer, latency counts
        _ppmv("kv_proj_token", KV, HIDDEN, 1, 128, "bf16"),
        # down projection of one token: the longest contraction
        _ppmv("down_token", HIDDEN, INTER, 1, 128, "bf16"),
        # a pruned layer of odd sizes with zero points, a few tokens of a chat turn
        _ppmv("ragged_turn", 1000, 777, 13, 32, "fp16", True),
        # output projection of the whole public prompt
        _ppmv("o_proj_prompt", HIDDEN, HIDDEN, PROMPT, 128, "bf16"),
        # gate and up projection of one token: half of a layer's weights
        _ppmv("gate_up_token", INTER, HIDDEN, 1, 64, "bf16", kind="gated"),
        # the same for a batch of requests, one token each
        _ppmv("gate_up_batch", INTER, HIDDEN, 48, 128, "fp16", kind="gated"),
        # and for the whole public prompt: the largest case
        _ppmv("gate_up_prompt", INTER, HIDDEN, PROMPT, 128, "bf16", kind="gated"),
        # one new public token for each of sixteen requests
        _cache("cache_token", 16, 8, HEAD, 1, 100, 4096, 16, "bf16"),
        # the public prompt written at once
        _cache("cache_prompt", 1, 8, HEAD, PROMPT, PROMPT, PROMPT, 64, "bf16"),
        # one token over the public prompt
        _attention("attend_token", 1, 32, 8, HEAD, 1, PROMPT, PROMPT, 64, True, "bf16"),
        # requests of very different lengths, one token each
        _attention("attend_batch", 32, 32, 8, HEAD, 1, 50, 16384, 16, True, "fp16"),
        # the public prompt over itself
        _attention("attend_prompt", 1, 32, 8, HEAD, PROMPT, PROMPT, PROMPT, 64, True, "bf16"),
    ]


# ---------------------------------------------------------------------------------------------------------------------
# drawn cases
# ---------------------------------------------------------------------------------------------------------------------
def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size of [lo, hi], spread over its logarithm: a multiple of 64 in half of the draws (where there is one), any number otherwise."""
    v = _log_int(rng, lo, hi)
    return max(lo, v // 64 * 64) if rng.random() < 0.5 and v >= 64 else v


def draw(rng):
    most = work(listed()[6])
    while True:
        kind = rng.choice(("ppmv", "ppmv", "gated", "cache", "attention", "attention"))
        dtype = rng.choice(("bf16", "fp16"))
        if kind in ("ppmv", "gated"):
            case = _ppmv("", _size(rng, 64, INTER), _size(rng, 64, INTER), rng.choice((1, _log_int(rng, 1, 64), _log_int(rng, 1, 4096))),
                         rng.choice((32, 64, 128)), dtype, rng.random() < 0.5, kind)
        else:
            q_max = rng.choice((1, 1, _log_int(rng, 1, 64), _log_int(rng, 1, 4096)))
            len_max = max(q_max, _log_int(rng, 16, 32768))
            len_min = _log_int(rng, 1, len_max)
            batch = rng.choice((1, _log_int(rng, 1, 64)))
            kv_heads, head_dim, page = rng.choice((1, 2, 4, 8)), rng.choice((64, 128)), rng.choice((16, 32, 48, 64, 128))
            if batch * len_max * kv_heads * head_dim > 1 << 28 or batch * q_max > 8192:
                continue
            if kind == "cache":
                case = _cache("", batch, kv_heads, head_dim, q_max, len_min, len_max, page, dtype)
            else:
                case = _attention("", batch, kv_heads * rng.choice((1, 2, 4, 7, 8)), kv_heads, head_dim, q_max, len_min, len_max, page,
                                  rng.random() < 0.8, dtype)
                if batch * case["heads"] * q_max * len_max > 1 << 29:      # the plain form holds every score
                    continue
        del case["name"]
        w = work(case)
        if w["flops"] <= most["flops"] and w["bytes"] <= 4 * most["bytes"]:
            return case


def _lengths(case):
    """(new tokens, tokens in the cache with them) of every sequence: a matter of the case, not of the seed."""
    rng = random.Random("%d %d %d %d" % (case["batch"], case["q_max"], case["len_min"], case["len_max"]))
    lens = [_log_int(rng, case["len_min"], case["len_max"]) for _ in range(case["batch"])]
    lens[0] = case["len_max"]
    news = [min(n, case["q_max"] if i == 0 else rng.randint(1, case["q_max"])) for i, n in enumerate(lens)]
    return news, lens


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _weights(case, gen):
    """Codes, two a byte (the even k in the low half), group scales and offsets (None where the case has none)."""
    M, K, groups, t = case["M"], case["K"], -(-case["K"] // case["group"]), TYPES[case["dtype"]]
    codes = torch.randint(0, 256, (M, (K + 1) // 2), dtype=torch.uint8, device="cuda", generator=gen)
    scales = (0.005 + 0.01 * torch.rand((M, groups), device="cuda", generator=gen)).to(t)
    offsets = (0.01 * torch.randn((M, groups), device="cuda", generator=gen)).to(t) if case["offsets"] else None
    return codes, scales, offsets


def _product_inputs(case, seed):
    gen = _generator(seed)
    weights = [_weights(case, gen) for _ in range(2 if case["kind"] == "gated" else 1)]
    x = torch.randn((case["T"], case["K"]), device="cuda", generator=gen).to(TYPES[case["dtype"]])
    return weights, x


def _sequences(case, seed):
    """Queries, K and V of all cached tokens of all sequences one after the other, and the page table: pages in random order."""
    gen = _generator(seed)
    news, lens = _lengths(case)
    t, H, D = TYPES[case["dtype"]], case["kv_heads"], case["head_dim"]
    channel = torch.randn((H, D), device="cuda", generator=gen)            # keys have channels of their own mean
    k = (torch.randn((sum(lens), H, D), device="cuda", generator=gen) + channel).to(t)
    v = torch.randn((sum(lens), H, D), device="cuda", generator=gen).to(t)
    q = torch.randn((sum(news), case.get("heads", 1), D), device="cuda", generator=gen).to(t)
    width = -(-max(lens) // case["page"])
    pages = case["batch"] * width
    table = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32).view(case["batch"], width)
    starts = torch.tensor([sum(news[:i]) for i in range(len(news) + 1)], dtype=torch.int32, device="cuda")
    all_starts = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
    return {"q": q, "k": k, "v": v, "table": table, "pages": pages, "starts": starts, "all_starts": all_starts,
            "lens": torch.tensor(lens, dtype=torch.int32, device="cuda"), "news": news, "all": lens}


def _newest(case, s):
    """Rows of the new tokens among all cached ones."""
    rows = [torch.arange(sum(s["all"][:i + 1]) - n, sum(s["all"][:i + 1]), device="cuda") for i, n in enumerate(s["news"])]
    return torch.cat(rows)


def prepare(case, seed):
    kind = case["kind"]
    if kind in ("ppmv", "gated"):
        weights, x = _product_inputs(case, seed)
        out = torch.empty((case["T"], case["M"]), dtype=x.dtype, device="cuda")
        state = {"kind": kind, "x": x, "out": out, "group": case["group"], "weights": weights}
        if own:
            import paper_2601_18511_amd as lib
            state["weights"] = [lib.ppmv_plan_create(c, s, case["K"], case["group"], offsets=o) for c, s, o in weights]
        return state
    s = _sequences(case, seed)
    H, D, page = case["kv_heads"], case["head_dim"], case["page"]
    state = {"kind": kind, "table": s["table"], "starts": s["starts"], "lens": s["lens"], "page": page, "q_max": max(s["news"]),
             "max_len": max(s["all"]), "causal": case.get("causal", True)}
    if own:
        import paper_2601_18511_amd as lib
        cache = lib.ppkv_cache_create(s["pages"], page, H, D, device="cuda")
        if kind == "attention":
            lib.ppkv_append(cache, s["k"], s["v"], s["all_starts"], s["lens"], s["table"])
    else:
        cache = [torch.zeros((s["pages"] * page, H, D // 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
        cache += [torch.zeros((s["pages"] * page, H, D // GROUP, 2), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        if kind == "attention":
            _plain_write(cache, s["k"], s["v"], _slots(s["all_starts"], s["lens"], s["table"], page, s["k"].shape[0]))
    state["cache"] = cache
    if kind == "attention":
        state["q"], state["out"] = s["q"], torch.empty_like(s["q"])
    else:
        rows = _newest(case, s)
        state["k"], state["v"] = s["k"][rows].contiguous(), s["v"][rows].contiguous()
        state["k_out"], state["v_out"] = torch.empty_like(state["k"]), torch.empty_like(state["v"])
    return state


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _plain_weight(codes, scales, offsets, K, group):
    c = torch.stack((codes & 15, codes >> 4), dim=2).view(codes.shape[0], -1)[:, :K].float() - 8.0
    w = c * scales.float().repeat_interleave(group, dim=1)[:, :K]
    return w if offsets is None else w + offsets.float().repeat_interleave(group, dim=1)[:, :K]


def _plain_product(state):
    x = state["x"].float()
    y = [x @ _plain_weight(c, s, o, x.shape[1], state["group"]).t() for c, s, o in state["weights"]]
    if state["kind"] == "gated":
        return (y[0] / (1.0 + torch.exp(-y[0])) * y[1]).to(state["x"].dtype)
    return y[0].to(state["x"].dtype)


def _slots(starts, lens, table, page, rows):
    """Where in the cache the rows of a packed batch lie: page * size + place in the page."""
    n = torch.arange(rows, device="cuda")
    b = torch.searchsorted(starts[1:].long(), n, right=True)
    position = lens.long()[b] - (starts.long()[b + 1] - n)
    return table.long()[b, position // page] * page + position % page


def _plain_quantise(x):
    """Codes and (scale, offset) of every 32 channels. In 64 bits: a code is a whole number, and a value next to a border must not fall on the other side."""
    g = x.double().view(*x.shape[:-1], -1, GROUP)
    low, high = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    s = ((high - low) / 15.0).float().bfloat16()
    b = (low - 16.0 * s.double()).float().bfloat16()
    c = torch.clamp(torch.round((g - b.double()) / s.double()) - 16.0, 0.0, 15.0).to(torch.uint8).view(x.shape)
    return c[..., 0::2] | (c[..., 1::2] << 4), torch.cat((s, b), dim=-1)


def _plain_write(cache, k, v, slots):
    for n, x in enumerate((k, v)):
        cache[n][slots], cache[2 + n][slots] = _plain_quantise(x)


def _plain_values(codes, params):
    c = torch.stack((codes & 15, codes >> 4), dim=-1).view(*codes.shape[:-1], -1, GROUP).float() + 16.0
    return (c * params[..., :1].float() + params[..., 1:].float()).view(*codes.shape[:-1], -1)


def _plain_cache(state):
    cache, slots = state["cache"], _slots(state["starts"], state["lens"], state["table"], state["page"], state["k"].shape[0])
    _plain_write(cache, state["k"], state["v"], slots)
    return tuple(_plain_values(cache[n][slots], cache[2 + n][slots]).to(state["k"].dtype) for n in range(2))


def _plain_attention(state):
    """Every sequence filled up to the longest one, every score at once."""
    q, starts, lens, page = state["q"], state["starts"].long(), state["lens"].long(), state["page"]
    B, T, L, D = lens.shape[0], state["q_max"], state["max_len"], q.shape[2]
    position = torch.arange(L, device="cuda")
    slots = state["table"].long()[:, position // page] * page + position % page
    k, v = (_plain_values(state["cache"][n][slots], state["cache"][2 + n][slots]).transpose(1, 2).contiguous() for n in range(2))
    H, news = k.shape[1], starts[1:] - starts[:-1]
    G = q.shape[1] // H
    row = torch.arange(T, device="cuda")
    index = torch.clamp(starts[:-1, None] + row, max=q.shape[0] - 1)
    live = row < news[:, None]
    x = q[index].float().view(B, T, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * T, D)
    last = lens[:, None] - news[:, None] + row if state["causal"] else (lens[:, None] - 1).expand(B, T)
    hidden = position > last.repeat(1, G)[:, None, :, None]
    scores = (x @ k.transpose(2, 3).contiguous() * D ** -0.5).masked_fill_(hidden, float("-inf"))
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    o = (p @ v / p.sum(-1, keepdim=True)).view(B, H, G, T, D).permute(0, 3, 1, 2, 4).reshape(B, T, H * G, D)
    return o[live].to(q.dtype)


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(state):
    kind = state["kind"]
    if not own:
        return _plain_product(state) if kind in ("ppmv", "gated") else _plain_cache(state) if kind == "cache" else _plain_attention(state)
    import paper_2601_18511_amd as lib
    if kind == "ppmv":
        lib.ppmv_run(state["weights"][0], state["x"], state["out"])
        return state["out"]
    if kind == "gated":
        lib.ppmv_gated_run(state["weights"][0], state["weights"][1], state["x"], state["out"])
        return state["out"]
    where = (state["starts"], state["lens"], state["table"])
    if kind == "cache":
        lib.ppkv_append(state["cache"], state["k"], state["v"], *where)
        lib.ppkv_read(state["cache"], state["k_out"], state["v_out"], *where)
        return state["k_out"], state["v_out"]
    lib.ppkv_attention(state["cache"], state["q"], state["out"], *where, max_q=state["q_max"], max_len=state["max_len"], causal=state["causal"])
    return state["out"]


def work(case):
    if case["kind"] in ("ppmv", "gated"):
        M, K, T, n = case["M"], case["K"], case["T"], 2 if case["kind"] == "gated" else 1
        params = M * -(-K // case["group"]) * (4 if case["offsets"] else 2)
        return {"bytes": n * (M * ((K + 1) // 2) + params) + 2 * T * (K + M), "flops": 2 * n * T * M * K}
    news, lens = _lengths(case)
    H, D = case["kv_heads"], case["head_dim"]
    held = D + 8 * (D // GROUP)                # bytes of a cached token and K/V head, K and V together
    if case["kind"] == "cache":                # K and V in, the cache, and the values read back
        return {"bytes": sum(news) * H * (4 * D + held + 4 * D), "flops": 0}
    pairs = sum(t * n - (t * (t - 1) // 2 if case["causal"] else 0) for t, n in zip(news, lens))
    return {"bytes": sum(lens) * H * held + 4 * sum(news) * case["heads"] * D, "flops": 4 * D * case["heads"] * pairs}


# ---------------------------------------------------------------------------------------------------------------------
# 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------------------------------
def _exact_held(x):
    """What the cache stands for: value = scale (16 + code) + offset."""
    groups = x.to(torch.float64).unflatten(-1, (x.shape[-1] // GROUP, GROUP))
    low = groups.min(dim=-1).values
    scale = ((groups.max(dim=-1).values - low) / 15).to(torch.float32).to(torch.bfloat16).to(torch.float64)
    offset = (low - 16 * scale).to(torch.float32).to(torch.bfloat16).to(torch.float64)
    steps = ((groups - offset[..., None]) / scale[..., None]).round().clamp(16, 31)
    return (scale[..., None] * steps + offset[..., None]).flatten(-2)


def exact(case, seed):
    if case["kind"] in ("ppmv", "gated"):
        weights, x = _product_inputs(case, seed)
        M, K, group = case["M"], case["K"], case["group"]
        k = torch.arange(K, device="cuda")
        results = []
        for codes, scales, offsets in weights:
            half = codes[:, k // 2].to(torch.int32)
            w = (torch.where(k % 2 == 0, half % 16, half // 16) - 8).double()
            w *= scales[:, k // group].double()
            if offsets is not None:
                w += offsets[:, k // group].double()
            results.append(x.double() @ w.T)
        if case["kind"] == "ppmv":
            return results[0]
        return results[0] * torch.sigmoid(results[0]) * results[1]
    s = _sequences(case, seed)
    if case["kind"] == "cache":
        rows = _newest(case, s)
        return _exact_held(s["k"][rows]), _exact_held(s["v"][rows])
    if sum(t * n for t, n in zip(*_lengths(case))) * case["heads"] > 1 << 31:
        return None
    k, v, q = _exact_held(s["k"]), _exact_held(s["v"]), s["q"].double()
    G, out = case["heads"] // case["kv_heads"], torch.empty_like(q)
    first, at = 0, 0
    for t, n in zip(s["news"], s["all"]):
        for h in range(case["heads"]):
            scores = q[first:first + t, h] @ k[at:at + n, h // G].T.contiguous() / math.sqrt(case["head_dim"])
            if case["causal"]:
                key, query = torch.arange(n, device="cuda"), torch.arange(n - t, n, device="cuda")
                scores[key[None, :] > query[:, None]] = -math.inf
            out[first:first + t, h] = torch.softmax(scores, dim=1) @ v[at:at + n, h // G]
        first, at = first + t, at + n
    return out
