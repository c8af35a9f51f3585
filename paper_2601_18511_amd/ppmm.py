"""ctypes binding of the clear track (include/ppmm.h): products of 4-bit weights and clear activations, the 4-bit K/V cache and
attention over it.  Same names as the C ABI, argument marshalling only; there is no CPU fallback.  Inference only: a tensor that requires a
gradient is refused while gradients are recorded.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from .pcmm import PCMM_OK, PcmmError, _raw_stream, _stream_handle, load_library as _load

PPMM_BF16, PPMM_FP16, PPMM_INT16 = range(3)

EXPORTED = (
    "ppmv_plan_create",
    "ppmv_plan_workspace_bytes",
    "ppmv_run",
    "ppmv_gated_run",
    "ppmv_plan_destroy",
    "ppkv_pool_bytes",
    "ppkv_append",
    "ppkv_read",
    "ppkv_attention_scratch_bytes",
    "ppkv_attention",
)

_TYPES = {torch.bfloat16: PPMM_BF16, torch.float16: PPMM_FP16}
_lib: Optional[ctypes.CDLL] = None


class _CCache(ctypes.Structure):
    _fields_ = [("pool", ctypes.c_void_p), ("pages", ctypes.c_int64), ("page_size", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32)]


class _CBatch(ctypes.Structure):
    _fields_ = [("starts", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("table", ctypes.c_void_p), ("batch", ctypes.c_int32),
                ("table_width", ctypes.c_int32)]


def load_library() -> ctypes.CDLL:
    """The library of pcmm.load_library, with the clear track's argument types."""
    global _lib
    if _lib is not None:
        return _lib
    lib = _load()
    vp, i64, i32, size = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
    cache, batch = ctypes.POINTER(_CCache), ctypes.POINTER(_CBatch)
    signatures = {
        "ppmv_plan_create": (i32, [ctypes.POINTER(vp), i64, i64, i32, i32, vp, vp, vp, i32, vp]),
        "ppmv_plan_workspace_bytes": (size, [vp]),
        "ppmv_run": (i32, [vp, i64, vp, i64, vp, i64, vp]),
        "ppmv_gated_run": (i32, [vp, vp, i64, vp, i64, vp, i64, vp]),
        "ppmv_plan_destroy": (None, [vp]),
        "ppkv_pool_bytes": (size, [i64, i32, i32, i32]),
        "ppkv_append": (i32, [cache, batch, i64, i32, vp, i64, i64, vp, i64, i64, i32, vp]),
        "ppkv_read": (i32, [cache, batch, i64, i32, i32, vp, i64, i64, vp, i64, i64, i32, vp]),
        "ppkv_attention_scratch_bytes": (size, [cache, batch, i64, i32, i32, i64, i32]),
        "ppkv_attention": (i32, [cache, batch, i64, i32, i32, vp, i64, i64, vp, i64, i64, ctypes.c_float, i32, i32, i64, vp, size, i32, vp]),
    }
    for name, (restype, argtypes) in signatures.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = restype, argtypes
    _lib = lib
    return lib


_I32, _I64 = range(-1 << 31, 1 << 31), range(-1 << 63, 1 << 63)        # ctypes cuts what does not fit


# a result that autograd keeps is not what it kept any more (the private name takes half the time of the public one)
_new_version = getattr(torch._C, "_increment_version", torch.autograd.graph.increment_version)


def _no_gradients() -> None:
    """For a call with a tensor that requires a gradient."""
    if torch.is_grad_enabled():
        raise ValueError("the clear track has no gradients: call it under torch.no_grad() or with detached tensors")


def _handle(device: int, stream) -> int:
    return _raw_stream(device) if stream is None else int(stream.cuda_stream)


# ---- products with 4-bit weights ----------------------------------------------------------------------------------------


class PpmvPlan:
    """Owner of one ppmv_plan handle."""

    def __init__(self, handle: int, M: int, K: int, group: int, dtype: torch.dtype, device: int):
        self.handle = handle
        self.M, self.K, self.group, self.dtype, self.device = M, K, group, dtype, device

    def destroy(self) -> None:
        if self.handle:
            load_library().ppmv_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def ppmv_plan_create(codes: torch.Tensor, scales: torch.Tensor, K: int, group: int, offsets: Optional[torch.Tensor] = None,
                     stream=None) -> PpmvPlan:
    """Plan for the 4-bit matrix w[m][k] = scales[m][k // group] * (c[m][k] - 8) + offsets[m][k // group].

    codes is [M][(K+1)//2] uint8, even k in the low half of a byte; scales (and offsets) [M][ceil(K / group)] bfloat16 or float16, the
    type of the activations and results too; group 32, 64 or 128."""
    K, group = int(K), int(group)
    if not codes.is_cuda or codes.dim() != 2 or codes.dtype != torch.uint8 or not codes.is_contiguous() or K < 1 or codes.shape[1] != (K + 1) // 2:
        raise ValueError("codes must be a contiguous [M][(K+1)//2] uint8 tensor on the GPU")
    if group not in (32, 64, 128):
        raise ValueError("group must be 32, 64 or 128")
    M = codes.shape[0]
    for name, t in (("scales", scales), ("offsets", offsets)):
        if t is None and name == "offsets":
            continue
        if t.device != codes.device or t.dtype not in _TYPES or t.dtype != scales.dtype or not t.is_contiguous() or tuple(t.shape) != (M, -(-K // group)):
            raise ValueError("%s must be a contiguous [M][ceil(K / group)] bfloat16 or float16 tensor on the codes' device" % name)
    out = ctypes.c_void_p()
    with torch.cuda.device(codes.device):
        rc = load_library().ppmv_plan_create(ctypes.byref(out), M, K, group, _TYPES[scales.dtype], codes.data_ptr(), scales.data_ptr(),
                                             None if offsets is None else offsets.data_ptr(), codes.device.index, _stream_handle(stream))
    if rc != PCMM_OK:
        raise PcmmError(rc, "ppmv_plan_create")
    return PpmvPlan(out.value, M, K, group, scales.dtype, codes.device.index)


def ppmv_plan_workspace_bytes(plan: PpmvPlan) -> int:
    return int(load_library().ppmv_plan_workspace_bytes(plan.handle))


def ppmv_plan_destroy(plan: PpmvPlan) -> None:
    plan.destroy()


def _rows(plan: PpmvPlan, name: str, t: torch.Tensor, width: int):
    """(rows, address, row stride) of a [T][width] tensor of the plan's type and device with neighbouring elements in a row"""
    if t.dtype is not plan.dtype or t.get_device() != plan.device:
        raise ValueError("%s must have the plan's type and device" % name)
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or shape[1] != width or (stride[1] != 1 and width > 1):
        raise ValueError("%s must be [T][%d] with neighbouring elements in a row" % (name, width))
    return shape[0], t.data_ptr(), stride[0] if shape[0] > 1 else width


def ppmv_run(plan: PpmvPlan, x: torch.Tensor, y: torch.Tensor, stream=None) -> None:
    """Enqueue y = x W^T: x is [T][K], y [T][M], both may have longer rows (any row stride). Asynchronous."""
    if plan.handle is None:
        raise ValueError("plan was destroyed")
    T, px, ldx = _rows(plan, "x", x, plan.K)
    Ty, py, ldy = _rows(plan, "y", y, plan.M)
    if T != Ty:
        raise ValueError("x and y must have the same number of rows")
    if x.requires_grad or y.requires_grad:
        _no_gradients()
    rc = (_lib or load_library()).ppmv_run(plan.handle, T, px, ldx, py, ldy, _handle(plan.device, stream))
    if rc != PCMM_OK:
        raise PcmmError(rc, "ppmv_run")
    _new_version((y,))


def ppmv_gated_run(gate: PpmvPlan, up: PpmvPlan, x: torch.Tensor, h: torch.Tensor, stream=None) -> None:
    """Enqueue h = silu(x Wg^T) * (x Wu^T): x is [T][K], h [T][M]. Asynchronous."""
    if gate.handle is None or up.handle is None:
        raise ValueError("plan was destroyed")
    T, px, ldx = _rows(gate, "x", x, gate.K)
    Th, ph, ldh = _rows(gate, "h", h, gate.M)
    if T != Th:
        raise ValueError("x and h must have the same number of rows")
    if x.requires_grad or h.requires_grad:
        _no_gradients()
    rc = (_lib or load_library()).ppmv_gated_run(gate.handle, up.handle, T, px, ldx, ph, ldh, _handle(gate.device, stream))
    if rc != PCMM_OK:
        raise PcmmError(rc, "ppmv_gated_run")
    _new_version((h,))


# ---- the 4-bit K/V cache ------------------------------------------------------------------------------------------------


def ppkv_pool_bytes(pages: int, page_size: int, kv_heads: int, head_dim: int) -> int:
    sizes = int(pages), int(page_size), int(kv_heads), int(head_dim)
    if sizes[0] not in _I64 or not all(x in _I32 for x in sizes[1:]):
        return 0
    return int(load_library().ppkv_pool_bytes(*sizes))


class PpkvCache:
    """A paged 4-bit K/V cache: the pool is a torch tensor."""

    def __init__(self, pool: torch.Tensor, pages: int, page_size: int, kv_heads: int, head_dim: int):
        if not pool.is_cuda or pool.dtype != torch.uint8 or not pool.is_contiguous() or pool.numel() != ppkv_pool_bytes(pages, page_size, kv_heads, head_dim):
            raise ValueError("pool must be a contiguous uint8 tensor of ppkv_pool_bytes bytes on the GPU")
        self.pool, self.pages, self.page_size, self.kv_heads, self.head_dim = pool, pages, page_size, kv_heads, head_dim
        self.device = pool.get_device()
        self._c = _CCache(pool.data_ptr(), pages, page_size, kv_heads, head_dim)


def ppkv_cache_create(pages: int, page_size: int, kv_heads: int, head_dim: int, device="cuda") -> PpkvCache:
    """A cache of `pages` pages of page_size tokens (a multiple of 16), kv_heads heads of head_dim (64 or 128) channels. Not cleared."""
    size = ppkv_pool_bytes(pages, page_size, kv_heads, head_dim)
    if size == 0:
        raise ValueError("pages, page_size, kv_heads or head_dim out of range")
    return PpkvCache(torch.empty(size, dtype=torch.uint8, device=device), int(pages), int(page_size), int(kv_heads), int(head_dim))


def _batch(cache: PpkvCache, starts: torch.Tensor, lens: torch.Tensor, table: torch.Tensor) -> _CBatch:
    device = cache.device
    shape, count = table.shape, lens.shape
    if not (starts.dtype is lens.dtype is table.dtype is torch.int32 and starts.get_device() == lens.get_device() == table.get_device() == device
            and starts.is_contiguous() and lens.is_contiguous() and table.is_contiguous() and len(shape) == 2 and len(count) == 1 and starts.dim() == 1):
        raise ValueError("starts, lens (1-D) and table (2-D) must be contiguous int32 tensors on the cache's device")
    if starts.shape[0] != count[0] + 1 or shape[0] != count[0]:
        raise ValueError("starts must have one entry more than lens, table one row for each of them")
    return _CBatch(starts.data_ptr(), lens.data_ptr(), table.data_ptr(), count[0], shape[1])


_READ_TYPES = {**_TYPES, torch.int16: PPMM_INT16}


def _packed(cache: PpkvCache, name: str, t: torch.Tensor, heads: int, types):
    """(rows, type, (address, token stride, head stride)) of a [tokens][heads][head_dim] tensor on the cache's device with neighbouring channels"""
    kind = types.get(t.dtype)
    if kind is None or t.get_device() != cache.device:
        raise ValueError("%s must be on the cache's device, of type %s" % (name, " or ".join(str(x) for x in types)))
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or shape[1] != heads or shape[2] != cache.head_dim or stride[2] != 1:
        raise ValueError("%s must be [tokens][%d][%d] with neighbouring channels" % (name, heads, cache.head_dim))
    return shape[0], kind, (t.data_ptr(), stride[0], stride[1])


def ppkv_append(cache: PpkvCache, k: torch.Tensor, v: torch.Tensor, starts: torch.Tensor, lens: torch.Tensor, table: torch.Tensor,
                stream=None) -> None:
    """Quantise the new tokens' keys and values ([tokens][kv_heads][head_dim]) into the cache. Row n belongs to the sequence b with
    starts[b] <= n < starts[b+1] and is its token lens[b] - (starts[b+1] - n), in page table[b][.. // page_size]. Asynchronous."""
    batch = _batch(cache, starts, lens, table)
    rows, kind, k_at = _packed(cache, "k", k, cache.kv_heads, _TYPES)
    v_rows, v_kind, v_at = _packed(cache, "v", v, cache.kv_heads, _TYPES)
    if rows != v_rows or kind != v_kind:
        raise ValueError("k and v must have the same type and shape")
    if k.requires_grad or v.requires_grad:
        _no_gradients()
    rc = (_lib or load_library()).ppkv_append(cache._c, batch, rows, kind, *k_at, *v_at, cache.device, _handle(cache.device, stream))
    if rc != PCMM_OK:
        raise PcmmError(rc, "ppkv_append")


def ppkv_read(cache: PpkvCache, k: Optional[torch.Tensor], v: Optional[torch.Tensor], starts: torch.Tensor, lens: torch.Tensor,
              table: torch.Tensor, frac_bits: int = 0, stream=None) -> None:
    """The cached values of the same tokens into k and v ([tokens][kv_heads][head_dim], either may be None). int16 tensors get
    rint(value 2^frac_bits): an operand of pcmm_plan_create. Asynchronous."""
    batch = _batch(cache, starts, lens, table)
    k_is = (None, None, (None, 0, 0)) if k is None else _packed(cache, "k", k, cache.kv_heads, _READ_TYPES)
    v_is = (None, None, (None, 0, 0)) if v is None else _packed(cache, "v", v, cache.kv_heads, _READ_TYPES)
    rows, kind = k_is[:2] if k is not None else v_is[:2]
    if rows is None:
        raise ValueError("neither k nor v is wanted")
    if k is not None and v is not None and k_is[:2] != v_is[:2]:
        raise ValueError("k and v must have the same type and shape")
    results = (v,) if k is None else (k,) if v is None else (k, v)
    if results[0].requires_grad or results[-1].requires_grad:
        _no_gradients()
    frac_bits = int(frac_bits)
    if frac_bits not in _I32:
        raise ValueError("frac_bits out of range")
    rc = (_lib or load_library()).ppkv_read(cache._c, batch, rows, kind, frac_bits, *k_is[2], *v_is[2], cache.device, _handle(cache.device, stream))
    if rc != PCMM_OK:
        raise PcmmError(rc, "ppkv_read")
    _new_version(results)


def ppkv_attention_scratch_bytes(cache: PpkvCache, tokens: int, heads: int, starts: torch.Tensor, lens: torch.Tensor, table: torch.Tensor,
                                 max_q: int, max_len: int = 0) -> int:
    batch = _batch(cache, starts, lens, table)
    tokens, heads, max_q, max_len = int(tokens), int(heads), int(max_q), int(max_len)
    if tokens not in _I64 or heads not in _I32 or max_q not in _I32 or max_len not in _I64:
        raise ValueError("tokens, heads, max_q or max_len out of range")
    return int(load_library().ppkv_attention_scratch_bytes(cache._c, batch, tokens, heads, max_q, max_len, cache.device))


def ppkv_attention(cache: PpkvCache, q: torch.Tensor, out: torch.Tensor, starts: torch.Tensor, lens: torch.Tensor, table: torch.Tensor,
                   max_q: int, max_len: int = 0, scale: Optional[float] = None, causal: bool = True, stream=None) -> None:
    """Enqueue attention of the new tokens' queries ([tokens][heads][head_dim]) over the cache; scale defaults to 1 / sqrt(head_dim).
    max_q: the largest number of new tokens of a sequence; max_len: the expected largest length. Asynchronous."""
    batch = _batch(cache, starts, lens, table)
    heads = q.shape[1] if q.dim() == 3 else 0
    if heads == 0 or heads % cache.kv_heads:
        raise ValueError("q must be [tokens][heads][head_dim] with a multiple of the cache's heads")
    tokens, kind, q_at = _packed(cache, "q", q, heads, _TYPES)
    out_tokens, out_kind, out_at = _packed(cache, "out", out, heads, _TYPES)
    if tokens != out_tokens or kind != out_kind:
        raise ValueError("q and out must have the same type and shape")
    if q.requires_grad or out.requires_grad:
        _no_gradients()
    lib, device, max_q, max_len = _lib or load_library(), cache.device, int(max_q), int(max_len)
    if max_q not in _I32 or max_len not in _I64:
        raise ValueError("max_q or max_len out of range")
    size = lib.ppkv_attention_scratch_bytes(cache._c, batch, tokens, heads, max_q, max_len, device)
    scratch = None
    if size:        # of the pool of the stream that uses it: whoever gets the memory next runs behind this call
        if stream is None:
            scratch = torch.empty(size, dtype=torch.uint8, device=cache.pool.device)
        else:
            with torch.cuda.stream(stream):
                scratch = torch.empty(size, dtype=torch.uint8, device=cache.pool.device)
    rc = lib.ppkv_attention(cache._c, batch, tokens, kind, heads, *q_at, *out_at, cache.head_dim ** -0.5 if scale is None else float(scale),
                            1 if causal else 0, max_q, max_len, scratch.data_ptr() if size else None, size, device, _handle(device, stream))
    if rc != PCMM_OK:
        raise PcmmError(rc, "ppkv_attention")
    _new_version((out,))
