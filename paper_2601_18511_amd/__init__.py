"""MI355X-native PCMM (plaintext-ciphertext matrix multiplication) for CKKS linear layers.

Thin Python binding over the C-ABI library libpcmm.so (see include/pcmm.h, and include/ppmm.h for the
clear track: 4-bit weights, 4-bit K/V cache and attention over it); every step of the
computation runs in the library's HIP kernels.  PyTorch is used for device memory and streams only.
"""
from .pcmm import (  # noqa: F401
    PcmmError,
    PcmmPlan,
    load_library,
    pcmm_mfma_probe,
    pcmm_plan_create,
    pcmm_plan_destroy,
    pcmm_plan_digits,
    pcmm_plan_workspace_bytes,
    pcmm_ring_compose,
    pcmm_ring_decompose,
    pcmm_run,
    pcmm_slot_rearrange,
    pcmm_run_noalloc,
    pcmm_run_profiled,
    pcmm_status_str,
    PcmvPlan,
    pcmv_plan_create,
    pcmv_plan_destroy,
    pcmv_plan_workspace_bytes,
    pcmv_run,
)
from .ppmm import (  # noqa: F401
    PpkvCache,
    PpmvPlan,
    ppkv_append,
    ppkv_attention,
    ppkv_attention_scratch_bytes,
    ppkv_cache_create,
    ppkv_pool_bytes,
    ppkv_read,
    ppmv_gated_run,
    ppmv_plan_create,
    ppmv_plan_destroy,
    ppmv_plan_workspace_bytes,
    ppmv_run,
)
