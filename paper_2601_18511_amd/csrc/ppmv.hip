// Products with weights held in 4 bits under group scales (include/ppmm.h; Section 5.1's linear layers for clear tokens), on
// MI355X (gfx950).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <new>

#include "ppmm_device.hpp"
#include "ppmm_host.hpp"
#include "pcmm_hip_util.hpp"

struct ppmv_plan {
    int64_t M, K;
    int32_t group, type, device;
    bool has_offsets;
    uint8_t *codes;
    uint16_t *scales, *offsets;
    size_t bytes;
};

namespace {

using ppmm::BF16;
using ppmm::FP16;

struct Weights {
    const uint8_t *codes;
    const uint16_t *scales, *offsets;
};

template <class T>
__device__ inline float dot(const Weights &w, const uint16_t *x, int64_t m, int64_t K, int32_t group)
{
    const int64_t groups = (K + group - 1) / group, half = (K + 1) / 2;
    float sum = 0.0f;
    for (int64_t k = threadIdx.x; k < K; k += 64) {
        const int c = w.codes[m * half + k / 2] >> (4 * (k & 1)) & 15;
        const float s = ppmm::to_f32<T>(w.scales[m * groups + k / group]);
        const float o = w.offsets ? ppmm::to_f32<T>(w.offsets[m * groups + k / group]) : 0.0f;
        sum = fmaf(ppmm::to_f32<T>(x[k]), fmaf(s, (float)(c - 8), o), sum);
    }
    for (int step = 32; step; step /= 2) sum += __shfl_xor(sum, step);
    return sum;
}

// One wave a result.
template <class T, bool kGated>
__global__ __launch_bounds__(64) void product_kernel(Weights a, Weights b, int64_t M, int64_t K, int32_t group, int64_t T_, const uint16_t *x,
                                                     int64_t ldx, uint16_t *y, int64_t ldy)
{
    const int64_t m = blockIdx.x;
    for (int64_t t = blockIdx.y; t < T_; t += gridDim.y) {
        float r = dot<T>(a, x + t * ldx, m, K, group);
        if (kGated) {
            const float u = dot<T>(b, x + t * ldx, m, K, group);
            r = r / (1.0f + expf(-r)) * u;
        }
        if (threadIdx.x == 0) y[t * ldy + m] = ppmm::from_f32<T>(r);
    }
}

template <bool kGated>
pcmm_status run(const ppmv_plan *p, const ppmv_plan *u, int64_t T, const void *x, int64_t ldx, void *y, int64_t ldy, void *stream)
{
    bool nothing;
    const pcmm_status rc = ppmm_host::check_product(p->M, p->K, T, x, ldx, y, ldy, &nothing);
    if (rc != PCMM_OK || nothing) return rc;
    pcmm_hip_util::DevGuard dg(p->device);
    if (!dg.ok) return PCMM_EDEVICE;
    auto kernel = p->type == PPMM_BF16 ? product_kernel<BF16, kGated> : product_kernel<FP16, kGated>;
    const Weights a{p->codes, p->scales, p->offsets}, b{u->codes, u->scales, u->offsets};
    hipLaunchKernelGGL(kernel, dim3((unsigned)p->M, (unsigned)(T < 128 ? T : 128)), dim3(64), 0, (hipStream_t)stream, a, b, p->M, p->K, p->group, T,
                       (const uint16_t *)x, ldx, (uint16_t *)y, ldy);
    return hipGetLastError() == hipSuccess ? PCMM_OK : PCMM_EDEVICE;
}

}  // namespace

extern "C" {

pcmm_status ppmv_plan_create(ppmv_plan **out, int64_t M, int64_t K, int32_t group, ppmm_type type, const uint8_t *codes_dev,
                             const void *scales_dev, const void *offsets_dev, int32_t device, void *stream)
{
    if (!out) return PCMM_EINVAL;
    *out = nullptr;
    const pcmm_status arc = ppmm_host::check_weights(M, K, group, type, codes_dev, scales_dev, device);
    if (arc != PCMM_OK) return arc;
    ppmv_plan *p = new (std::nothrow) ppmv_plan();
    if (!p) return PCMM_ENOMEM;
    p->M = M; p->K = K; p->group = group; p->type = type; p->device = device; p->has_offsets = offsets_dev != nullptr;
    pcmm_hip_util::DevGuard dg(device);
    if (!dg.ok) { delete p; return PCMM_EDEVICE; }
    hipStream_t st = (hipStream_t)stream;
    const size_t code_bytes = (size_t)M * ((K + 1) / 2), param_bytes = (size_t)M * ((K + group - 1) / group) * 2;
    pcmm_status rc = PCMM_OK;
    if (hipMalloc((void **)&p->codes, code_bytes) != hipSuccess || hipMalloc((void **)&p->scales, param_bytes) != hipSuccess ||
        (offsets_dev && hipMalloc((void **)&p->offsets, param_bytes) != hipSuccess)) {
        (void)hipGetLastError();
        rc = PCMM_ENOMEM;
    }
    p->bytes = code_bytes + param_bytes * (offsets_dev ? 2 : 1);
    if (rc == PCMM_OK &&
        (hipMemcpyAsync(p->codes, codes_dev, code_bytes, hipMemcpyDeviceToDevice, st) != hipSuccess ||
         hipMemcpyAsync(p->scales, scales_dev, param_bytes, hipMemcpyDeviceToDevice, st) != hipSuccess ||
         (offsets_dev && hipMemcpyAsync(p->offsets, offsets_dev, param_bytes, hipMemcpyDeviceToDevice, st) != hipSuccess) ||
         hipStreamSynchronize(st) != hipSuccess))
        rc = PCMM_EDEVICE;
    if (rc != PCMM_OK) { ppmv_plan_destroy(p); return rc; }
    *out = p;
    return PCMM_OK;
}

size_t ppmv_plan_workspace_bytes(const ppmv_plan *plan) { return plan ? plan->bytes : 0; }

pcmm_status ppmv_run(const ppmv_plan *plan, int64_t T, const void *x_dev, int64_t ldx, void *y_dev, int64_t ldy, void *stream)
{
    if (!plan) return PCMM_EINVAL;
    return run<false>(plan, plan, T, x_dev, ldx, y_dev, ldy, stream);
}

pcmm_status ppmv_gated_run(const ppmv_plan *gate, const ppmv_plan *up, int64_t T, const void *x_dev, int64_t ldx, void *h_dev, int64_t ldh,
                           void *stream)
{
    if (!gate || !up) return PCMM_EINVAL;
    if (gate->M != up->M || gate->K != up->K || gate->group != up->group || gate->type != up->type || gate->device != up->device ||
        gate->has_offsets != up->has_offsets)
        return PCMM_EINVAL;
    return run<true>(gate, up, T, x_dev, ldx, h_dev, ldh, stream);
}

void ppmv_plan_destroy(ppmv_plan *plan)
{
    if (!plan) return;
    pcmm_hip_util::DevGuard dg(plan->device);
    (void)hipFree(plan->codes);
    (void)hipFree(plan->scales);
    (void)hipFree(plan->offsets);
    delete plan;
}

}  // extern "C"
