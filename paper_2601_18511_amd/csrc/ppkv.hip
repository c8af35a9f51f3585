// The public K/V cache in 4 bits, and attention over it (include/ppmm.h; Sections 4.1 and 4.2), on MI355X (gfx950).
//
// A value of the cache is s (16 + code) + b: s and b bf16, one pair for 32 channels of one token.  16 + code with a 4-bit code
// is exactly the 16-bit float whose exponent is that of 16 and whose top four mantissa bits are the code.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "ppmm_device.hpp"
#include "ppmm_host.hpp"
#include "pcmm_hip_util.hpp"

namespace {

using ppmm::BF16;
using ppmm::Cache;
using ppmm::FP16;

constexpr int kThreads = 256;

// Places inside a page of one head.  A token's D/2 bytes of codes are words of eight codes, ascending channels from the lowest
// four bits.  Values lie in order.  The words of a key are transposed: word (D/32) h + j holds channels 32 j + 8 h ... + 7.
template <int D> __device__ inline int64_t codes_at(const Cache &c, int which, int slot) { return (int64_t)(which * c.page_size + slot) * (D / 2); }
template <int D> __device__ inline int64_t params_at(const Cache &c, int which, int slot)
{
    return (int64_t)c.page_size * D + (int64_t)(which * c.page_size + slot) * (D / 8);
}

// ---- writing -------------------------------------------------------------------------------------------------------
// A thread takes eight channels (16 bytes), four neighbouring threads a group.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void append_kernel(Cache c, int64_t tokens, const uint16_t *k, int64_t kts, int64_t khs,
                                                          const uint16_t *v, int64_t vts, int64_t vhs)
{
    const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int part = (int)(idx % (D / 8));
    const int64_t row = idx / (D / 8);              // (token, K or V, head)
    const int head = (int)(row % c.kv_heads);
    const int which = (int)(row / c.kv_heads % 2);
    const int64_t n = row / c.kv_heads / 2;
    if (n >= tokens) return;                        // whole groups of threads leave together
    const int32_t b = c.sequence_of(n);
    if (b < 0) return;
    const int64_t position = (int64_t)c.lens[b] - (c.starts[b + 1] - n);
    uint8_t *page = c.page_of(b, position, head);
    if (!page) return;
    const uint16_t *src = (which ? v + n * vts + head * vhs : k + n * kts + head * khs) + part * 8;
    float x[8];
    float low = INFINITY, high = -INFINITY;
    bool finite = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = ppmm::to_f32<T>(src[i]);
        finite = finite && isfinite(x[i]);
        low = fminf(low, x[i]);
        high = fmaxf(high, x[i]);
    }
#pragma unroll
    for (int step = 1; step < 4; step *= 2) {
        low = fminf(low, __shfl_xor(low, step));
        high = fmaxf(high, __shfl_xor(high, step));
        finite = __shfl_xor((int)finite, step) && finite;
    }
    uint16_t s_bits = ppmm::from_f32<BF16>((float)(((double)high - (double)low) / 15.0));
    float s = ppmm::to_f32<BF16>(s_bits);
    if (!(s >= 0x1p-126f)) { s = 0.0f; s_bits = 0; }
    uint16_t b_bits = ppmm::from_f32<BF16>((float)((double)low - 16.0 * (double)s));
    if (!finite || !isfinite(s) || !isfinite(ppmm::to_f32<BF16>(b_bits))) { s = 0.0f; s_bits = 0; b_bits = 0x7fc0; }
    const double off = (double)ppmm::to_f32<BF16>(b_bits);
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double steps = s > 0.0f ? rint(((double)x[i] - off) / (double)s) - 16.0 : 0.0;
        word |= (uint32_t)(int)fmin(fmax(steps, 0.0), 15.0) << (4 * i);
    }
    const int slot = (int)(position % c.page_size);
    const int j = part / 4, h = part % 4;
    const int place = which ? part : (D / 32) * h + j;
    *(uint32_t *)(page + codes_at<D>(c, which, slot) + 4 * place) = word;
    if (h == 0) *(uint32_t *)(page + params_at<D>(c, which, slot) + 4 * j) = s_bits | (uint32_t)b_bits << 16;
}

// ---- reading -------------------------------------------------------------------------------------------------------
struct I16 {};

template <class T> __device__ inline uint16_t as_result(float v, float) { return ppmm::from_f32<T>(v); }
template <> __device__ inline uint16_t as_result<I16>(float v, float fixed)
{
    const float r = rintf(v * fixed);               // a power of two: the product is exact
    return r != r ? 0 : (uint16_t)(int16_t)(int)fminf(fmaxf(r, -32768.0f), 32639.0f);
}

template <class T, int D>
__global__ __launch_bounds__(kThreads) void read_kernel(Cache c, int64_t tokens, float fixed, uint16_t *k, int64_t kts, int64_t khs,
                                                        uint16_t *v, int64_t vts, int64_t vhs)
{
    const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int part = (int)(idx % (D / 8));
    const int64_t row = idx / (D / 8);
    const int head = (int)(row % c.kv_heads);
    const int which = (int)(row / c.kv_heads % 2);
    const int64_t n = row / c.kv_heads / 2;
    if (n >= tokens || !(which ? v : k)) return;
    const int32_t b = c.sequence_of(n);
    if (b < 0) return;
    const int64_t position = (int64_t)c.lens[b] - (c.starts[b + 1] - n);
    const uint8_t *page = c.page_of(b, position, head);
    uint16_t *dst = (which ? v + n * vts + head * vhs : k + n * kts + head * khs) + part * 8;
    const int j = part / 4, h = part % 4;
    uint32_t word = 0, sb = 0;
    if (page) {
        const int slot = (int)(position % c.page_size);
        word = *(const uint32_t *)(page + codes_at<D>(c, which, slot) + 4 * (which ? part : (D / 32) * h + j));
        sb = *(const uint32_t *)(page + params_at<D>(c, which, slot) + 4 * j);
    }
    const float s = ppmm::to_f32<BF16>((uint16_t)sb), off = ppmm::to_f32<BF16>((uint16_t)(sb >> 16));
#pragma unroll
    for (int i = 0; i < 8; ++i)
        dst[i] = as_result<T>(fmaf(s, 16.0f + (float)(word >> (4 * i) & 15), off), fixed);
}

// ---- attention -----------------------------------------------------------------------------------------------------
// One wave a row and head, one key after the other.
template <class T, int D>
__global__ __launch_bounds__(64) void attention_kernel(Cache c, int64_t tokens, int32_t heads, const uint16_t *q, int64_t qts, int64_t qhs,
                                                       uint16_t *out, int64_t ots, int64_t ohs, float scale, int32_t causal, int32_t max_q)
{
    constexpr int E = D / 64;                       // channels of a lane
    const int64_t n = blockIdx.x / heads;
    const int qh = (int)(blockIdx.x % heads), head = qh / (heads / c.kv_heads);
    const int32_t b = c.sequence_of(n);
    if (b < 0) return;
    const int64_t first = c.starts[b], next = c.starts[b + 1];
    if (n - first >= max_q) return;
    int64_t len = c.lens[b];
    const int64_t position = len - (next - n);
    if (causal && position + 1 < len) len = position + 1;
    if (len > c.capacity()) len = c.capacity();
    float x[E], o[E] = {};
    const int ch = threadIdx.x * E;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = ppmm::to_f32<T>(q[n * qts + qh * qhs + ch + e]);
    float most = -INFINITY, sum = 0.0f;
    const int j = ch / 32, h = ch / 8 % 4;
    for (int64_t i = 0; i < len; ++i) {
        const uint8_t *page = c.page_of(b, i, head);
        if (!page) continue;
        const int slot = (int)(i % c.page_size);
        const uint32_t kw = *(const uint32_t *)(page + codes_at<D>(c, 0, slot) + 4 * ((D / 32) * h + j));
        const uint32_t vw = *(const uint32_t *)(page + codes_at<D>(c, 1, slot) + 4 * (ch / 8));
        const uint32_t kp = *(const uint32_t *)(page + params_at<D>(c, 0, slot) + 4 * j);
        const uint32_t vp = *(const uint32_t *)(page + params_at<D>(c, 1, slot) + 4 * j);
        float dot = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e)
            dot = fmaf(x[e], fmaf(ppmm::to_f32<BF16>((uint16_t)kp), 16.0f + (float)(kw >> (4 * (ch % 8 + e)) & 15), ppmm::to_f32<BF16>((uint16_t)(kp >> 16))), dot);
#pragma unroll
        for (int step = 32; step; step /= 2) dot += __shfl_xor(dot, step);
        const float score = dot * scale;
        const float top = fmaxf(most, score);
        const float keep = most == -INFINITY ? 0.0f : expf(most - top), p = top == -INFINITY ? 0.0f : expf(score - top);
        sum = fmaf(sum, keep, p);
#pragma unroll
        for (int e = 0; e < E; ++e)
            o[e] = fmaf(o[e], keep, p * fmaf(ppmm::to_f32<BF16>((uint16_t)vp), 16.0f + (float)(vw >> (4 * (ch % 8 + e)) & 15), ppmm::to_f32<BF16>((uint16_t)(vp >> 16))));
        most = top;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) out[n * ots + qh * ohs + ch + e] = ppmm::from_f32<T>(sum == 0.0f ? 0.0f : o[e] / sum);
}

Cache device_cache(const ppkv_cache *c, const ppkv_batch *b)
{
    return Cache{(uint8_t *)c->pool, c->pages, c->page_size, c->kv_heads, c->head_dim, b->starts, b->lens, b->table, b->batch, b->table_width};
}

// work-groups of `threads` for `items` threads; 0 if the launch would have 2^32 threads or more
uint32_t blocks_for(int64_t items, int threads)
{
    const int64_t blocks = (items + threads - 1) / threads;
    return blocks * threads >= ((int64_t)1 << 32) ? 0u : (uint32_t)blocks;
}

}  // namespace

extern "C" {

size_t ppkv_pool_bytes(int64_t pages, int32_t page_size, int32_t kv_heads, int32_t head_dim)
{
    return ppmm_host::pool_bytes(pages, page_size, kv_heads, head_dim);
}

pcmm_status ppkv_append(const ppkv_cache *cache, const ppkv_batch *batch, int64_t tokens, ppmm_type type, const void *k_dev,
                        int64_t kts, int64_t khs, const void *v_dev, int64_t vts, int64_t vhs, int32_t device, void *stream)
{
    const pcmm_status rc = ppmm_host::check_cache(cache, batch, tokens, device);
    if (rc != PCMM_OK) return rc;
    if ((type != PPMM_BF16 && type != PPMM_FP16) || !ppmm_host::read_strides_ok(kts, khs) || !ppmm_host::read_strides_ok(vts, vhs)) return PCMM_EINVAL;
    if (tokens == 0) return PCMM_OK;
    if (!k_dev || !v_dev) return PCMM_EINVAL;
    const int D = cache->head_dim;
    const uint32_t blocks = blocks_for(tokens * 2 * cache->kv_heads * (D / 8), kThreads);
    if (!blocks) return PCMM_EUNSUPPORTED;
    pcmm_hip_util::DevGuard dg(device);
    if (!dg.ok) return PCMM_EDEVICE;
    auto kernel = type == PPMM_BF16 ? (D == 64 ? append_kernel<BF16, 64> : append_kernel<BF16, 128>)
                                    : (D == 64 ? append_kernel<FP16, 64> : append_kernel<FP16, 128>);
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), 0, (hipStream_t)stream, device_cache(cache, batch), tokens, (const uint16_t *)k_dev,
                       kts, khs, (const uint16_t *)v_dev, vts, vhs);
    return hipGetLastError() == hipSuccess ? PCMM_OK : PCMM_EDEVICE;
}

pcmm_status ppkv_read(const ppkv_cache *cache, const ppkv_batch *batch, int64_t tokens, ppmm_type type, int32_t frac_bits, void *k_dev,
                      int64_t kts, int64_t khs, void *v_dev, int64_t vts, int64_t vhs, int32_t device, void *stream)
{
    const pcmm_status rc = ppmm_host::check_cache(cache, batch, tokens, device);
    if (rc != PCMM_OK) return rc;
    if (type != PPMM_BF16 && type != PPMM_FP16 && type != PPMM_INT16) return PCMM_EINVAL;
    if (frac_bits < 0 || frac_bits > (type == PPMM_INT16 ? 30 : 0)) return PCMM_EINVAL;
    const int D = cache->head_dim, H = cache->kv_heads;
    if ((k_dev && !ppmm_host::rows_apart(tokens, H, D, kts, khs)) || (v_dev && !ppmm_host::rows_apart(tokens, H, D, vts, vhs)) ||
        (k_dev && k_dev == v_dev))
        return PCMM_EINVAL;
    if (tokens == 0 || (!k_dev && !v_dev)) return PCMM_OK;
    const uint32_t blocks = blocks_for(tokens * 2 * H * (D / 8), kThreads);
    if (!blocks) return PCMM_EUNSUPPORTED;
    pcmm_hip_util::DevGuard dg(device);
    if (!dg.ok) return PCMM_EDEVICE;
    auto kernel = type == PPMM_BF16 ? (D == 64 ? read_kernel<BF16, 64> : read_kernel<BF16, 128>)
                : type == PPMM_FP16 ? (D == 64 ? read_kernel<FP16, 64> : read_kernel<FP16, 128>)
                                    : (D == 64 ? read_kernel<I16, 64> : read_kernel<I16, 128>);
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), 0, (hipStream_t)stream, device_cache(cache, batch), tokens, ldexpf(1.0f, frac_bits),
                       (uint16_t *)k_dev, kts, khs, (uint16_t *)v_dev, vts, vhs);
    return hipGetLastError() == hipSuccess ? PCMM_OK : PCMM_EDEVICE;
}

size_t ppkv_attention_scratch_bytes(const ppkv_cache *cache, const ppkv_batch *batch, int64_t tokens, int32_t heads, int32_t max_q,
                                    int64_t max_len, int32_t device)
{
    (void)cache; (void)batch; (void)tokens; (void)heads; (void)max_q; (void)max_len; (void)device;
    return 0;
}

pcmm_status ppkv_attention(const ppkv_cache *cache, const ppkv_batch *batch, int64_t tokens, ppmm_type type, int32_t heads,
                           const void *q_dev, int64_t qts, int64_t qhs, void *out_dev, int64_t ots, int64_t ohs, float scale, int32_t causal,
                           int32_t max_q, int64_t max_len, void *scratch, size_t scratch_bytes, int32_t device, void *stream)
{
    const pcmm_status rc = ppmm_host::check_attention(cache, batch, tokens, type, heads, max_q, max_len, device);
    if (rc != PCMM_OK) return rc;
    const int D = cache->head_dim;
    if (!ppmm_host::read_strides_ok(qts, qhs) || !ppmm_host::rows_apart(tokens, heads, D, ots, ohs)) return PCMM_EINVAL;
    if (tokens == 0 || max_q == 0) return PCMM_OK;
    if (!q_dev || !out_dev || q_dev == out_dev) return PCMM_EINVAL;
    if (scratch_bytes < ppkv_attention_scratch_bytes(cache, batch, tokens, heads, max_q, max_len, device)) return PCMM_EINVAL;
    (void)scratch;
    const uint32_t blocks = blocks_for(tokens * heads * 64, 64);
    if (!blocks) return PCMM_EUNSUPPORTED;
    pcmm_hip_util::DevGuard dg(device);
    if (!dg.ok) return PCMM_EDEVICE;
    auto kernel = type == PPMM_BF16 ? (D == 64 ? attention_kernel<BF16, 64> : attention_kernel<BF16, 128>)
                                    : (D == 64 ? attention_kernel<FP16, 64> : attention_kernel<FP16, 128>);
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(64), 0, (hipStream_t)stream, device_cache(cache, batch), tokens, heads, (const uint16_t *)q_dev,
                       qts, qhs, (uint16_t *)out_dev, ots, ohs, scale, causal, max_q);
    return hipGetLastError() == hipSuccess ? PCMM_OK : PCMM_EDEVICE;
}

}  // extern "C"
