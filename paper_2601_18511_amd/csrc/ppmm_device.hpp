// Device helpers of the clear track: 16-bit types, and where the tokens of a batch lie in the paged cache.
#ifndef PPMM_DEVICE_HPP
#define PPMM_DEVICE_HPP

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ppmm.h"

namespace ppmm {

struct BF16 { using type = __bf16; };
struct FP16 { using type = _Float16; };

template <class T> __device__ inline float to_f32(uint16_t bits) { return (float)__builtin_bit_cast(typename T::type, bits); }
template <class T> __device__ inline uint16_t from_f32(float v) { return __builtin_bit_cast(uint16_t, (typename T::type)v); }   // to nearest even

// A pool and a batch as the kernels take them.  Offsets into the pool are 64-bit.
struct Cache {
    uint8_t *pool;
    int64_t pages;
    int32_t page_size, kv_heads, head_dim;
    const int32_t *starts, *lens, *table;
    int32_t batch, table_width;

    // bytes of one page of one head: [codes of keys][codes of values][(s, b) of keys][(s, b) of values]
    __device__ int64_t page_bytes() const { return (int64_t)page_size * (head_dim + head_dim / 4); }
    __device__ int64_t capacity() const { return (int64_t)table_width * page_size; }

    // sequence of row n, or -1.  The last b with starts[b] <= n; what does not ascend finds no sequence or one that holds n.
    __device__ int32_t sequence_of(int64_t n) const
    {
        int32_t lo = 0, hi = batch;             // invariant for ascending starts: starts[lo] <= n < starts[hi]
        while (hi - lo > 1) {
            const int32_t mid = lo + (hi - lo) / 2;
            if (starts[mid] <= n) lo = mid; else hi = mid;
        }
        return starts[lo] <= n && n < starts[lo + 1] ? lo : -1;
    }

    // start of the page of head h that holds token `position` of sequence b, or null
    __device__ uint8_t *page_of(int32_t b, int64_t position, int32_t h) const
    {
        if (position < 0 || position >= capacity()) return nullptr;
        const int32_t page = table[(int64_t)b * table_width + position / page_size];
        if (page < 0 || page >= pages) return nullptr;
        return pool + ((int64_t)page * kv_heads + h) * page_bytes();
    }
};

}  // namespace ppmm

#endif  // PPMM_DEVICE_HPP
