// Device helpers of the clear track: 16-bit types, and where the tokens of a batch lie in the paged cache.
#ifndef PPMM_DEVICE_HPP
#define PPMM_DEVICE_HPP

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ppmm.h"

namespace ppmm {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// The two 16-bit types.  kSixteen: the bits of 16.0; a 4-bit code in the top four mantissa bits, at kCodeBit, makes it 16 + code
// exactly.  kMinus24: the bits of -24.0 = -(16 + 8), twice.  mma: D = A B + C on a 16 x 16 tile with 32 values of k: lane l holds
// row (A) or column (B) l % 16 and k = 8 (l / 16) ... + 7, of C and D column l % 16 and rows 4 (l / 16) ... + 3.
struct BF16 {
    using type = __bf16;
    static constexpr int kCodeBit = 3;
    static constexpr uint32_t kSixteen = 0x41804180u, kMinus24 = 0xC1C0C1C0u;
    static __device__ inline f32x4 mma(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
struct FP16 {
    using type = _Float16;
    static constexpr int kCodeBit = 6;
    static constexpr uint32_t kSixteen = 0x4C004C00u, kMinus24 = 0xCE00CE00u;
    static __device__ inline f32x4 mma(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};

__device__ inline uint32_t rotate_right(uint32_t v, int by) { return __builtin_amdgcn_alignbit(v, v, by); }

// Eight codes -> eight values 16 + code.  Of the word's nibbles, counted from bit kCodeBit on and around the end, number i and
// number 4 + i become the pair i: a rotation and a mask-and-or each.  The instruction takes one constant from a scalar register, so
// the other one is kept in a vector register (as literals the compiler splits it in two, 11 instructions for 7).
template <class T> struct Unpacker {
    uint32_t mask, sixteen;
    __device__ inline Unpacker() : mask(0x000F000Fu << T::kCodeBit), sixteen(T::kSixteen) { asm("" : "+s"(mask), "+v"(sixteen)); }
    // kFirst: the bit at which nibble 0 lies
    template <int kFirst = T::kCodeBit> __device__ inline u32x4 get(uint32_t w) const
    {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int by = (4 * i + kFirst - T::kCodeBit + 32) % 32;
            v[i] = ((by ? rotate_right(w, by) : w) & mask) | sixteen;
        }
        return v;
    }
    __device__ inline u32x4 operator()(uint32_t w) const { return get(w); }
};

template <class T> __device__ inline float to_f32(uint16_t bits) { return (float)__builtin_bit_cast(typename T::type, bits); }
template <class T> __device__ inline uint16_t from_f32(float v) { return __builtin_bit_cast(uint16_t, (typename T::type)v); }   // to nearest even

// A pool and a batch as the kernels take them.  Offsets into the pool are 64-bit.
struct Cache {
    uint8_t *pool;
    int64_t pages;
    int32_t page_size, kv_heads, head_dim;
    const int32_t *starts, *lens, *table;
    int32_t batch, table_width;

    // bytes of one page of one head: [codes of keys][codes of values][scales and offsets of keys][of values]
    __device__ int64_t page_bytes() const { return (int64_t)page_size * (head_dim + head_dim / 4); }
    __device__ int64_t capacity() const { return (int64_t)table_width * page_size; }

    // sequence of row n, the same for the whole wave, or -1: 64 places at a time.  The last b with starts[b] <= n; where the starts do
    // not ascend, none or one that holds n.
    __device__ int32_t sequence_of(int64_t n) const
    {
        const int lane = threadIdx.x % 64;
        int32_t lo = 0;
        for (int32_t left = batch; left > 1;) {             // the sequence is among lo ... lo + left - 1
            const int32_t stride = (left + 63) / 64, at = lane * stride;
            const int below = __popcll(__ballot(at < left && starts[lo + (at < left ? at : 0)] <= n));
            if (below == 0) return -1;
            lo += (below - 1) * stride;
            left = left - (below - 1) * stride < stride ? left - (below - 1) * stride : stride;
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
