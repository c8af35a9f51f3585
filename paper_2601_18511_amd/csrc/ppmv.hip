// Products with weights held in 4 bits under group scales (include/ppmm.h; Section 5.1's linear layers for clear tokens), on
// MI355X (gfx950).
//
//     y[t][m] = sum_g s[m][g] sum_{k in g} (c[m][k] - 8) x[t][k]  +  sum_g o[m][g] sum_{k in g} x[t][k]
//
// A code never becomes a scaled 16-bit weight, which would round it: the matrix cores multiply x with 16 + c, which a 16-bit
// float holds exactly and which one mask-and-or makes of a code, and with -24 = -(16 + 8) in the same chain; the 32-bit sum over
// a group is then scaled.  The chain of -24 x also is the group's sum of x that the offsets need.
//
// Layout of a plan.  Blocks of 16 rows x 128 k, 1 KiB, in the order of the matrix instruction's operand: lane l has row l % 16
// and 16 bytes, word j of it k = 32 j + 8 (l / 16) ... + 7.  A wave fetches a block with one 16-byte load per lane, and a
// work-group's waves read neighbouring blocks.  What a lane needs of a block's scales (and offsets), its four rows of every group,
// lies side by side: 8 to 64 bytes.
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
    uint32_t *codes;     // [ceil(M/16)][ceil(K/128)][64 lanes][4 words]
    uint16_t *params;    // [ceil(M/16)][ceil(K/128)][4 quarters][128/group][scales, offsets if any][4 rows of the quarter]
    size_t bytes;
};

namespace {

using ppmm::BF16;
using ppmm::f32x4;
using ppmm::FP16;
using ppmm::u32x2;
using ppmm::u32x4;

struct Weights {
    const u32x4 *codes;
    const uint16_t *params;
};

// ---- packing -------------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void pack_codes_kernel(const uint8_t *codes, uint32_t *out, int64_t M, int64_t K, int64_t kblocks, int64_t first, int64_t words,
                                                         int code_bit)
{
    const int64_t idx = first + (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (idx >= first + words) return;
    const int j = (int)(idx % 4), lane = (int)(idx / 4 % 64);
    const int64_t block = idx / 256, m = block / kblocks * 16 + lane % 16, k = block % kblocks * 128 + 32 * j + 8 * (lane / 16);
    const int64_t half = (K + 1) / 2;
    uint32_t w = 0;
    if (m < M)
        for (int i = 0; i < 4; ++i) {
            const int64_t at = k / 2 + i;
            const uint32_t pair = at < half ? codes[m * half + at] : 0;
            w |= (pair & 15) << (4 * i) | (pair >> 4) << (16 + 4 * i);
        }
    out[idx] = w << code_bit | w >> (32 - code_bit);
}

__global__ __launch_bounds__(256) void pack_params_kernel(const uint16_t *scales, const uint16_t *offsets, uint16_t *out, int64_t M, int64_t groups,
                                                          int64_t kblocks, int per_block, int64_t first, int64_t count)
{
    const int64_t idx = first + (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (idx >= first + count) return;
    const int kinds = offsets ? 2 : 1;
    const int64_t row = idx % 4, kind = idx / 4 % kinds, in_block = idx / 4 / kinds % per_block, rest = idx / 4 / kinds / per_block;
    const int64_t quarter = rest % 4, kb = rest / 4 % kblocks, m = rest / 4 / kblocks * 16 + 4 * quarter + row, g = kb * per_block + in_block;
    out[idx] = m < M && g < groups ? (kind ? offsets : scales)[m * groups + g] : 0;
}

// ---- a few tokens --------------------------------------------------------------------------------------------------
// HBM-bound: the weights stream through once and every token rides along.  A work-group of kWaves waves takes 16 rows (of both
// matrices, if gated) and up to 16 tokens; its waves share out the blocks of K and add up through LDS.

// Eight values of one token from k on, zero behind K.  Elements are aligned to two bytes; the loads take any such address.
__device__ inline u32x4 load_x(const uint16_t *row, int64_t k, int64_t K)
{
    u32x4 v = {0, 0, 0, 0};
    if (k + 8 <= K) __builtin_memcpy(&v, row + k, 16);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < K) v[i / 2] |= (uint32_t)row[k + i] << (16 * (i % 2));
    return v;
}

template <class T> __device__ inline f32x4 four(u32x2 v)
{
    return f32x4{ppmm::to_f32<T>((uint16_t)v[0]), ppmm::to_f32<T>((uint16_t)(v[0] >> 16)), ppmm::to_f32<T>((uint16_t)v[1]), ppmm::to_f32<T>((uint16_t)(v[1] >> 16))};
}

__device__ inline float silu_times(float g, float u)
{
    return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * g)) * u;
}

// Scales and offsets of one block: kGroups groups of the lane's four rows.
template <int kGroups, bool kOffsets> struct Params {
    static constexpr int kKinds = kOffsets ? 2 : 1, kStride = kGroups * kKinds * 16;      // 16-bit words of a block
    static constexpr int kLoads = kGroups * kKinds > 1 ? kGroups * kKinds / 2 : 1;
    u32x2 v[kGroups * kKinds];
    __device__ inline void load(const uint16_t *block, int h)
    {
        const uint16_t *p = block + h * kGroups * kKinds * 4;
        if constexpr (kGroups * kKinds == 1) v[0] = *(const u32x2 *)p;
        else
#pragma unroll
            for (int i = 0; i < kGroups * kKinds; i += 2) {
                const u32x4 w = *(const u32x4 *)(p + 4 * i);
                v[i] = u32x2{w[0], w[1]};
                v[i + 1] = u32x2{w[2], w[3]};
            }
    }
};

// -24 times the sum of x over each group of a block, in every row of the tile
template <class T, int kGroups> __device__ inline void group_sums(f32x4 (&base)[kGroups], const u32x4 (&x)[4])
{
    constexpr int kSteps = 4 / kGroups;
    const u32x4 minus24 = {T::kMinus24, T::kMinus24, T::kMinus24, T::kMinus24};
#pragma unroll
    for (int j = 0; j < 4; ++j) base[j / kSteps] = T::mma(minus24, x[j], j % kSteps ? base[j / kSteps] : f32x4{0, 0, 0, 0});
}

// sum += block times the kTok tiles of x
template <class T, int kTok, int kGroups, bool kOffsets>
__device__ inline void add_block(const ppmm::Unpacker<T> &unpack, f32x4 (&sum)[kTok], u32x4 codes, const Params<kGroups, kOffsets> &p, const u32x4 (&x)[kTok][4],
                                 const f32x4 (&base)[kTok][kGroups])
{
    constexpr int kSteps = 4 / kGroups, kKinds = kOffsets ? 2 : 1;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        f32x4 acc[kTok];
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            const u32x4 v = unpack(codes[g * kSteps + j]);
#pragma unroll
            for (int t = 0; t < kTok; ++t) acc[t] = T::mma(v, x[t][g * kSteps + j], j ? acc[t] : base[t][g]);
        }
        const f32x4 s = four<T>(p.v[g * kKinds]);
#pragma unroll
        for (int t = 0; t < kTok; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[t][e] = fmaf(s[e], acc[t][e], sum[t][e]);
        if constexpr (kOffsets) {
            const f32x4 o = four<T>(p.v[g * kKinds + 1]) * (-1.0f / 24.0f);
#pragma unroll
            for (int t = 0; t < kTok; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[t][e] = fmaf(o[e], base[t][g][e], sum[t][e]);
        }
    }
    // The sums are finished here.  Sunk below a branch by the compiler they have read a matrix instruction's result too early: its
    // hazard waits were missing on the way through the branch, and the hardware has none.
#pragma unroll
    for (int t = 0; t < kTok; ++t) asm volatile("" : "+v"(sum[t]));
}

// Adds up what the waves left in part and stores 16 tokens of 16 rows: 256 threads finish a result each.
template <class T, int kWaves, bool kGated>
__device__ inline void finish(const f32x4 (&part)[kWaves][kGated ? 2 : 1][64], int64_t tile, int64_t M, int64_t tokens, uint16_t *y, int64_t ldy)
{
    constexpr int kMats = kGated ? 2 : 1;
    if (threadIdx.x >= 256) return;
    const int e = threadIdx.x % 4, l = threadIdx.x / 4;
    float v[kMats];
#pragma unroll
    for (int w = 0; w < kMats; ++w) {
        v[w] = 0.0f;
#pragma unroll
        for (int q = 0; q < kWaves; ++q) v[w] += part[q][w][l][e];
    }
    const int64_t m = tile * 16 + 4 * (l / 16) + e, n = l % 16;
    if (m < M && n < tokens) y[n * ldy + m] = ppmm::from_f32<T>(kGated ? silu_times(v[0], v[kMats - 1]) : v[0]);
}

// Up to four tokens whose rows fit LDS together.  Columns without a token carry the last one's values and are not stored.  With x
// out of the way nothing but weights is in the queue of loads, and a wave asks for its next block before it uses the present one;
// more blocks ahead (2 or 4) took registers and with them waves: 14336 x 4096 gated, group 64, 14.6 and 15.5 us for 14.0.
template <class T, int kWaves, int kGroups, bool kGated, bool kOffsets>
__global__ __launch_bounds__(64 * kWaves) void stream_kernel(Weights a, Weights b, int64_t M, int K, int kblocks, int tokens, const uint16_t *x,
                                                             int64_t ldx, uint16_t *y, int64_t ldy)
{
    constexpr int kMats = kGated ? 2 : 1;
    using Par = Params<kGroups, kOffsets>;
    extern __shared__ u32x4 rows[];                 // [tokens][kblocks * 16 + 1]
    __shared__ f32x4 part[kWaves][kMats][64];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), h = lane / 16, col = lane % 16;
    const int64_t tile = blockIdx.x;
    u32x4 codes[kMats];
    Par params[kMats];
    const auto fetch = [&](int kb) __attribute__((always_inline)) {
#pragma unroll
        for (int w = 0; w < kMats; ++w) {
            const Weights &m = w ? b : a;
            codes[w] = m.codes[(tile * kblocks + kb) * 64 + lane];
            params[w].load(m.params + (tile * kblocks + kb) * Par::kStride, h);
        }
    };
    if (wave < kblocks) fetch(wave);
    const int pitch = kblocks * 16 + 1;             // the odd one keeps the rows on different banks
    for (int t = 0; t < tokens; ++t)
        for (int i = threadIdx.x; i < kblocks * 16; i += 64 * kWaves) rows[t * pitch + i] = load_x(x + t * ldx, 8 * i, K);
    __syncthreads();
    const u32x4 *mine = rows + (col < tokens ? col : tokens - 1) * pitch + h;
    const ppmm::Unpacker<T> unpack;
    f32x4 sum[kMats][1] = {};
    for (int kb = wave; kb < kblocks; kb += kWaves) {
        u32x4 xs[1][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) xs[0][j] = mine[kb * 16 + 4 * j];
        f32x4 base[1][kGroups];
        group_sums<T, kGroups>(base[0], xs[0]);
#pragma unroll
        for (int w = 0; w < kMats; ++w) add_block<T, 1, kGroups, kOffsets>(unpack, sum[w], codes[w], params[w], xs, base);
        fetch(kb + kWaves < kblocks ? kb + kWaves : kb);
    }
#pragma unroll
    for (int w = 0; w < kMats; ++w) part[wave][w][lane] = sum[w][0];
    __syncthreads();
    finish<T, kWaves, kGated>(part, tile, M, tokens, y, ldy);
}

// Sixteen tokens of any length a work-group; x comes from the caches as the matrix instruction wants it.
template <class T, int kWaves, int kGroups, bool kGated, bool kOffsets>
__global__ __launch_bounds__(64 * kWaves) void few_tokens_kernel(Weights a, Weights b, int64_t M, int64_t K, int kblocks, int64_t all_tokens,
                                                                 const uint16_t *all_x, int64_t ldx, uint16_t *all_y, int64_t ldy)
{
    constexpr int kMats = kGated ? 2 : 1;
    using Par = Params<kGroups, kOffsets>;
    __shared__ f32x4 part[kWaves][kMats][64];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), h = lane / 16, col = lane % 16;
    const uint32_t tiles = (uint32_t)((M + 15) / 16);       // of rows; the next tokens come behind them all
    const int64_t tile = blockIdx.x % tiles, t0 = (int64_t)(blockIdx.x / tiles) * 16, tokens = all_tokens - t0;
    const uint16_t *row = all_x + (t0 + col) * ldx;
    u32x4 codes[kMats];
    Par params[kMats];
    const auto fetch = [&](int kb) __attribute__((always_inline)) {
#pragma unroll
        for (int w = 0; w < kMats; ++w) {
            const Weights &m = w ? b : a;
            codes[w] = m.codes[(tile * kblocks + kb) * 64 + lane];
            params[w].load(m.params + (tile * kblocks + kb) * Par::kStride, h);
        }
    };
    const ppmm::Unpacker<T> unpack;
    f32x4 sum[kMats][1] = {};
    if (wave < kblocks) fetch(wave);
    for (int kb = wave; kb < kblocks; kb += kWaves) {
        u32x4 xs[1][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            xs[0][j] = u32x4{0, 0, 0, 0};
            if (col < tokens) xs[0][j] = load_x(row, (int64_t)kb * 128 + 32 * j + 8 * h, K);
        }
        f32x4 base[1][kGroups];
        group_sums<T, kGroups>(base[0], xs[0]);
#pragma unroll
        for (int w = 0; w < kMats; ++w) add_block<T, 1, kGroups, kOffsets>(unpack, sum[w], codes[w], params[w], xs, base);
        fetch(kb + kWaves < kblocks ? kb + kWaves : kb);
    }
#pragma unroll
    for (int w = 0; w < kMats; ++w) part[wave][w][lane] = sum[w][0];
    __syncthreads();
    finish<T, kWaves, kGated>(part, tile, M, tokens, all_y + t0 * ldy, ldy);
}

// ---- a batch of tokens ---------------------------------------------------------------------------------------------
// Too many tokens to fetch x anew for every tile of rows, too few for large tiles.  Of a work-group's eight waves kRowWaves take 16
// rows each (of both matrices, if gated) with the same 16 kTok tokens out of LDS; kWays such teams take one block of K in kWays each
// and add up at the end.  Weights are asked for two steps ahead, x one.  64 tokens in groups of 32 have more values than registers: gated 13
// to 22 of them lie in memory (27 us a round of the chip for 15 with up to 48 tokens), plain with offsets 5 (bf16, two row waves).
constexpr int kBatchWaves = 8;

template <class T, int kTok, int kRowWaves, int kGroups, bool kGated, bool kOffsets>
__global__ __launch_bounds__(64 * kBatchWaves) void batch_kernel(Weights a, Weights b, int64_t M, int64_t K, int kblocks, int64_t all_tokens,
                                                                 const uint16_t *all_x, int64_t ldx, bool buffered, uint16_t *all_y, int64_t ldy)
{
    using Par = Params<kGroups, kOffsets>;
    constexpr int kMats = kGated ? 2 : 1, kPieces = kTok * 16 * 16, kWays = kBatchWaves / kRowWaves, kLoads = kTok * 4 / kRowWaves;
    __shared__ union {
        u32x4 x[2][kWays][kPieces];                 // two steps in turn, the block of each team
        f32x4 part[kWays - 1][kRowWaves][kMats][kTok][64];
    } lds;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), h = lane / 16, col = lane % 16;
    const int team = wave / kRowWaves, member = wave % kRowWaves;
    const int64_t tiles = (M + 15) / 16;
    const uint32_t sets = (uint32_t)((tiles + kRowWaves - 1) / kRowWaves);     // of rows; the next tokens come behind them all
    const int64_t t0 = (int64_t)(blockIdx.x / sets) * 16 * kTok;
    const int tokens = all_tokens - t0 < 16 * kTok ? (int)(all_tokens - t0) : 16 * kTok;
    const uint16_t *x = all_x + t0 * ldx;
    const int64_t own = (int64_t)(blockIdx.x % sets) * kRowWaves + member, tile = own < tiles ? own : tiles - 1;
    const auto rows = __builtin_amdgcn_make_buffer_rsrc((void *)x, 0, buffered ? (int)(((tokens - 1) * ldx + K) * 2) : 0, 0x00027000);
    const auto stage = [&](int step) __attribute__((always_inline)) {       // this team's block: a member brings 4 kLoads tokens
        const int kb = kWays * step + team;
        u32x4 *to = lds.x[step % 2][team] + member * kLoads * 64;
        int l = lane;
        asm volatile("" : "+v"(l));                 // the addresses are not kept from step to step
        if (buffered && (kb + 1) * 128 <= K) {
#pragma unroll
            for (int n = 0; n < kLoads; ++n) {
                const int token = (member * kLoads + n) * 4 + l / 16;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (__attribute__((address_space(3))) void *)(to + 64 * n), 16,
                                                         token * (int)ldx * 2 + ((l % 16 ^ token % 16) * 8 + kb * 128) * 2, 0, 0, 0);
            }
        } else if ((kb + 1) * 128 <= K) {           // rows that are not aligned: through registers
            constexpr int kHold = kLoads > 4 ? kLoads / 2 : kLoads;      // 1, 2, 3, 4, 6 or 8 loads in all
#pragma unroll
            for (int n0 = 0; n0 < kLoads; n0 += kHold) {
                u32x4 v[kHold];
#pragma unroll
                for (int n = 0; n < kHold; ++n) {
                    const int token = (member * kLoads + n0 + n) * 4 + l / 16;
                    v[n] = u32x4{0, 0, 0, 0};
                    if (token < tokens) __builtin_memcpy(&v[n], x + token * ldx + (int64_t)kb * 128 + 8 * (l % 16 ^ token % 16), 16);
                }
#pragma unroll
                for (int n = 0; n < kHold; ++n) to[64 * (n0 + n) + l] = v[n];
            }
        } else {                                    // the last block, part of it behind K
#pragma unroll 1
            for (int n = 0; n < kLoads; ++n) {
                const int token = (member * kLoads + n) * 4 + l / 16;
                to[64 * n + l] = token < tokens ? load_x(x + token * ldx, (int64_t)kb * 128 + 8 * (l % 16 ^ token % 16), K) : u32x4{0, 0, 0, 0};
            }
        }
    };
    struct Raw {
        u32x4 codes[kMats];
        Par params[kMats];
    };
    const auto fetch = [&](Raw &r, int step) __attribute__((always_inline)) {
        const int kb = kWays * step + team < kblocks ? kWays * step + team : kblocks - 1;      // behind the last block x is zero
#pragma unroll
        for (int w = 0; w < kMats; ++w) {
            const Weights &m = w ? b : a;
            r.codes[w] = (m.codes + (tile * kblocks + kb) * 64)[lane];
            r.params[w].load(m.params + (tile * kblocks + kb) * Par::kStride, h);
        }
    };
    const int steps = (kblocks + kWays - 1) / kWays;
    const ppmm::Unpacker<T> unpack;
    f32x4 sum[kMats][kTok] = {};
    Raw raw[2];
    const auto take = [&](Raw &r, int step) __attribute__((always_inline)) {
        // loads are counted in their order: this step's x is here, the weights asked for behind it may be under way
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kMats * (1 + Par::kLoads)) : "memory");
        __syncthreads();                            // everyone's x is, and nobody reads the other step's any more
        if (step + 1 < steps) stage(step + 1);
        asm volatile("" ::: "memory");
        const Raw now = r;
        fetch(r, step + 2);
        const u32x4 *from = lds.x[step % 2][team] + col * 16;
        u32x4 xs[kTok][4];
        f32x4 base[kTok][kGroups];
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
#pragma unroll
            for (int j = 0; j < 4; ++j) xs[t][j] = from[16 * t * 16 + ((4 * j + h) ^ col)];
            group_sums<T, kGroups>(base[t], xs[t]);
        }
#pragma unroll
        for (int w = 0; w < kMats; ++w) add_block<T, kTok, kGroups, kOffsets>(unpack, sum[w], now.codes[w], now.params[w], xs, base);
    };
    stage(0);
    asm volatile("" ::: "memory");
    fetch(raw[0], 0);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    fetch(raw[1], 1);
    for (int step = 0; step < steps; step += 2) {
        take(raw[0], step);
        if (step + 1 < steps) take(raw[1], step + 1);
    }
    __syncthreads();
    if (team)
#pragma unroll
        for (int w = 0; w < kMats; ++w)
#pragma unroll
            for (int t = 0; t < kTok; ++t) lds.part[team - 1][member][w][t][lane] = sum[w][t];
    __syncthreads();
    if (team || own >= tiles) return;
#pragma unroll
    for (int t = 0; t < kTok; ++t) {
        const int n = 16 * t + col;
        if (n >= tokens) continue;
        f32x4 v[kMats];
#pragma unroll
        for (int w = 0; w < kMats; ++w) {
            v[w] = sum[w][t];
#pragma unroll
            for (int q = 0; q < kWays - 1; ++q) v[w] += lds.part[q][member][w][t][lane];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t m = own * 16 + 4 * h + e;
            if (m < M) all_y[(t0 + n) * ldy + m] = ppmm::from_f32<T>(kGated ? silu_times(v[0][e], v[kMats - 1][e]) : v[0][e]);
        }
    }
}

// ---- many tokens ---------------------------------------------------------------------------------------------------
// MFMA-bound.  A work-group of 2 x 2 waves takes 128 rows (64 of either matrix, if gated) and 128 tokens, a wave 64 x 64; x goes
// through LDS in blocks of 128 k, two of them in turn, and codes go straight from memory to the registers of the wave that
// unpacks them.  The 16-byte pieces of a token's row lie in LDS at place p ^ (token % 16): the sixteen rows that a read takes
// them from are on different banks.
//
// 4096 -> 4096 of 3968 tokens: 162 us.  About 34 of them do not depend on K (K = 128 takes 37: the start and 32 MB of results, stored by
// two bytes); the rest runs at 1.0 PFLOP/s, with a fifth of the matrix instructions making -24 sum x.  4096 tokens, which fill both
// rounds of the chip, take the same.  With offsets 9 to 14 registers lie in memory (bf16 in groups of 128, fp16 in groups of 32).
constexpr int kTileRows = 128, kTileTokens = 128;

template <class T, int kGroups, bool kGated, bool kOffsets>
__global__ __launch_bounds__(256, 2) void many_tokens_kernel(Weights a, Weights b, int64_t M, int64_t K, int kblocks, int64_t tokens, uint32_t row_tiles,
                                                             uint32_t token_tiles, const uint16_t *x, int64_t ldx, bool buffered, uint16_t *y, int64_t ldy)
{
    using Par = Params<kGroups, kOffsets>;
    constexpr int kSteps = 4 / kGroups, kMats = kGated ? 2 : 1, kRows = 4 / kMats;
    __shared__ u32x4 tile[2][kTileTokens * 16];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), h = lane / 16, col = lane % 16;
    // An XCD gets neighbouring tiles: eight tiles of tokens and all rows, then the next eight.
    const uint32_t all = row_tiles * token_tiles, share = (all + 7) / 8;
    const uint32_t id = blockIdx.x % 8 * share + blockIdx.x / 8;
    if (id >= all) return;                          // the whole work-group
    const uint32_t strip = id / (8 * row_tiles), width = token_tiles - 8 * strip < 8 ? token_tiles - 8 * strip : 8, in = id - strip * 8 * row_tiles;
    const int64_t t0 = (int64_t)(8 * strip + in % width) * kTileTokens, first = (int64_t)(in / width) * (kTileRows / 16 / kMats) + wave / 2 * kRows;
    const int64_t tiles = (M + 15) / 16;
    const u32x4 *codes_of[4];
    const uint16_t *params_of[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {                   // a tile behind the last one is the last one once more
        const Weights &w = i / kRows ? b : a;
        const int64_t at = first + i % kRows < tiles ? first + i % kRows : tiles - 1;
        codes_of[i] = w.codes + at * kblocks * 64;
        params_of[i] = w.params + at * kblocks * Par::kStride;
    }
    // x: a wave brings 32 tokens, four at a time, a lane the piece that belongs at its own place.  Whole blocks go to LDS without a
    // register in between; the buffer ends with the tile's last token, and what lies behind reads as zero.
    const int64_t held = tokens - t0 < kTileTokens ? tokens - t0 : kTileTokens;
    const auto rows = __builtin_amdgcn_make_buffer_rsrc((void *)(x + t0 * ldx), 0, buffered ? (int)(((held - 1) * ldx + K) * 2) : 0, 0x00027000);
    const auto stage = [&](int kb) __attribute__((always_inline)) {
        u32x4 *to = tile[kb % 2] + wave * 32 * 16;
        // opaque, so that nothing of the addresses is kept in registers from one block to the next
        int l = lane;
        const uint16_t *from = x;
        asm volatile("" : "+v"(l), "+s"(from));
        if (buffered && (kb + 1) * 128 <= K) {
#pragma unroll
            for (int n = 0; n < 8; ++n)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (__attribute__((address_space(3))) void *)(to + 64 * n), 16,
                                                         (wave * 32 + 4 * n + l / 16) * (int)ldx * 2 + ((l % 16 ^ (4 * n + l / 16) % 16) * 8 + kb * 128) * 2, 0, 0, 0);
        } else if ((kb + 1) * 128 <= K) {           // rows that are not aligned: through registers, four at a time (1000 tokens 4001 ->
                                                    // 4099: 121 us, one at a time 160; aligned rows of that size take 64)
#pragma unroll
            for (int n0 = 0; n0 < 8; n0 += 4) {
                u32x4 v[4];
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const int token = wave * 32 + 4 * (n0 + n) + l / 16;
                    v[n] = u32x4{0, 0, 0, 0};
                    if (token < held) __builtin_memcpy(&v[n], from + (t0 + token) * ldx + (int64_t)kb * 128 + 8 * (l % 16 ^ token % 16), 16);
                }
#pragma unroll
                for (int n = 0; n < 4; ++n) to[64 * (n0 + n) + l] = v[n];
            }
        } else {                                    // the last block, part of it behind K
#pragma unroll 1
            for (int n = 0; n < 8; ++n) {
                const int token = wave * 32 + 4 * n + l / 16;
                to[64 * n + l] = token < held ? load_x(from + (t0 + token) * ldx, (int64_t)kb * 128 + 8 * (l % 16 ^ token % 16), K) : u32x4{0, 0, 0, 0};
            }
        }
    };
    u32x4 codes[4];
    Par params[4];
    const auto fetch = [&](int kb) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            codes[i] = (codes_of[i] + (int64_t)kb * 64)[lane];
            params[i].load(params_of[i] + (int64_t)kb * Par::kStride, h);
        }
    };
    const u32x4 minus24 = {T::kMinus24, T::kMinus24, T::kMinus24, T::kMinus24};
    const ppmm::Unpacker<T> unpack;
    f32x4 sum[4][4] = {};
    stage(0);
    asm volatile("" ::: "memory");
    fetch(0);
    for (int kb = 0; kb < kblocks; ++kb) {
        // this wave's part of the block is in LDS; the loads of weights behind it may be under way
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 + 4 * Par::kLoads) : "memory");
        __syncthreads();                                        // everyone's is, and nobody reads the other block any more
        // Loads are counted in their order: the wait for this block's codes stands here, in front of the next loads of x, or it would
        // be a wait for those too; and the next codes come behind them.
        asm volatile("" : "+v"(codes[0]), "+v"(codes[1]), "+v"(codes[2]), "+v"(codes[3]));
        if (kb + 1 < kblocks) stage(kb + 1);
        asm volatile("" ::: "memory");
        const u32x4 *from = tile[kb % 2] + (wave % 2 * 64 + col) * 16;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            u32x4 v[4][kSteps];
            f32x4 s[4], o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int j = 0; j < kSteps; ++j) v[i][j] = unpack(codes[i][g * kSteps + j]);
                s[i] = four<T>(params[i].v[g * Par::kKinds]);
                if constexpr (kOffsets) o[i] = four<T>(params[i].v[g * 2 + 1]) * (-1.0f / 24.0f);
            }
            if (g == kGroups - 1) fetch(kb + 1 < kblocks ? kb + 1 : kb);      // without a branch: sums would sink below it
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                u32x4 xs[kSteps];
#pragma unroll
                for (int j = 0; j < kSteps; ++j) xs[j] = from[16 * t * 16 + ((4 * (g * kSteps + j) + h) ^ col)];
                f32x4 base = {0, 0, 0, 0}, acc[4];
#pragma unroll
                for (int j = 0; j < kSteps; ++j) base = T::mma(minus24, xs[j], base);
#pragma unroll
                for (int j = 0; j < kSteps; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[i] = T::mma(v[i][j], xs[j], j ? acc[i] : base);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sum[i][t][e] = fmaf(s[i][e], acc[i][e], sum[i][t][e]);
                        if constexpr (kOffsets) sum[i][t][e] = fmaf(o[i][e], base[e], sum[i][t][e]);
                    }
                if constexpr (kGroups == 4) if (t == 1) __builtin_amdgcn_sched_barrier(0);
            }
            // the compiler otherwise starts on the other groups at once and runs out of registers
            __builtin_amdgcn_sched_barrier(0);
        }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int64_t n = t0 + wave % 2 * 64 + 16 * t + col;
        if (n >= tokens) continue;
#pragma unroll
        for (int i = 0; i < kRows; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t m = (first + i) * 16 + 4 * h + e;
                if (m < M) y[n * ldy + m] = ppmm::from_f32<T>(kGated ? silu_times(sum[i][t][e], sum[i + kRows * (kMats - 1)][t][e]) : sum[i][t][e]);
            }
    }
}

struct Call {
    const ppmv_plan *p, *u;
    int64_t T;
    const uint16_t *x;
    int64_t ldx;
    uint16_t *y;
    int64_t ldy;
    hipStream_t stream;
};

// x in aligned pieces, and 32-bit offsets in a tile of 128 tokens
bool buffered(const Call &c) { return ((uintptr_t)c.x & 15) == 0 && c.ldx % 8 == 0 && c.ldx < (1 << 22); }

template <class T, int kGroups, bool kGated> void launch_few(const Call &c)
{
    const ppmv_plan *p = c.p, *u = c.u;
    const Weights a{(const u32x4 *)p->codes, p->params}, b{(const u32x4 *)u->codes, u->params};
    auto kernel = p->has_offsets ? few_tokens_kernel<T, 8, kGroups, kGated, true> : few_tokens_kernel<T, 8, kGroups, kGated, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((p->M + 15) / 16 * ((c.T + 15) / 16))), dim3(64 * 8), 0, c.stream, a, b, p->M, p->K,
                       (int)((p->K + 127) / 128), c.T, c.x, c.ldx, c.y, c.ldy);
}

template <class T, int kWaves, int kGroups, bool kGated> void launch_stream(const Call &c)
{
    const ppmv_plan *p = c.p, *u = c.u;
    const int kblocks = (int)((p->K + 127) / 128);
    const Weights a{(const u32x4 *)p->codes, p->params}, b{(const u32x4 *)u->codes, u->params};
    auto kernel = p->has_offsets ? stream_kernel<T, kWaves, kGroups, kGated, true> : stream_kernel<T, kWaves, kGroups, kGated, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((p->M + 15) / 16)), dim3(64 * kWaves), (size_t)c.T * (kblocks * 16 + 1) * 16, c.stream, a, b, p->M, (int)p->K,
                       kblocks, (int)c.T, c.x, c.ldx, c.y, c.ldy);
}

template <class T, int kGroups, bool kGated> void launch_many(const Call &c)
{
    const ppmv_plan *p = c.p, *u = c.u;
    const int64_t rows = kGated ? kTileRows / 2 : kTileRows;
    const uint32_t row_tiles = (uint32_t)((p->M + rows - 1) / rows), token_tiles = (uint32_t)((c.T + kTileTokens - 1) / kTileTokens);
    const Weights a{(const u32x4 *)p->codes, p->params}, b{(const u32x4 *)u->codes, u->params};
    auto kernel = p->has_offsets ? many_tokens_kernel<T, kGroups, kGated, true> : many_tokens_kernel<T, kGroups, kGated, false>;
    // check_product: at most 2^22 tiles of 16 x 64, so these count in 32 bits and launch fewer than 2^32 threads
    hipLaunchKernelGGL(kernel, dim3((row_tiles * token_tiles + 7) / 8 * 8), dim3(256), 0, c.stream, a, b, p->M, p->K, (int)((p->K + 127) / 128), c.T, row_tiles,
                       token_tiles, c.x, c.ldx, buffered(c), c.y, c.ldy);
}

template <class T, int kTok, int kRowWaves, int kGroups, bool kGated> void launch_batch(const Call &c)
{
    const ppmv_plan *p = c.p, *u = c.u;
    const Weights a{(const u32x4 *)p->codes, p->params}, b{(const u32x4 *)u->codes, u->params};
    auto kernel = batch_kernel<T, kTok, kRowWaves, kGroups, kGated, false>;
    if constexpr (ppmm_host::batch_has(16 * kTok, kGated, 128 / kGroups, true))
        if (p->has_offsets) kernel = batch_kernel<T, kTok, kRowWaves, kGroups, kGated, true>;
    const dim3 grid((unsigned)(((p->M + 15) / 16 + kRowWaves - 1) / kRowWaves * ((c.T + 16 * kTok - 1) / (16 * kTok))));
    hipLaunchKernelGGL(kernel, grid, dim3(64 * kBatchWaves), 0, c.stream, a, b, p->M, p->K, (int)((p->K + 127) / 128), c.T, c.x, c.ldx, buffered(c), c.y,
                       c.ldy);
}

template <class T, int kRowWaves, int kGroups, bool kGated> void launch_batches(const Call &c, int tokens)
{
    if (tokens == 16) launch_batch<T, 1, kRowWaves, kGroups, kGated>(c);
    else if (tokens == 32) launch_batch<T, 2, kRowWaves, kGroups, kGated>(c);
    else if (tokens == 48) launch_batch<T, 3, kRowWaves, kGroups, kGated>(c);
    else launch_batch<T, 4, kRowWaves, kGroups, kGated>(c);
}

template <class T, int kGroups, bool kGated> void launch(const Call &c)
{
    using ppmm_host::Form;
    const Form form = ppmm_host::choose(c.p->M, c.p->K, c.T, c.p->group, kGated, c.p->has_offsets);
    if (form.kernel == Form::kMany) return launch_many<T, kGroups, kGated>(c);
    if (form.kernel == Form::kFew) return launch_few<T, kGroups, kGated>(c);
    if (form.kernel == Form::kBatch) {
        if (form.waves == 2) return launch_batches<T, 2, kGroups, kGated>(c, form.tokens);
        return launch_batches<T, 4, kGroups, kGated>(c, form.tokens);
    }
    if constexpr (ppmm_host::stream_has(16, kGated, 128 / kGroups))
        if (form.waves == 16) return launch_stream<T, 16, kGroups, kGated>(c);
    launch_stream<T, 8, kGroups, kGated>(c);
}

template <class T, bool kGated> void by_group(const Call &c)
{
    if (c.p->group == 128) launch<T, 1, kGated>(c);
    else if (c.p->group == 64) launch<T, 2, kGated>(c);
    else launch<T, 4, kGated>(c);
}

template <bool kGated>
pcmm_status run(const ppmv_plan *p, const ppmv_plan *u, int64_t T, const void *x, int64_t ldx, void *y, int64_t ldy, void *stream)
{
    bool nothing;
    const pcmm_status rc = ppmm_host::check_product(p->M, p->K, T, x, ldx, y, ldy, &nothing);
    if (rc != PCMM_OK || nothing) return rc;
    pcmm_hip_util::DevGuard dg(p->device);
    if (!dg.ok) return PCMM_EDEVICE;
    const Call c{p, u, T, (const uint16_t *)x, ldx, (uint16_t *)y, ldy, (hipStream_t)stream};
    if (p->type == PPMM_BF16) by_group<BF16, kGated>(c);
    else by_group<FP16, kGated>(c);
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
    const int64_t tiles = (M + 15) / 16, kblocks = (K + 127) / 128, words = tiles * kblocks * 256;
    const int64_t count = tiles * kblocks * (128 / group) * (offsets_dev ? 32 : 16);
    pcmm_status rc = PCMM_OK;
    if (hipMalloc((void **)&p->codes, (size_t)words * 4) != hipSuccess || hipMalloc((void **)&p->params, (size_t)count * 2) != hipSuccess) {
        (void)hipGetLastError();
        rc = PCMM_ENOMEM;
    }
    p->bytes = (size_t)words * 4 + (size_t)count * 2;
    if (rc == PCMM_OK) {
        // check_weights holds words to 2^33; no launch has 2^32 threads or more
        const int64_t most = (int64_t)1 << 31;
        for (int64_t at = 0; at < words; at += most) {
            const int64_t n = words - at < most ? words - at : most;
            hipLaunchKernelGGL(pack_codes_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, codes_dev, p->codes, M, K, kblocks, at, n,
                               type == PPMM_BF16 ? BF16::kCodeBit : FP16::kCodeBit);
        }
        for (int64_t at = 0; at < count; at += most) {
            const int64_t n = count - at < most ? count - at : most;
            hipLaunchKernelGGL(pack_params_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, (const uint16_t *)scales_dev,
                               (const uint16_t *)offsets_dev, p->params, M, (K + group - 1) / group, kblocks, 128 / group, at, n);
        }
        if (hipGetLastError() != hipSuccess || hipStreamSynchronize(st) != hipSuccess) rc = PCMM_EDEVICE;
    }
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
    (void)hipFree(plan->params);
    delete plan;
}

}  // extern "C"
