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
using ppmm::f32x4;
using ppmm::FP16;
using ppmm::u32x4;

constexpr int kThreads = 256;

// Places inside a page of one head.  A token's D/2 bytes of codes are words of eight codes; the words of a value lie in order, its
// channels from the lowest four bits up.  The words of a key are transposed: word (D/32) h + j holds channels 32 j + 8 h ... + 7, so
// that a lane of the matrix instruction (quarter h) reads its words of all groups at once; of the eight channels the even ones are
// nibbles 0..3 and the odd ones 4..7, and the word is rotated by three bits, as Unpacker wants them.  A token's scales (one for
// each group) lie in front of its offsets.
constexpr int kKeyBit = BF16::kCodeBit;

template <int D> __device__ inline int64_t codes_at(const Cache &c, int which, int slot) { return (int64_t)(which * c.page_size + slot) * (D / 2); }
template <int D> __device__ inline int64_t params_at(const Cache &c, int which, int slot)
{
    return (int64_t)c.page_size * D + (int64_t)(which * c.page_size + slot) * (D / 8);
}

// word of eight codes, in the order of the channels, as a key's word, and back
__device__ inline uint32_t key_word(uint32_t w)
{
    uint32_t v = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) v |= (w >> (8 * i) & 15) << (4 * i) | (w >> (8 * i + 4) & 15) << (4 * i + 16);
    return v << kKeyBit | v >> (32 - kKeyBit);
}
__device__ inline uint32_t code_of(uint32_t word, int which, int i)       // channel i of the word
{
    if (which) return word >> (4 * i) & 15;
    return ppmm::rotate_right(word, (4 * (i / 2) + 16 * (i % 2) + kKeyBit) % 32) & 15;
}

// ---- writing -------------------------------------------------------------------------------------------------------
// The sequence of every lane's row.  A wave's rows follow one another: it looks for one after the other together.
__device__ inline int32_t sequences(const Cache &c, int64_t n)
{
    const int64_t first = (int64_t)__builtin_amdgcn_readfirstlane((int)n), last = (int64_t)__builtin_amdgcn_readlane((int)n, 63);      // below 2^31
    int32_t mine = -1;
    for (int64_t t = first; t <= last; ++t) {
        const int32_t b = c.sequence_of(t);
        if (n == t) mine = b;
    }
    return mine;
}

// A thread takes eight channels (16 bytes), four neighbouring threads a group.  The grid is filled up to whole waves, and a lane
// without a row looks for its sequence with the others.
//
// A code is rint((x - b) / s) - 16 of the 64-bit quotient.  In 32 bits the quotient is off by less than `unsure`, so its nearest
// whole number is the right one unless it is that close to the middle of two; only then it is divided in 64 bits.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void append_kernel(Cache c, int64_t tokens, const uint16_t *k, int64_t kts, int64_t khs,
                                                          const uint16_t *v, int64_t vts, int64_t vhs)
{
    const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int part = (int)(idx % (D / 8));
    const uint32_t row = (uint32_t)(idx / (D / 8)); // (token, K or V, head): below 2^32 threads
    const int head = (int)(row % (uint32_t)c.kv_heads);
    const int which = (int)(row / (uint32_t)c.kv_heads % 2);
    const int64_t n = row / (uint32_t)c.kv_heads / 2;
    u32x4 bits = {0, 0, 0, 0};                      // asked for before the place is looked up
    if (n < tokens) __builtin_memcpy(&bits, (which ? v + n * vts + head * vhs : k + n * kts + head * khs) + part * 8, 16);
    const int32_t b = sequences(c, n);
    if (n >= tokens || b < 0) return;               // whole groups of threads leave together
    const int64_t position = (int64_t)c.lens[b] - (c.starts[b + 1] - n);
    uint8_t *page = c.page_of(b, position, head);
    if (!page) return;
    float x[8];
    float low = INFINITY, high = -INFINITY;
    bool finite = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = ppmm::to_f32<T>((uint16_t)(bits[i / 2] >> (16 * (i % 2))));
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
    uint32_t word = 0;
    if (s > 0.0f) {
        // x - b is off by 2^-24 (|x| + |b|), 1 / s and the product by 2^-23 of the quotient, which is below 64: within 2^-21 (|b| / s + 64)
        const float off = ppmm::to_f32<BF16>(b_bits), each = 1.0f / s, unsure = 0x1p-20f * (fabsf(off) * each + 64.0f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float quotient = (x[i] - off) * each;
            float steps = rintf(quotient);
            if (!(fabsf(quotient - steps) < 0.5f - unsure)) steps = (float)rint(((double)x[i] - (double)off) / (double)s);
            word |= (uint32_t)(int)fminf(fmaxf(steps - 16.0f, 0.0f), 15.0f) << (4 * i);
        }
    }
    const int slot = (int)(position % c.page_size);
    const int j = part / 4, h = part % 4;
    const int place = which ? part : (D / 32) * h + j;
    *(uint32_t *)(page + codes_at<D>(c, which, slot) + 4 * place) = which ? word : key_word(word);
    uint16_t *params = (uint16_t *)(page + params_at<D>(c, which, slot));
    if (h == 0) params[j] = s_bits;
    if (h == 1) params[D / 32 + j] = b_bits;
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
    const uint32_t row = (uint32_t)(idx / (D / 8));
    const int head = (int)(row % (uint32_t)c.kv_heads);
    const int which = (int)(row / (uint32_t)c.kv_heads % 2);
    const int64_t n = row / (uint32_t)c.kv_heads / 2;
    const int32_t b = sequences(c, n);
    if (n >= tokens || b < 0 || !(which ? v : k)) return;
    const int64_t position = (int64_t)c.lens[b] - (c.starts[b + 1] - n);
    const uint8_t *page = c.page_of(b, position, head);
    uint16_t *dst = (which ? v + n * vts + head * vhs : k + n * kts + head * khs) + part * 8;
    const int j = part / 4, h = part % 4;
    uint32_t word = 0;
    float s = 0.0f, off = 0.0f;
    if (page) {
        const int slot = (int)(position % c.page_size);
        word = *(const uint32_t *)(page + codes_at<D>(c, which, slot) + 4 * (which ? part : (D / 32) * h + j));
        const uint16_t *params = (const uint16_t *)(page + params_at<D>(c, which, slot));
        s = ppmm::to_f32<BF16>(params[j]);
        off = ppmm::to_f32<BF16>(params[D / 32 + j]);
    }
    u32x4 bits = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        bits[i / 2] |= (uint32_t)as_result<T>(fmaf(s, 16.0f + (float)code_of(word, which, i), off), fixed) << (16 * (i % 2));
    __builtin_memcpy(dst, &bits, 16);
}

// ---- attention -----------------------------------------------------------------------------------------------------
// Tiles of 64 keys, 16 at a time as the rows of a matrix product with queries as its columns.  Nothing is dequantised:
//
//   score     sum_j s_j (sum_{c in j} q_c (16 + code_c))  +  sum_j b_j sum_{c in j} q_c
//   output    sum_i (p_i s_ij) (16 + code_ic - 24)        +  sum_i p_i (b_ij + 24 s_ij)  for a channel c of group j
//
// q (16 + code) is exact.  p s enters as two bf16 numbers, rounded to 16 bits or more, and -24 p s as the same numbers' product with
// -24: what their rounding leaves out is weighed with code - 8.  Every tile's sum starts with it, so that no sum grows by 24 p s, which the
// offsets would take off again only at the end: of 3968 tokens' results in bf16 2.5 % were not the nearest number to the exact one
// without it (and with the first number cut instead of rounded), 0.26 % are; 564 and 620 us.  Three bf16 parts, all bits of p s: 0.18 %, 654 us.
// A key's scales and offsets are 16 bytes, which are an operand of the matrix instruction as they are: times a one (and 24 for the
// scale beside its offset) they come out in the layout of the scores, times the groups' sums of q (in three bf16 parts) they are the
// score's second sum.  The values' codes go through LDS, whose transposing read hands a lane sixteen keys of one channel.  The sixteen
// keys are those whose scores the lane holds, so probabilities stay where they are.
//
// Few queries (kFew): a column is a pair of group and query, 16 / (D/32) queries a tile: the products of all groups with their
// scales are one instruction each, and lanes do not work on empty columns.  Otherwise a column is a query, and the groups follow one
// another.
//
// The four waves of a work-group share out the tiles of its keys and join at the end; where there are few rows, several
// work-groups share out the keys of a row and a second kernel joins them.

// over the four lanes of a column
__device__ inline float across_quarters(float v) { v += __shfl_xor(v, 16); return v + __shfl_xor(v, 32); }
__device__ inline float most_of_quarters(float v)
{
    const uint32_t a = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);        // the even rows of lanes twice, and the odd ones
    v = fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
    const uint32_t c = __builtin_bit_cast(uint32_t, v);
    const auto t = __builtin_amdgcn_permlane32_swap(c, c, false, false);        // the lower half twice, and the upper one
    return fmaxf(__builtin_bit_cast(float, (uint32_t)t[0]), __builtin_bit_cast(float, (uint32_t)t[1]));
}
template <int kCtrl> __device__ inline float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), kCtrl, 0xf, 0xf, true));
}
constexpr int kRor4 = 0x124, kRor8 = 0x128;         // rotations of 16 lanes

__device__ inline uint32_t high_part(float v) { return __builtin_bit_cast(uint32_t, v) & 0xffff0000u; }
__device__ inline float as_float(uint32_t v) { return __builtin_bit_cast(float, v); }
__device__ inline uint32_t pack_bf16(float lo, float hi)       // to nearest even
{
    typedef __bf16 Pair __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, Pair{(__bf16)lo, (__bf16)hi});
}

// 64 lanes' 16 or 4 bytes from memory to neighbouring places in LDS, without a register in between
typedef const __attribute__((address_space(1))) void *GlobalPtr;
typedef __attribute__((address_space(3))) void *LdsPtr;
__device__ inline void pieces_to_lds(uint64_t from, void *to) { __builtin_amdgcn_global_load_lds((GlobalPtr)from, (LdsPtr)to, 16, 0, 0); }
__device__ inline void words_to_lds(uint64_t from, void *to) { __builtin_amdgcn_global_load_lds((GlobalPtr)from, (LdsPtr)to, 4, 0, 0); }

// a token's scales and offsets as an operand: the first words of a lane's sixteen bytes
template <int kWords, class Words> __device__ inline u32x4 operand(Words v)
{
    u32x4 r = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < kWords; ++w) r[w] = v[w];
    return r;
}

// Rows of one sequence and K/V head: row r is new token r / G, head G * kv_head + r % G.
struct Rows {
    int64_t first, next, tokens, length, capacity;
    uint32_t G;
    int32_t kv_head;
    bool causal;
    __device__ inline int64_t token(uint32_t r) const { return first + r / G; }
    __device__ inline int32_t limit(uint32_t r) const        // keys that row r attends to
    {
        const int64_t held = length < capacity ? length : capacity, own = length - (next - token(r)) + 1;
        const int64_t n = causal && own < held ? own : held;
        return n > 0 ? (int32_t)n : 0;                      // the capacity is below 2^31
    }
};

// A row's result.  Without keys both sums are zero, and so is the row; where all keys are NaN no maximum was found and l is zero
// too, but not v.
template <class T> __device__ inline uint16_t divided(float v, float l) { return ppmm::from_f32<T>(v / (l == 0.0f ? 1.0f : l)); }

// Keys of one split: a multiple of unit, which is whole rounds of the four waves.
__device__ inline int64_t split_size(int64_t length, int splits, int unit)
{
    const uint32_t n = length > 0 ? (uint32_t)length : 0;
    return (int64_t)((n + splits - 1) / splits + unit - 1) / unit * unit;
}

template <class T, int D, int kTiles, bool kFew>
__global__ __launch_bounds__(256, 2) void attention_kernel(Cache c, int64_t tokens, int32_t heads, const uint16_t *q, int64_t qts, int64_t qhs, uint16_t *out,
                                                           int64_t ots, int64_t ohs, float scale, int32_t causal, int32_t max_q, uint32_t row_sets, int32_t splits, int32_t unit, float *scratch)
{
    constexpr int kGroups = D / 32, kChannelTiles = D / 16, kQueries = kFew ? 16 / kGroups : 16, kRows = kQueries * kTiles;
    typedef uint32_t Words __attribute__((ext_vector_type(kGroups)));       // a lane's codes, and a token's scales and offsets
    struct Tile {                                   // as in the pages, but a value's 16-byte pieces lie at place piece ^ (token / 4)
        u32x4 keys[64 * D / 32], values[64 * D / 32];
        Words key_params[64], value_params[64];
    };
    __shared__ union {                              // the waves' tiles, and after the last key their results
        Tile tiles[4][2];                           // with D = 128 half of a compute unit's 160 KiB to the byte
        struct {
            float joined[4][kQueries][D + 4], stats[2][4][kTiles][16];
        } end;
    } lds;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), h = lane / 16, col = lane % 16;
    // Heads first, then sequences, then sets of rows from the last one on (they attend to the most), then splits: neighbouring
    // work-groups go to different XCDs, and what neighbours have to do should be alike.
    uint32_t id = blockIdx.x;
    const int32_t kv_head = id % c.kv_heads;
    id /= c.kv_heads;
    const int32_t b = id % c.batch;
    id /= c.batch;
    const uint32_t set = row_sets - 1 - id % row_sets;
    const int32_t split = id / row_sets;
    Rows rows{c.starts[b], c.starts[b + 1], tokens, c.lens[b], c.capacity(), (uint32_t)(heads / c.kv_heads), kv_head, causal != 0};
    const int64_t news = rows.next - rows.first < max_q ? rows.next - rows.first : max_q;
    if (news <= 0) return;
    const uint32_t count = (uint32_t)news * rows.G, row0 = set * kRows;       // max_q * G is below 2^31
    if (row0 >= count) return;
    const int32_t held = (int32_t)(rows.length < rows.capacity ? rows.length : rows.capacity);
    const int64_t part = split_size(held, splits, unit);
    const int64_t begin = split * part;
    if (split > 0 && begin >= held) return;
    const uint32_t last = row0 + kRows < count ? row0 + kRows - 1 : count - 1;
    const int32_t end = rows.limit(last) < begin + part ? rows.limit(last) : (int32_t)(begin + part);      // behind the keys of any row
    const int32_t clear = rows.limit(row0);         // keys in front of this belong to every row

    const int mine = kFew ? col / kQueries : 0;     // the column's group
    const int query = kFew ? col % kQueries : col;
    // the column's queries as the second operand, and its sums in three parts, one a quarter of the lanes
    u32x4 qs[kTiles][kGroups], qsum[kTiles];
    int32_t limit[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const uint32_t r = row0 + t * kQueries + query;
        const int64_t n = rows.token(r);
        const bool live = r < count && n >= 0 && n < tokens;
        limit[t] = live ? rows.limit(r) : 0;
        qsum[t] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            u32x4 v = {0, 0, 0, 0};
            if (live && (!kFew || mine == j)) __builtin_memcpy(&v, q + n * qts + (rows.kv_head * rows.G + r % rows.G) * qhs + 32 * j + 8 * h, 16);
            qs[t][j] = v;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += ppmm::to_f32<T>((uint16_t)v[i]) + ppmm::to_f32<T>((uint16_t)(v[i] >> 16));
            sum = across_quarters(sum);
            const uint32_t p0 = high_part(sum), p1 = high_part(sum - as_float(p0)), p2 = high_part(sum - as_float(p0) - as_float(p1));
            const uint32_t p = h == 0 ? p0 : h == 1 ? p1 : h == 2 ? p2 : 0;
            qsum[t][(kGroups + j) / 2] |= (kGroups + j) % 2 ? p : p >> 16;
        }
    }
    // ones that bring out a scale, and an offset with 24 scales: of the column's group, or of every group in all columns
    constexpr int kSums = kFew ? 1 : kGroups;
    u32x4 one_s[kSums], one_b[kSums];
#pragma unroll
    for (int n = 0; n < kSums; ++n) {
        one_s[n] = one_b[n] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < kGroups; ++j)
            if (h == 0 && (kFew ? mine == j : n == j)) {
                one_s[n][j / 2] = j % 2 ? 0x3f800000u : 0x3f80u;
                one_b[n][j / 2] = j % 2 ? 0x41c00000u : 0x41c0u;
                one_b[n][(kGroups + j) / 2] = (kGroups + j) % 2 ? 0x3f800000u : 0x3f80u;
            }
    }
    f32x4 o[kTiles][kChannelTiles] = {};
    float z[kTiles][kSums] = {}, most[kTiles], sum[kTiles] = {};
#pragma unroll
    for (int t = 0; t < kTiles; ++t) most[t] = -INFINITY;

    // ---- a tile goes from its pages to LDS one tile ahead, its page numbers are looked up two tiles ahead ----
    uint32_t bad_ahead = 0;                         // 16 keys in a page that is none
    int32_t page_ahead = -1;                        // of 16 keys each: lane l has the tile's part l % 4
    uint32_t slot_ahead = 0;
    const uint32_t page_blocks = (uint32_t)c.page_size / 16;
    const int64_t value_codes = (int64_t)c.page_size * (D / 2), value_params = (int64_t)c.page_size * (D / 8), params_after = (int64_t)c.page_size * D;
    const auto look_ahead = [&](int32_t k0) __attribute__((always_inline)) {
        const uint32_t block = (uint32_t)k0 / 16 + lane % 4, at = block / page_blocks;
        slot_ahead = (block - at * page_blocks) * 16;
        page_ahead = -1;
        if (at < (uint32_t)c.table_width) page_ahead = c.table[(int64_t)b * c.table_width + at];
    };
    const auto fetch = [&](Tile &to) __attribute__((always_inline)) {
        // a page behind the table or outside the pool: page 0 instead, and its keys do not count
        const bool none = page_ahead < 0 || page_ahead >= c.pages;
        bad_ahead = (uint32_t)__ballot(none) & 15;
        const uint64_t page = (uint64_t)(none ? 0 : page_ahead) * c.kv_heads + rows.kv_head;
        const uint64_t base = (uint64_t)c.pool + page * (uint64_t)c.page_bytes();
        const uint64_t codes = base + slot_ahead * (D / 2), params = base + params_after + slot_ahead * (D / 8);
        const auto of_lane = [&](uint64_t v, int i) __attribute__((always_inline)) {
            return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), i) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, i);
        };
        // 16 keys are D/2 pieces of 16 bytes of codes and D/2 words of scales and offsets: 64 lanes take 16 keys (D = 128) or 32
        constexpr int kEach = 64 / (D / 2), kPieces = D / 32;                // parts of a load, pieces of a token
        const int in = lane % (D / 2), token = in / kPieces, swapped = token * kPieces + (in % kPieces ^ token / 4 % kPieces);
#pragma unroll
        for (int i = 0; i < 4; i += kEach) {
            uint64_t k = of_lane(codes, i), s = of_lane(params, i);
            if constexpr (kEach == 2) {
                const uint64_t k1 = of_lane(codes, i + 1), s1 = of_lane(params, i + 1);
                k = lane < 32 ? k : k1;
                s = lane < 32 ? s : s1;
            }
            pieces_to_lds(k + 16 * in, &to.keys[i * (D / 2)]);
            pieces_to_lds(k + value_codes + 16 * swapped, &to.values[i * (D / 2)]);
            words_to_lds(s + 4 * in, &to.key_params[16 * i]);
            words_to_lds(s + value_params + 4 * in, &to.value_params[16 * i]);
        }
    };
    const ppmm::Unpacker<T> unpack;
    const ppmm::Unpacker<BF16> unpack_values;
    Tile *const tiles = lds.tiles[wave];
    int32_t k0 = (int32_t)begin + 64 * wave;        // lengths are below 2^31
    if (k0 < end) {
        look_ahead(k0);
        fetch(tiles[0]);
        if (k0 < end - 256) look_ahead(k0 + 256);
    }
    for (int turn = 0; k0 < end; k0 = k0 < end - 256 ? k0 + 256 : end, turn ^= 1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // the tile is in LDS; it is this wave's alone
        const Tile &now = tiles[turn];
        const uint32_t wrong = bad_ahead;
        if (k0 < end - 256) {
            fetch(tiles[turn ^ 1]);
            if (k0 < end - 512) look_ahead(k0 + 512);
        }
        const bool whole = k0 <= clear - 64 && !wrong;
        // ---- scores ----
        f32x4 p[kTiles][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u32x4 params = operand<kGroups>(now.key_params[16 * i + col]);
            const Words codes = ((const Words *)now.keys)[(16 * i + col) * 4 + h];
            const f32x4 zero = {0, 0, 0, 0};
            f32x4 s[kSums];
#pragma unroll
            for (int n = 0; n < kSums; ++n) s[n] = BF16::mma(params, one_s[n], zero);
            u32x4 keys[kGroups];
#pragma unroll
            for (int j = 0; j < kGroups; ++j) keys[j] = unpack.template get<kKeyBit>(codes[j]);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                f32x4 score = BF16::mma(params, qsum[t], zero);
                if constexpr (kFew) {
                    f32x4 acc = zero;
#pragma unroll
                    for (int j = 0; j < kGroups; ++j) acc = T::mma(keys[j], qs[t][j], acc);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float v = fmaf(s[0][e], acc[e], score[e]);
                        v += dpp<kRor8>(v);
                        if constexpr (kGroups == 4) v += dpp<kRor4>(v);
                        score[e] = v;
                    }
                } else {
                    f32x4 acc[kGroups];
#pragma unroll
                    for (int j = 0; j < kGroups; ++j) acc[j] = T::mma(keys[j], qs[t][j], zero);
#pragma unroll
                    for (int j = 0; j < kGroups; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) score[e] = fmaf(s[j][e], acc[j][e], score[e]);
                }
                p[t][i] = score * scale;
            }
        }
        if (!whole) {
            asm volatile("");                       // a branch, not 48 selects in every tile
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (16 * i + 4 * h + e >= limit[t] - k0 || (wrong >> i & 1)) p[t][i][e] = -INFINITY;
        }
        // ---- probabilities: the largest score counts from where it was unless it grew by more than 2^8 ----
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            float top = fmaxf(fmaxf(p[t][0][0], p[t][0][1]), fmaxf(p[t][0][2], p[t][0][3]));
#pragma unroll
            for (int i = 1; i < 4; ++i) top = fmaxf(top, fmaxf(fmaxf(p[t][i][0], p[t][i][1]), fmaxf(p[t][i][2], p[t][i][3])));
            top = most_of_quarters(top);
            const bool grew = top > most[t] + 8.0f || most[t] == -INFINITY;
            if (__ballot(grew && top != -INFINITY)) {
                const float now = grew ? fmaxf(top, most[t]) : most[t];
                const float keep = most[t] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(most[t] - now);
                most[t] = now;
                sum[t] *= keep;
#pragma unroll
                for (int n = 0; n < kSums; ++n) z[t][n] *= keep;
#pragma unroll
                for (int n = 0; n < kChannelTiles; ++n) o[t][n] *= keep;
            }
            const float from = most[t] == -INFINITY ? 0.0f : most[t];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[t][i][e] = __builtin_amdgcn_exp2f(p[t][i][e] - from);
                    sum[t] += p[t][i][e];
                }
        }
        // ---- values ----
        Words vp[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            vp[i] = now.value_params[16 * i + col];
        }
        if (!whole) {
            asm volatile("");
            // values that do not count: whatever lies there, scale and offset are zero
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int w = 0; w < kGroups; ++w) vp[i][w] = 16 * i + col >= held - k0 || (wrong >> i & 1) ? 0 : vp[i][w];
        }
        // Groups of values that read as NaN: their offset would spoil other groups and rows that do not attend to them (0 * NaN).  It is
        // taken out, and the sums of the rows that do attend to them become NaN.
        typedef uint16_t v2u16 __attribute__((ext_vector_type(2)));
        v2u16 largest = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int w = kGroups / 2; w < kGroups; ++w)
                largest = __builtin_elementwise_max(largest, __builtin_bit_cast(v2u16, vp[i][w] & 0x7fff7fffu));
        if (__ballot(largest[0] >= 0x7f80 || largest[1] >= 0x7f80)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                u32x4 flags = {0, 0, 0, 0};
#pragma unroll
                for (int w = kGroups / 2; w < kGroups; ++w) {
                    const uint32_t v = vp[i][w], lo = (v & 0x7f80u) == 0x7f80u, hi = (v & 0x7f800000u) == 0x7f800000u;
                    flags[w] = (lo ? 0x3f80u : 0) | (hi ? 0x3f800000u : 0);
                    vp[i][w] = v & ((lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u));
                }
#pragma unroll
                for (int n = 0; n < kSums; ++n) {
                    const f32x4 flag = BF16::mma(flags, one_b[n], f32x4{0, 0, 0, 0});
#pragma unroll
                    for (int t = 0; t < kTiles; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (flag[e] != 0.0f && 16 * i + 4 * h + e < limit[t] - k0) z[t][n] = NAN;
                }
            }
        }
        const int token = 16 * (col / 4) + 4 * h + col % 4;      // whose values this lane hands in
        const uint8_t *from = (const uint8_t *)now.values + token * (D / 2);
        const auto add_values = [&](int n, const u32x4 (&weights)[2][kTiles][2], const f32x4 (&start)[kTiles]) __attribute__((always_inline)) {
            typedef int v2i __attribute__((ext_vector_type(2)));
            const v2i w = __builtin_amdgcn_ds_read_tr4_b64_v2i32((__attribute__((address_space(3))) v2i *)(from + 16 * (n / 2 ^ h % (D / 32)) + 8 * (n % 2)));
            const u32x4 v0 = unpack_values.get<0>((uint32_t)w[0]), v1 = unpack_values.get<0>((uint32_t)w[1]);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                f32x4 acc = start[t];
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    acc = BF16::mma(v0, weights[part][t][0], acc);
                    acc = BF16::mma(v1, weights[part][t][1], acc);
                }
                o[t][n] += acc;
            }
        };
        // p times scale in two parts, and p times (offset + 24 scale)
        const auto weigh = [&](int t, int n, const f32x4 (&sj)[4], const f32x4 (&bj)[4], u32x4 (&weights)[2][kTiles][2]) __attribute__((always_inline)) {
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = p[t][2 * half][e] * sj[2 * half][e], y = p[t][2 * half + 1][e] * sj[2 * half + 1][e];
#pragma unroll
                    for (int part = 0; part < 2; ++part) {
                        const uint32_t w = pack_bf16(x, y);
                        weights[part][t][half][e] = w;
                        x -= as_float(w << 16);
                        y -= as_float(w & 0xffff0000u);
                    }
                    z[t][n] = fmaf(p[t][2 * half][e], bj[2 * half][e], z[t][n]);
                    z[t][n] = fmaf(p[t][2 * half + 1][e], bj[2 * half + 1][e], z[t][n]);
                }
        };
#pragma unroll
        for (int n = 0; n < kSums; ++n) {           // one group, or in every column its own
            f32x4 s[4], off[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[i] = BF16::mma(operand<kGroups>(vp[i]), one_s[n], f32x4{0, 0, 0, 0});
                off[i] = BF16::mma(operand<kGroups>(vp[i]), one_b[n], f32x4{0, 0, 0, 0});
            }
            u32x4 weights[2][kTiles][2];
#pragma unroll
            for (int t = 0; t < kTiles; ++t) weigh(t, n, s, off, weights);
            const u32x4 minus24 = {BF16::kMinus24, BF16::kMinus24, BF16::kMinus24, BF16::kMinus24};
            f32x4 start[kTiles];                    // the small parts first: their roundings are small then
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                start[t] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int part = 1; part >= 0; --part)
#pragma unroll
                    for (int half = 0; half < 2; ++half) start[t] = BF16::mma(minus24, weights[part][t][half], start[t]);
            }
#pragma unroll
            for (int k = 0; k < kChannelTiles / kSums; ++k) add_values(n * (kChannelTiles / kSums) + k, weights, start);
        }
    }

    // ---- the four waves' parts together ----
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        sum[t] = across_quarters(sum[t]);
#pragma unroll
        for (int n = 0; n < kSums; ++n) z[t][n] = across_quarters(z[t][n]);
        if (h == 0) {
            lds.end.stats[0][wave][t][col] = most[t];
            lds.end.stats[1][wave][t][col] = sum[t];
        }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, lds.end.stats[0][w][t][col]);
        const float keep = most[t] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(most[t] - top);
        if (t) __syncthreads();
#pragma unroll
        for (int n = 0; n < kChannelTiles; ++n)
            if (!kFew || mine == n / 2)
#pragma unroll
                for (int e = 0; e < 4; ++e) lds.end.joined[wave][query][16 * n + 4 * h + e] = (o[t][n][e] + z[t][kFew ? 0 : n / 2]) * keep;
        __syncthreads();
        for (int i = threadIdx.x; i < kQueries * D; i += 256) {
            const int k = i / D, ch = i % D;
            float m = -INFINITY, l = 0.0f, v = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) m = fmaxf(m, lds.end.stats[0][w][t][k]);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float mw = lds.end.stats[0][w][t][k];
                l += mw == -INFINITY ? 0.0f : lds.end.stats[1][w][t][k] * __builtin_amdgcn_exp2f(mw - m);
                v += lds.end.joined[w][k][ch];
            }
            const uint32_t r = row0 + t * kQueries + k;
            const int64_t n = rows.token(r);
            if (r >= count || n < 0 || n >= tokens) continue;
            const int head = rows.kv_head * rows.G + (int)(r % rows.G);
            if (splits == 1) out[n * ots + head * ohs + ch] = divided<T>(v, l);
            else {
                float *to = scratch + ((n * heads + head) * splits + split) * (D + 2);
                to[ch] = v;
                if (ch == 0) { to[D] = m; to[D + 1] = l; }
            }
        }
    }
}

// Joins the splits of a row, of which there are at most 64: a work-group a row and head, whose waves share the splits out.  Every lane
// looks at one split's maximum and sum; four splits' results are under way at a time.
template <class T, int D>
__global__ __launch_bounds__(256) void join_kernel(Cache c, int64_t tokens, int32_t heads, uint16_t *out, int64_t ots, int64_t ohs, int32_t max_q, int32_t splits,
                                                   int32_t unit, const float *scratch)
{
    constexpr int E = D / 64;
    __shared__ float part_sums[4][D];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t row = blockIdx.x, n = row / heads;
    const int32_t b = c.sequence_of(n);
    if (b < 0 || n - c.starts[b] >= max_q) return;              // the whole work-group
    const int64_t held = c.lens[b] < c.capacity() ? c.lens[b] : c.capacity(), part = split_size(held, splits, unit);
    const int used = held > part ? (int)((held + part - 1) / part) : 1;
    const float *from = scratch + row * splits * (D + 2);
    const bool live = lane < used;
    const float mine = live ? from[lane * (D + 2) + D] : -INFINITY, mine_sum = live ? from[lane * (D + 2) + D + 1] : 0.0f;
    float m = mine;
#pragma unroll
    for (int step = 32; step; step /= 2) m = fmaxf(m, __shfl_xor(m, step));
    const float keep = mine == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mine - m);
    float l = keep * mine_sum, v[E] = {};
#pragma unroll
    for (int step = 32; step; step /= 2) l += __shfl_xor(l, step);
    for (int s0 = 4 * wave; s0 < used; s0 += 16) {
        float x[4][E], w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = s0 + i < used ? s0 + i : used - 1;
            w[i] = s0 + i < used ? __shfl(keep, s) : 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) x[i][e] = from[s * (D + 2) + lane * E + e];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = fmaf(w[i], x[i][e], v[e]);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) part_sums[wave][lane * E + e] = v[e];
    __syncthreads();
    const int ch = threadIdx.x;
    if (ch < D) {
        const float sum = part_sums[0][ch] + part_sums[1][ch] + part_sums[2][ch] + part_sums[3][ch];
        out[n * ots + row % heads * ohs + ch] = divided<T>(sum, l);
    }
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
    if ((type != PPMM_BF16 && type != PPMM_FP16) || !ppmm_host::read_strides_ok(tokens, kts, khs, cache->kv_heads) ||
        !ppmm_host::read_strides_ok(tokens, vts, vhs, cache->kv_heads)) return PCMM_EINVAL;
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
    if (ppmm_host::check_attention(cache, batch, tokens, PPMM_BF16, heads, max_q, max_len, device) != PCMM_OK) return 0;
    const ppmm_host::Division d = ppmm_host::divide(*cache, *batch, heads, max_q, max_len, tokens);
    return d.splits == 1 ? 0 : (size_t)tokens * heads * d.splits * (cache->head_dim + 2) * sizeof(float);
}

pcmm_status ppkv_attention(const ppkv_cache *cache, const ppkv_batch *batch, int64_t tokens, ppmm_type type, int32_t heads,
                           const void *q_dev, int64_t qts, int64_t qhs, void *out_dev, int64_t ots, int64_t ohs, float scale, int32_t causal,
                           int32_t max_q, int64_t max_len, void *scratch, size_t scratch_bytes, int32_t device, void *stream)
{
    const pcmm_status rc = ppmm_host::check_attention(cache, batch, tokens, type, heads, max_q, max_len, device);
    if (rc != PCMM_OK) return rc;
    const int D = cache->head_dim;
    if (!ppmm_host::read_strides_ok(tokens, qts, qhs, heads) || !ppmm_host::rows_apart(tokens, heads, D, ots, ohs)) return PCMM_EINVAL;
    if (tokens == 0 || max_q == 0) return PCMM_OK;
    if (!q_dev || !out_dev || q_dev == out_dev) return PCMM_EINVAL;
    const ppmm_host::Division d = ppmm_host::divide(*cache, *batch, heads, max_q, max_len, tokens);
    if (d.splits > 1 && (!scratch || ((uintptr_t)scratch & 15) || scratch_bytes < ppkv_attention_scratch_bytes(cache, batch, tokens, heads, max_q, max_len, device)))
        return PCMM_EINVAL;
    const int64_t join_blocks = tokens * heads;
    const int64_t blocks = d.row_sets * d.splits * cache->kv_heads;                               // of one sequence
    if (blocks > 0xffffff / batch->batch || (d.splits > 1 && join_blocks > 0xffffff)) return PCMM_EUNSUPPORTED;      // no launch of 2^32 threads
    pcmm_hip_util::DevGuard dg(device);
    if (!dg.ok) return PCMM_EDEVICE;
    const Cache c = device_cache(cache, batch);
    const float scale2 = scale * 1.44269504f;
    const dim3 grid((unsigned)(blocks * batch->batch));
    const auto launch = [&](auto kernel, auto join) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)stream, c, tokens, heads, (const uint16_t *)q_dev, qts, qhs, (uint16_t *)out_dev, ots, ohs,
                           scale2, causal, max_q, (uint32_t)d.row_sets, (int32_t)d.splits, d.unit, (float *)scratch);
        if (d.splits > 1)
            hipLaunchKernelGGL(join, dim3((unsigned)join_blocks), dim3(256), 0, (hipStream_t)stream, c, tokens, heads, (uint16_t *)out_dev, ots, ohs, max_q,
                               (int32_t)d.splits, d.unit, (const float *)scratch);
    };
    const auto by_shape = [&](auto tag) {
        using T = decltype(tag);
        if (D == 128) {
            if (d.few && d.tiles == 1) launch(attention_kernel<T, 128, 1, true>, join_kernel<T, 128>);
            else if (d.few) launch(attention_kernel<T, 128, 2, true>, join_kernel<T, 128>);
            else launch(attention_kernel<T, 128, 1, false>, join_kernel<T, 128>);
        } else {
            if (d.few) launch(attention_kernel<T, 64, 1, true>, join_kernel<T, 64>);
            else launch(attention_kernel<T, 64, 1, false>, join_kernel<T, 64>);
        }
    };
    if (type == PPMM_BF16) by_shape(BF16());
    else by_shape(FP16());
    return hipGetLastError() == hipSuccess ? PCMM_OK : PCMM_EDEVICE;
}

}  // extern "C"
