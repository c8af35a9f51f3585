// Argument checks and sizes of the clear track (include/ppmm.h).  No HIP here: the host tests compile this file alone.
#ifndef PPMM_HOST_HPP
#define PPMM_HOST_HPP

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/ppmm.h"

namespace ppmm_host {

constexpr int64_t kMaxRows = (int64_t)1 << 24;        // M and T
constexpr int64_t kMaxK = (int64_t)1 << 22;
constexpr int64_t kMaxCodes = (int64_t)1 << 36;
constexpr int64_t kMaxStride = (int64_t)1 << 40;      // elements; keeps every byte offset below 2^63

inline int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// ---- 4-bit weights -------------------------------------------------------------------------------------------------

inline pcmm_status check_weights(int64_t M, int64_t K, int32_t group, int32_t type, const void *codes, const void *scales, int32_t device)
{
    if (M <= 0 || K <= 0 || M > kMaxRows || K > kMaxK || device < 0 || !codes || !scales) return PCMM_EINVAL;
    if (group != 32 && group != 64 && group != 128) return PCMM_EINVAL;
    if (type != PPMM_BF16 && type != PPMM_FP16) return PCMM_EINVAL;
    if (up(M, 16) * up(K, 128) > kMaxCodes) return PCMM_EUNSUPPORTED;
    return PCMM_OK;
}

// *nothing: no tokens, a valid call without work
inline pcmm_status check_product(int64_t M, int64_t K, int64_t T, const void *x, int64_t ldx, const void *y, int64_t ldy, bool *nothing)
{
    *nothing = false;
    if (T < 0 || ldx < 0 || ldy < M) return PCMM_EINVAL;
    if (T == 0) { *nothing = true; return PCMM_OK; }
    if (!x || !y || x == y) return PCMM_EINVAL;
    if (ldx != 0 && ldx < K) return PCMM_EINVAL;
    if (T > kMaxRows || ldx > kMaxStride / T || ldy > kMaxStride / T) return PCMM_EUNSUPPORTED;
    if ((up(M, 16) / 16) * (up(T, 64) / 64) > ((int64_t)1 << 22)) return PCMM_EUNSUPPORTED;      // no launch of 2^32 threads, whatever the kernel
    return PCMM_OK;
}

// Which kernel takes a product, and in which of its forms: one for every size, so that tests see the choice without a GPU.
struct Form {
    enum Kernel { kStream, kFew, kBatch, kMany } kernel;
    int waves;      // kStream: of a work-group; kBatch: waves that take rows
    int tokens;     // kBatch: tokens of a work-group
};

// Two matrices in groups of 32 do not fit the registers of sixteen waves, nor with offsets those of a batch of more than 32 tokens.
inline constexpr bool stream_has(int waves, bool gated, int group) { return waves == 8 || !(gated && group == 32); }
inline constexpr bool batch_has(int tokens, bool gated, int group, bool offsets) { return tokens <= 32 || !(gated && group == 32 && offsets); }

inline Form choose(int64_t M, int64_t K, int64_t T, int group, bool gated, bool offsets)
{
    const int64_t tiles = (M + 15) / 16, mats = gated ? 2 : 1;
    // x in LDS: 28 KiB, at most 30 with K filled up to 128 and the odd pitch, beside at most 32 KiB of the waves' sums; what a larger
    // share would do for 2 to 4 tokens of a K that just misses it (4 tokens of 4096) is not measured
    if (T <= 4 && T * K <= 14336) {
        // with no more than two work-groups a compute unit and a long contraction, twice the waves: 14336 -> 4096 10.0 -> 7.8 us;
        // 4096 -> 4096 3.5 and 3.7 us, 4096 -> 14336 12.3 and 13.9 us.
        if (M <= 8192 && K > 8192 && stream_has(16, gated, group)) return Form{Form::kStream, 16, 0};
        return Form{Form::kStream, 8, 0};
    }
    // Sixteen tokens a work-group while there is no more than one for a compute unit: 64 tokens 4096 -> 1024 6.5 us and 11.9 with x shared
    // by two waves, gated 7.2 and 15.2; with two for each the gain is gone (32 tokens 4096 -> 4096 10.8 and 8.9).  Up to 16 tokens
    // also with two: there is no x to share.  4096 -> 14336 gated 21.9 and, x shared by four, 15.5.
    if (tiles * ((T + 15) / 16) <= 256 || (T <= 16 && tiles * mats <= 512)) return Form{Form::kFew, 8, 16};
    // Otherwise the least of an estimate, in tenths of a microsecond at K = 4096 (all three grow alike with K): x shared by two waves, by
    // four, or large tiles.  Work-groups of 16 to 64 tokens count in rounds of the chip's 256 compute units, large tiles, of which two share
    // a compute unit, in proportion past the first 256.  Measured with 2100 to 14336 rows, 20 to 1000 tokens, all groups, with and without offsets: the
    // choice takes 0.4 % more than the best on average and 23 % at the most (6000 rows, 700 tokens, groups of 128, gated, offsets: 159 us, 129 by four).
    // Two matrices in groups of 32 and more than 48 tokens keep part of their values outside the registers: 27 us a round for 15.
    const bool narrow = group == 32;
    const int longest = T >= 64 ? 64 : (int)(T + 15) / 16 * 16, tokens = batch_has(longest, gated, group, offsets) ? longest : 32;
    const int64_t chunks = (T + tokens - 1) / tokens, large = (tiles * mats + 7) / 8 * ((T + 127) / 128);
    const double round = !gated ? 125 : narrow && tokens > 48 ? 270 : 150;
    const double two = round * (((tiles + 1) / 2 * chunks + 255) / 256), four = 1.55 * round * (((tiles + 3) / 4 * chunks + 255) / 256);
    const double many = (580.0 + std::max<int64_t>(0, large - 256)) * (offsets ? 1.25 : 1.0) * (narrow ? 1.25 : 1.0);
    if (T > 64 && many < two && many < four) return Form{Form::kMany, 4, 128};
    return Form{Form::kBatch, two < four ? 2 : 4, tokens};
}

// ---- cache ---------------------------------------------------------------------------------------------------------

inline bool geometry_ok(int64_t pages, int32_t page_size, int32_t kv_heads, int32_t head_dim)
{
    return pages > 0 && pages <= 0x7fffffff && page_size > 0 && page_size <= 65536 && page_size % 16 == 0 && kv_heads > 0 &&
           kv_heads <= 1024 && (head_dim == 64 || head_dim == 128);
}

// bytes of one page of one head: codes of keys and values, then (scale, offset) of keys and of values
inline int64_t page_bytes(int32_t page_size, int32_t head_dim) { return (int64_t)page_size * (head_dim + head_dim / 4); }

inline size_t pool_bytes(int64_t pages, int32_t page_size, int32_t kv_heads, int32_t head_dim)
{
    if (!geometry_ok(pages, page_size, kv_heads, head_dim)) return 0;
    const int64_t per_page = page_bytes(page_size, head_dim) * kv_heads;
    if (pages >= (((int64_t)1 << 47) + per_page - 1) / per_page) return 0;
    return (size_t)(pages * per_page);
}

inline pcmm_status check_cache(const ppkv_cache *c, const ppkv_batch *b, int64_t tokens, int32_t device)
{
    if (!c || !b || device < 0 || tokens < 0 || tokens > 0x7fffffff) return PCMM_EINVAL;
    if (!c->pool || ((uintptr_t)c->pool & 15) || pool_bytes(c->pages, c->page_size, c->kv_heads, c->head_dim) == 0) return PCMM_EINVAL;
    if (!b->starts || !b->lens || !b->table || b->batch <= 0 || b->batch > 65535 || b->table_width <= 0) return PCMM_EINVAL;
    if ((int64_t)b->table_width * c->page_size > 0x7fffffff) return PCMM_EINVAL;
    return PCMM_OK;
}

// neither all tokens nor all heads reach further than 2^59 elements
inline bool read_strides_ok(int64_t tokens, int64_t token_stride, int64_t head_stride, int64_t heads = 1)
{
    const int64_t most = (int64_t)1 << 59;
    return token_stride >= 0 && head_stride >= 0 && head_stride <= kMaxStride && head_stride <= most / heads && token_stride <= most / (tokens > 0 ? tokens : 1);
}

// no two of tokens x heads rows of D elements overlap
inline bool rows_apart(int64_t tokens, int64_t heads, int64_t D, int64_t token_stride, int64_t head_stride)
{
    if (!read_strides_ok(tokens, token_stride, head_stride, heads)) return false;
    const bool token_inner = heads == 1 || (tokens > 0 && head_stride >= (tokens - 1) * token_stride + D);
    const bool head_inner = tokens <= 1 || token_stride >= (heads - 1) * head_stride + D;
    return (head_inner && (heads == 1 || head_stride >= D)) || (token_inner && (tokens <= 1 || token_stride >= D));
}

inline pcmm_status check_attention(const ppkv_cache *c, const ppkv_batch *b, int64_t tokens, int32_t type, int32_t heads, int32_t max_q,
                                   int64_t max_len, int32_t device)
{
    const pcmm_status rc = check_cache(c, b, tokens, device);
    if (rc != PCMM_OK) return rc;
    if ((type != PPMM_BF16 && type != PPMM_FP16) || max_q < 0 || max_len < 0) return PCMM_EINVAL;
    if (heads <= 0 || heads % c->kv_heads != 0 || heads / c->kv_heads > 65536) return PCMM_EINVAL;
    if ((int64_t)max_q * (heads / c->kv_heads) > 0x7fffffff - 64) return PCMM_EUNSUPPORTED;      // rows of a sequence count in 32 bits
    return PCMM_OK;
}

// How attention is divided among work-groups: `tiles` tiles of columns each, `splits` of the keys.
struct Division {
    bool few;           // a column is a pair of group and query
    int tiles;
    int64_t row_sets, splits;
    int32_t unit;       // a split's keys are a multiple of this
};

constexpr int64_t kMaxScratch = (int64_t)1 << 27;     // bytes

// tokens: rows of the scratch, 0: no more than max_q a sequence
inline Division divide(const ppkv_cache &c, const ppkv_batch &b, int32_t heads, int32_t max_q, int64_t max_len, int64_t tokens = 0)
{
    const int64_t rows = (int64_t)max_q * (heads / c.kv_heads), per_tile = 16 / (c.head_dim / 32), capacity = (int64_t)b.table_width * c.page_size;
    const int64_t longest = max_len > 0 && max_len < capacity ? max_len : capacity;
    Division d;
    const int most = c.head_dim == 128 ? 2 : 1;     // tiles of few queries that a work-group takes
    d.few = rows <= most * per_tile;
    d.tiles = d.few ? (int)((rows + per_tile - 1) / per_tile) : 1;
    const int64_t set = d.few ? d.tiles * per_tile : 16;
    d.row_sets = rows > 0 ? (rows + set - 1) / set : 0;
    // Enough work-groups for the chip, none with less than a round of its four waves (256 keys).  With few queries also no split with
    // more than four rounds, and none with fewer unless the chip needs them: lengths differ, and starting and joining cost a
    // work-group as much as two rounds.  With more queries a split writes as much as it saves: 100, 500 and 2000 new tokens over 32768, 32 heads
    // over 8, took 338, 1455 and 5715 us in splits of four rounds and take 290, 1132 and 4174.
    const int64_t groups = d.row_sets * c.kv_heads * b.batch, rounds = (longest + 255) / 256;
    const int64_t fill = groups > 0 ? (1024 + groups - 1) / groups : 1, even = d.few && groups < 4096 ? (rounds + 3) / 4 : 1;
    d.unit = groups >= 256 ? 1024 : groups >= 128 ? 512 : 256;
    d.splits = fill > even ? fill : even;
    if (d.splits > (longest + d.unit - 1) / d.unit) d.splits = (longest + d.unit - 1) / d.unit;
    if (d.splits < 1) d.splits = 1;
    if (d.splits > 64) d.splits = 64;
    // and no more than kMaxScratch holds: rows without a sequence have their place in it too
    const int64_t all = (tokens > 0 ? tokens : (int64_t)max_q * b.batch) * heads, fit = all > 0 ? kMaxScratch / 4 / (c.head_dim + 2) / all : 64;
    if (d.splits > fit) d.splits = fit > 1 ? fit : 1;
    return d;
}

}  // namespace ppmm_host

#endif  // PPMM_HOST_HPP
