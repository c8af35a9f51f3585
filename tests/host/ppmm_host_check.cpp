// The clear track's argument checks and sizes at their limits (built with the sanitizers by the tests).
#include <cstdio>
#include <cstdlib>

#include "ppmm_host.hpp"

using namespace ppmm_host;

#define CHECK(x) do { if (!(x)) { std::printf("failed: %s (line %d)\n", #x, __LINE__); std::exit(1); } } while (0)

int main()
{
    const void *a = (const void *)0x1000, *b = (const void *)0x2000;
    bool nothing;
    CHECK(check_product(16, 64, 1, a, 64, b, 16, &nothing) == PCMM_OK && !nothing);
    CHECK(check_product(16, 64, 0, nullptr, 64, nullptr, 16, &nothing) == PCMM_OK && nothing);
    CHECK(check_product(16, 64, -1, a, 64, b, 16, &nothing) == PCMM_EINVAL);
    CHECK(check_product(16, 64, 1, a, 63, b, 16, &nothing) == PCMM_EINVAL);
    CHECK(check_product(16, 64, 9, a, 0, b, 16, &nothing) == PCMM_OK);
    CHECK(check_product(16, 64, 1, a, 64, b, 15, &nothing) == PCMM_EINVAL);
    CHECK(check_product(16, 64, 1, a, 64, a, 16, &nothing) == PCMM_EINVAL);
    CHECK(check_product(16, 64, 1, nullptr, 64, b, 16, &nothing) == PCMM_EINVAL);
    CHECK(check_product(16, 64, kMaxRows + 1, a, 64, b, 16, &nothing) == PCMM_EUNSUPPORTED);
    CHECK(check_product(16, 64, 2, a, INT64_MAX, b, 16, &nothing) == PCMM_EUNSUPPORTED);
    CHECK(check_product(kMaxRows, 64, kMaxRows, a, 64, b, kMaxRows, &nothing) == PCMM_EUNSUPPORTED);
    CHECK(check_product(kMaxRows, 64, 256, a, 64, b, kMaxRows, &nothing) == PCMM_OK);
    CHECK(check_product(kMaxRows, 64, 257, a, 64, b, kMaxRows, &nothing) == PCMM_EUNSUPPORTED);
    CHECK(check_product(16, 64, kMaxRows, a, 64, b, 16, &nothing) == PCMM_OK);

    CHECK(check_weights(kMaxRows, 4096, 32, PPMM_FP16, a, b, 0) == PCMM_OK);
    CHECK(check_weights(kMaxRows, 4097, 32, PPMM_FP16, a, b, 0) == PCMM_EUNSUPPORTED);

    CHECK(pool_bytes(0x7fffffff, 16, 1, 64) == (size_t)0x7fffffff * 16 * 80);
    CHECK(pool_bytes(0x7fffffff, 65536, 1024, 128) == 0);
    CHECK(pool_bytes(((int64_t)1 << 47) / 1280, 16, 1, 64) != 0 || ((int64_t)1 << 47) / 1280 > 0x7fffffff);

    // rows of D elements that must not overlap
    CHECK(rows_apart(3, 2, 64, 128, 64) && rows_apart(3, 2, 64, 64, 192) && rows_apart(1, 2, 64, 0, 64) && rows_apart(3, 1, 64, 64, 0));
    CHECK(!rows_apart(3, 2, 64, 127, 64) && !rows_apart(3, 2, 64, 64, 191) && !rows_apart(3, 2, 64, 0, 64) && !rows_apart(3, 1, 64, 63, 64));
    CHECK(!rows_apart(3, 2, 64, -128, 64) && !rows_apart(0x7fffffff, 2, 64, INT64_MAX, 64) && !rows_apart(2, 1024, 64, 64, INT64_MAX));
    CHECK(rows_apart(0, 2, 64, 128, 64));
    // the last token of every sequence of a [batch][tokens][heads][D] array
    CHECK(rows_apart(64, 8, 128, (int64_t)1 << 30, 128) && read_strides_ok(64, (int64_t)1 << 40, 128));
    // brute force over small strides
    for (int tokens = 1; tokens <= 4; ++tokens)
        for (int heads = 1; heads <= 4; ++heads)
            for (int ts = 0; ts <= 14; ++ts)
                for (int hs = 0; hs <= 14; ++hs) {
                    bool apart = true;
                    const int D = 3;
                    for (int i = 0; i < tokens * heads && apart; ++i)
                        for (int j = 0; j < i && apart; ++j) {
                            const int x = i / heads * ts + i % heads * hs, y = j / heads * ts + j % heads * hs;
                            apart = x - y >= D || y - x >= D;
                        }
                    if (rows_apart(tokens, heads, D, ts, hs)) CHECK(apart);      // what is accepted does not overlap
                }
    // attention's division of the work: every row and key has a place, a join never sees more than 64 splits
    for (int D = 64; D <= 128; D += 64)
        for (int kv = 1; kv <= 8; kv += 7)
            for (int G = 1; G <= 9; ++G)
                for (int batch = 1; batch <= 4096; batch *= 8)
                    for (int max_q = 1; max_q <= 5000; max_q = max_q * 3 + 1)
                        for (int64_t max_len = 0; max_len <= 1 << 22; max_len = max_len * 5 + 77) {
                            const ppkv_cache c{(void *)0x1000, 1000, 64, kv, D};
                            const ppkv_batch bt{(const int32_t *)a, (const int32_t *)a, (const int32_t *)a, batch, 1 << 16};
                            const Division d = divide(c, bt, kv * G, max_q, max_len);
                            const int64_t per = d.few ? d.tiles * (16 / (D / 32)) : 16;
                            CHECK(d.splits >= 1 && d.splits <= 64 && d.unit % 256 == 0 && d.tiles >= 1 && d.tiles <= 2);
                            CHECK(d.row_sets * per >= (int64_t)max_q * G && (d.row_sets - 1) * per < (int64_t)max_q * G);
                        }
    std::printf("all checks held\n");
    return 0;
}
