// Strides of the clear track's arrays at their limits: what is accepted has byte offsets below 2^63 and rows that are apart, and no
// check overflows (built with the sanitizers by the tests).
#include <cstdio>
#include <cstdlib>

#include "ppmm_host.hpp"

using namespace ppmm_host;

#define CHECK(x) do { if (!(x)) { std::printf("failed: %s (line %d)\n", #x, __LINE__); std::exit(1); } } while (0)

int main()
{
    const int64_t one = 1;
    CHECK(!rows_apart(2, one << 26, 128, one << 58, one << 40));       // the last head alone lies 2^67 bytes away
    CHECK(rows_apart(2, one << 26, 128, one << 58, one << 32));
    CHECK(!read_strides_ok(2, one << 20, one << 40, one << 26) && read_strides_ok(2, one << 20, one << 33, one << 26));
    const int64_t strides[] = {0, 1, 127, 128, 4096, one << 20, one << 26, one << 33, (one << 33) + 1, one << 34, one << 40, (one << 40) + 1, one << 58, one << 59, INT64_MAX};
    for (int64_t tokens = 1; tokens <= 0x7fffffff; tokens = tokens * 8 - 1)
        for (int64_t heads = 1; heads <= one << 26; heads *= 4)
            for (int64_t ts : strides)
                for (int64_t hs : strides) {
                    const __int128 farthest = ((__int128)(tokens - 1) * ts + (__int128)(heads - 1) * hs + 128) * 2;
                    if (read_strides_ok(tokens, ts, hs, heads)) CHECK(farthest < (__int128)1 << 63);
                    if (!rows_apart(tokens, heads, 128, ts, hs)) continue;
                    CHECK(farthest < (__int128)1 << 63);
                    const bool outer = tokens == 1 || (__int128)ts >= (__int128)(heads - 1) * hs + 128, inner = heads == 1 || (__int128)hs >= (__int128)(tokens - 1) * ts + 128;
                    CHECK(outer || inner);
                }
    std::printf("all checks held\n");
    return 0;
}
