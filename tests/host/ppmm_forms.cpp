// Prints the kernel and form that takes each product: lines of "M K T group gated offsets" in, "kernel waves tokens" out.
#include <cstdio>

#include "ppmm_host.hpp"

int main()
{
    const char *names[] = {"stream", "few", "batch", "many"};
    long long M, K, T;
    int group, gated, offsets;
    while (std::scanf("%lld %lld %lld %d %d %d", &M, &K, &T, &group, &gated, &offsets) == 6) {
        const ppmm_host::Form f = ppmm_host::choose(M, K, T, group, gated != 0, offsets != 0);
        std::printf("%s %d %d\n", names[f.kernel], f.waves, f.tokens);
    }
    return 0;
}
