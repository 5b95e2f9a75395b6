// Which kernel computes a product: reads "M N K halves bytes" from each line (compiled and run by product_plan.py; no device code,
// no GPU) and writes the kernel's index and whether its outputs stay in the caches.
#include <cstdio>
#include "lnmod_product_plan.hpp"

int main() {
    long long M, N, K;
    int halves, bytes;
    while (std::scanf("%lld %lld %lld %d %d", &M, &N, &K, &halves, &bytes) == 5)
        std::printf("%d %d\n", lnmod::pick_product(M, N, K, halves != 0), lnmod::keeps_products(M, N, bytes) ? 1 : 0);
}
