// host-only sanitizer run of the sizes whose product may leave 64 bits
#include "extent.h"
#include <cstdio>
int main() {
    using ddp::product_reaches;
    const int64_t limit = int64_t(1) << 28, most = INT64_MAX;
    struct { bool want, got; } t[] = {
        {true, product_reaches(limit, {int64_t(1) << 20, 4096, int64_t(1) << 24, int64_t(1) << 24, 4})},      // 2^82: all limits of a call at once
        {true, product_reaches(limit, {int64_t(1) << 20, 4096, int64_t(1) << 18, int64_t(1) << 13, 2})},      // 2^64: 0 where it wraps
        {true, product_reaches(limit, {1 << 14, 1 << 14})},
        {false, product_reaches(limit, {(1 << 14) - 1, 1 << 14})},
        {false, product_reaches(limit, {most, most, 0})},
        {true, product_reaches(limit, {most, most, 1})},
        {false, product_reaches(limit, {})},
        {true, product_reaches(1, {1})},
        {false, product_reaches(1, {0})},
        {true, product_reaches(most, {most})},
        {false, product_reaches(most, {most - 1, 1})},
        {true, product_reaches(7, {7, 1, 1})},
        {false, product_reaches(7, {2, 3})},
    };
    int n = 0;
    for (const auto& x : t) {
        if (x.want != x.got) {
            std::printf("row %d\n", n);
            return 1;
        }
        ++n;
    }
    std::printf("ok\n");
    return 0;
}
