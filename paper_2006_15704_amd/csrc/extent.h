// Sizes whose product may leave 64 bits.  Host only, no HIP.
#pragma once
#include <cstdint>
#include <initializer_list>

namespace ddp {

// Whether the product of numbers from 0 on is `limit` (above 0) or more.
inline bool product_reaches(int64_t limit, std::initializer_list<int64_t> factors) {
    int64_t product = 1;
    for (const int64_t f : factors)
        if (f == 0) return false;
    for (const int64_t f : factors) {
        if (product > (limit - 1) / f) return true;
        product *= f;
    }
    return product >= limit;
}

}  // namespace ddp
