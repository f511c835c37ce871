#pragma once

#include <stdint.h>

// Division of 0 <= n < 2^31 by a fixed d >= 1 without a divide: with l = ceil(log2 d) and mul = ceil(2^(31 + l) / d) < 2^32,
// mul d exceeds 2^(31 + l) by less than 2^l, so that n mul / 2^(31 + l) is off by less than 1 / d.
struct FastDiv {
    uint32_t mul;
    int shift, d;
};
static inline FastDiv fast_div(int d) {
    int l = 0;
    while ((1u << l) < (uint32_t)d) ++l;
    return {d == 1 ? 0u : (uint32_t)(((1ull << (31 + l)) + (uint32_t)d - 1) / (uint32_t)d), l - 1, d};
}
__device__ __forceinline__ int quotient(int n, const FastDiv& f) { return f.shift < 0 ? n : (int)(__umulhi((uint32_t)n, f.mul) >> f.shift); }
