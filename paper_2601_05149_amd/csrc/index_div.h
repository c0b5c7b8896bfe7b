// Index arithmetic of kernels that find out from their block's number what they work on.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mulo {

// Division of x < 2^32 by a number that the host knows, by multiplication: with 2^(l - 1) < d <= 2^l and
// m = floor(2^32 (2^l - d) / d) + 1, t = the high word of m x, the quotient is (t + (x - t) / 2^min(l, 1)) / 2^max(l - 1, 0)
// (Granlund and Montgomery, "Division by invariant integers using multiplication").  A division by a kernel argument is
// some 30 instructions in a row, and a workgroup has eight in front of its first load.
struct Div {
    uint32_t d, m, s1, s2;
    Div() = default;
    explicit Div(uint32_t by) : d(by) {
        uint32_t l = 0;
        while (((uint64_t)1 << l) < d) ++l;
        m = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << l) - d)) / d + 1);
        s1 = l < 1 ? l : 1;
        s2 = l < 1 ? 0 : l - 1;
    }
    __device__ __forceinline__ int of(int x) const {
        const uint32_t t = __umulhi(m, (uint32_t)x);
        return (int)((t + (((uint32_t)x - t) >> s1)) >> s2);
    }
};

}  // namespace mulo
