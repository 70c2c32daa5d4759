// Division by a number that the host knows.
#ifndef INTFA_DIVISOR_H
#define INTFA_DIVISOR_H

#include <hip/hip_runtime.h>

namespace ifa {

// n / d for n < 2^31 by a multiplication: the quotient's multiplier, 2^(32 + s) / d rounded up, has 33 bits, the 33rd being the + n (T. Granlund, P. L. Montgomery, "Division by Invariant Integers
// using Multiplication", 1994; n < 2^31 spares their sum its second shift)
struct Divisor {
    unsigned d, m, s;
    explicit Divisor(unsigned d_) : d(d_), s(0) {
        while ((1ull << s) < d) ++s;
        m = static_cast<unsigned>(((1ull << 32) * ((1ull << s) - d)) / d + 1);
    }
    __device__ __forceinline__ unsigned of(unsigned n) const { return (__umulhi(n, m) + n) >> s; }
};

}  // namespace ifa

#endif  // INTFA_DIVISOR_H
