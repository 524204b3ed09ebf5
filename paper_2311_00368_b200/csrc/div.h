// Division of indices by a number that a launch fixes.
#pragma once

namespace b2sp {

// n / d for 0 <= n < 2^31 by one multiplication (Granlund and Montgomery's round-up method).
struct Div {
    unsigned d, m, s;
    Div() = default;
    explicit Div(unsigned d_) : d(d_), s(0)
    {
        while ((1ull << s) < d) ++s;
        m = (unsigned)(((1ull << 32) * ((1ull << s) - d)) / d + 1);
    }
    __device__ __forceinline__ unsigned operator()(unsigned n) const { return (__umulhi(n, m) + n) >> s; }
};

}  // namespace b2sp
