// Whether tensors share memory: host-side checks of arguments.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <initializer_list>
#include <utility>

namespace b2sp {

// Rows of `bytes` at p + i * stride + j * stride + ...; dims: (size, stride in bytes) of each index.  Those of one element, or of stride 0, say nothing.
struct Spread {
    uintptr_t at;
    int n = 0;
    long long size[3], stride[3];   // widest stride first
    __int128 extent[4];             // of what dimensions i, i + 1 ... span
    Spread(const void *p, long long bytes, std::initializer_list<std::pair<long long, long long>> dims = {}) : at(reinterpret_cast<uintptr_t>(p))
    {
        if (!p) bytes = 0;
        for (const auto &x : dims) {
            if (x.first < 1) bytes = 0;
            if (x.first < 2 || x.second == 0) continue;
            int i = n++;
            for (; i > 0 && stride[i - 1] < x.second; --i) { size[i] = size[i - 1]; stride[i] = stride[i - 1]; }
            size[i] = x.first;
            stride[i] = x.second;
        }
        extent[n] = bytes;
        for (int i = n - 1; i >= 0; --i) extent[i] = bytes ? extent[i + 1] + (__int128)(size[i] - 1) * stride[i] : 0;
    }
    bool operator==(const Spread &o) const
    {
        return at == o.at && n == o.n && extent[n] == o.extent[n] && std::equal(size, size + n, o.size) && std::equal(stride, stride + n, o.stride);
    }
};

// Whether rows of a (from dimension i on) and of b (from j on), whose first one lies `ahead` behind a's, have a byte in common.  Exact for tensors that lie
// beside or in one another with the same wide strides (heads of one projection, keys beside values, a page's mean behind its rows) and for anything in one
// piece; what would take more than kTries blocks of one to compare counts as shared.
inline bool share(const Spread &a, int i, const Spread &b, int j, __int128 ahead)
{
    constexpr int kTries = 16;
    if (ahead >= a.extent[i] || -ahead >= b.extent[j]) return false;
    if (i == a.n && j == b.n) return true;
    const long long sa = i < a.n ? a.stride[i] : 0, sb = j < b.n ? b.stride[j] : 0, s = std::max(sa, sb);
    const int of_a = sa >= sb, of_b = sb >= sa;   // whose dimension it is
    const __int128 ea = a.extent[i + of_a], eb = b.extent[j + of_b];
    // block k: k strides further in a than in b; those with -eb < ahead - k s < ea can meet
    const auto down = [&](__int128 x) { return x >= 0 ? x / s : -((-x + s - 1) / s); };
    const __int128 lo = std::max<__int128>(of_b ? -(b.size[j] - 1) : 0, down(ahead - ea) + 1);
    const __int128 hi = std::min<__int128>(of_a ? a.size[i] - 1 : 0, -down(-(ahead + eb)) - 1);
    if (hi - lo >= kTries) return true;
    for (__int128 k = lo; k <= hi; ++k)
        if (share(a, i + of_a, b, j + of_b, ahead - k * s)) return true;
    return false;
}
inline bool share(const Spread &a, const Spread &b) { return share(a, 0, b, 0, (__int128)b.at - (__int128)a.at); }

}  // namespace b2sp
