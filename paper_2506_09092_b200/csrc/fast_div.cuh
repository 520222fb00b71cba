#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace cudallm {

// Division of a 32-bit unsigned number by a divisor fixed on the host (1 <= d <
// 2^31): q = (t + ((n - t) >> sh1)) >> sh2 with t = the high half of mul * n
// (the round-up method for invariant divisors).  Exact for every 32-bit n.
struct FastDiv {
    uint32_t mul;
    uint16_t sh1, sh2;
};
__device__ __forceinline__ uint32_t fast_div(uint32_t n, FastDiv d)
{
    const uint32_t t = __umulhi(d.mul, n);
    return (t + ((n - t) >> d.sh1)) >> d.sh2;
}
inline FastDiv make_fast_div(uint32_t d)
{
    int l = 0;
    while ((1ull << l) < d) ++l;                         // l = ceil(log2 d)
    FastDiv f;
    f.mul = static_cast<uint32_t>((((1ull << 32) * ((1ull << l) - d)) / d) + 1);
    f.sh1 = static_cast<uint16_t>(l < 1 ? l : 1);
    f.sh2 = static_cast<uint16_t>(l ? l - 1 : 0);
    return f;
}

}  // namespace cudallm
