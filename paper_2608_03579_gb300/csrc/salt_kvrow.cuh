// How a row lies in the 8-bit cache: its exponent byte and its place.
#pragma once

#include "salt_internal.cuh"

namespace salt {

// Exponent byte of a row whose largest magnitude has the float bits `a`: with a = f * 2^E (1 <= f < 2), 448 = 1.75 *
// 2^8 gives the smallest k with a <= 448 * 2^k, E - 8 where f <= 1.75, else E - 7.
__device__ __forceinline__ uint32_t row_exp(uint32_t a)
{
    const int E = (int)(a >> 23);
    if (E == 255) return 255u;
    if (a == 0) return 0u;
    const int e = E - 8 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)max(e, 1);
}
// 2^-k of a row's exponent byte, 0 for a row that stands for NaN: a normal float, so that scaling by it is exact
__device__ __forceinline__ float row_inv(uint32_t e) { return __uint_as_float(e == 255u ? 0u : (254u - max(e, 1u)) << 23); }

// The row's number in the cache (they are below 2^31); first_page is the layer's.
__device__ __forceinline__ uint32_t cache_row(const KvDev &c, uint32_t first_page, int page, int slot, int h)
{
    return ((first_page + page) * c.heads + h) * c.page + (slot & (c.page - 1));
}

}  // namespace salt
