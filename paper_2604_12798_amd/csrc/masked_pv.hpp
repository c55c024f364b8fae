// Values that are not finite, in tiles that some rows do not see whole.
#pragma once
#include "common.hpp"

namespace {

// A weight of zero times an infinity or a NaN among the values is a NaN, also in rows that do not see that key.  So a tile that some rows see in part is looked
// through before its product.  Where it holds such values (rare, and slow), they are cleared in LDS, and added afterwards, key by key, to the rows that see them.

// Looks through pieces [u0, u0 + NU) (1 KiB of whole rows each) of a tile of values, clears what is not finite, and returns the keys that have any.
template <int D, int NU>
__device__ __forceinline__ uint64_t clear_not_finite(uint8_t* vt, int u0, int lane) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    using T = Tile<D>;
    constexpr int RPI = 1024 / T::ROWB;
    uint8_t* const at = vt + u0 * 1024 + lane * 16;
    u16x2 most = {0, 0};
#pragma unroll 4
    for (int u = 0; u < NU; ++u) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(at + u * 1024);
#pragma unroll
        for (int e = 0; e < 4; ++e) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, w[e] & 0x7fff7fffu));
    }
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(most[0] >= 0x7f80 || most[1] >= 0x7f80) == 0, 1)) return 0;
    uint64_t keys = 0;
#pragma unroll 1
    for (int u = 0; u < NU; ++u) {
        u32x4 w = *reinterpret_cast<const u32x4*>(at + u * 1024);
        bool bad = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool lo = (w[e] & 0x7f80u) == 0x7f80u, up = (w[e] & 0x7f800000u) == 0x7f800000u;
            w[e] = (lo ? 0u : w[e] & 0xffffu) | (up ? 0u : w[e] & 0xffff0000u);
            bad = bad || lo || up;
        }
        *reinterpret_cast<u32x4*>(at + u * 1024) = w;
        const uint64_t found = __builtin_amdgcn_ballot_w64(bad);
#pragma unroll
        for (int r = 0; r < RPI; ++r) keys |= (found >> (r * T::CH) & ((1ull << T::CH) - 1)) ? 1ull << (RPI * (u0 + u) + r) : 0;
    }
    return keys;
}

// The values of a key that are not finite, from memory, for a row that sees it.
template <int D>
__device__ __forceinline__ void add_not_finite(const uint16_t* value, bool seen, f32x16* ot, int hh) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            __builtin_amdgcn_sched_barrier(0);  // (one load at a time: it must not take registers from the rest)
            const u32x2 w = *reinterpret_cast<const u32x2*>(value + 32 * db + 8 * q + 4 * hh);  // features 32 db + 8 q + 4 hh + (0..3)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
                ot[db][4 * q + e] += seen && !(__builtin_fabsf(v) < INFINITY) ? v : 0.f;
            }
        }
}

}  // namespace
