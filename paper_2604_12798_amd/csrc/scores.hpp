// Scores that are capped, or get a bias by distance.
#pragma once
#include "common.hpp"

namespace {

// x = cap * tanh(s * scale / cap) - slope * |distance|, in log2 units.  tanh(y) = 1 - 2 / (1 + e^(2 y)): one exponential and one reciprocal, absolute error
// 2^-23 or so, which times the cap is an error of the exponent: caps go up to 1000 (error 2e-4 of a weight).  An infinite score gives +-cap.
struct Scores {
    const float* slopes;  // [Hq] or null
    float cap2;           // cap * log2(e), or 0
    float capk;           // 2 * scale / cap * log2(e): e^(2 y) = 2^(capk * raw score)
};
// What the tile's scores are multiplied with: raw scores are in units of c, changed ones in log2 units already.
__device__ __forceinline__ float score_units(const Scores& s, float c) { return s.cap2 > 0.f || s.slopes ? 1.f : c; }

__device__ __forceinline__ float cap_score(const Scores& s, float x) {
    const float e = __builtin_amdgcn_exp2f(x * s.capk);
    return __builtin_fmaf(-2.f * s.cap2, __builtin_amdgcn_rcpf(1.f + e), s.cap2);
}
__device__ __forceinline__ void cap_scores(const Scores& s, f32x16* st) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) st[t][r] = cap_score(s, st[t][r]);
}
// away: the row's position minus that of the tile's key 4 * hh
__device__ __forceinline__ void bias_scores(const Scores& s, float c, f32x16* st, float slope2, float away) {
    const float u = s.cap2 > 0.f ? 1.f : c;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float dist = __builtin_fabsf(away - (float)(32 * t + 8 * (r >> 2) + (r & 3)));
            st[t][r] = __builtin_fmaf(-slope2, dist, st[t][r] * u);
        }
}

// Softmax step of one tile, exact running max, the rescale branched over in tiles that do not raise it.  HALVES: the lane's weights without `upper` of
// their bits, rounded towards zero (what is left of a weight has 16 bits); else rounded to bf16, which the matrix unit takes and which costs nothing, where columns are not free for a second
// half.  (The sum that divides has the weights whole, so with halves an output is low by up to 2^-16 of itself, a 256th of its own rounding, and rounding to the nearest would take an
// instruction a weight.)
template <bool HALVES, int DB>
__device__ __forceinline__ void softmax_halves(f32x16* st, uint32_t* pk, f32x16* ot, float& m2, float& lsum, float c, uint32_t upper) {
    if (!HALVES) {
        softmax_tile<true, false, DB, true, true>(st, pk, ot, m2, lsum, c, 0, 0, 0, 0.f);
        return;
    }
    const float m_new = fmaxf(m2, xhalf_max(tile_rowmax<false>(st, 0, 0, 0)) * c);
    const float msub = finite_max(m_new);
    if (__builtin_amdgcn_ballot_w64(m_new != m2) != 0) {
        const float alpha = __builtin_amdgcn_exp2f(m2 - msub);
        lsum *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) ot[db] *= alpha;
        m2 = m_new;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
            float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(st[t][r], c, -msub)), e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(st[t][r + 1], c, -msub));
            lsum += e0;
            lsum += e1;
            e0 -= __uint_as_float(__float_as_uint(e0) & upper);
            e1 -= __uint_as_float(__float_as_uint(e1) & upper);
            pk[8 * t + (r >> 1)] = __builtin_amdgcn_perm(__float_as_uint(e1), __float_as_uint(e0), 0x07060302u);
        }
}

}  // namespace
