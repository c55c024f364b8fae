// Norms of queries and keys for each head, the rotation by position, and the head-major layout of the attention calls, in one pass.
#pragma once
#include "common.hpp"

namespace {

// ---------------------------------------------------------------------------------------------
// A row (one head of one token) x of D features becomes
//   z = x * (mean(x^2) + eps)^(-1/2) * w                    (queries and keys; NORM)
//   y_a = z_a cos - z_b sin,  y_b = z_b cos + z_a sin       (pair i < rot / 2 of features: (i, i + rot / 2) or (2 i, 2 i + 1); PAIRS)
// in 32 bits, rounded once.  Values are copied.  D / 16 lanes hold a row, 16 features each: the two halves of eight pairs, so that the
// rotation needs no other lane, and the sum of squares log2(D / 16) steps of DPP.
enum Pairs { PAIRS_NONE = 0, PAIRS_HALF = 1, PAIRS_NEXT = 2 };
struct RopeParams {
    const uint16_t* X[3];    // queries, keys, values [B, N, heads, D] with strides (elements); values may be null
    long long sb[3], sn[3], sh[3];
    uint16_t* Y[3];          // [B, heads, N, D]
    const uint16_t* W[2];    // [D] or null
    const float* cos_sin;    // [n_pos, rot]: rot / 2 cosines, then as many sines
    const int* first_pos;    // [B] or null
    int first, n_pos, rot, N, tokens;  // tokens = B * N
    int Hq, Hkv, heads;      // heads = Hq + Hkv (+ Hkv with values)
    float eps;
};

__device__ __forceinline__ void unpack_bf16(const u32x4& r, float* v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(r[e] << 16);
        v[2 * e + 1] = __uint_as_float(r[e] & 0xffff0000u);
    }
}
__device__ __forceinline__ u32x4 pack_bf16x8(const float* v) {
    return u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
}
// Sum over the D / 16 lanes of a row: neighbours, pairs, quads.
template <int D>
__device__ __forceinline__ float row_sum(float x) {
    auto add = [](float a, auto ctrl) {
        return a + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, a), decltype(ctrl)::value, 0xf, 0xf, false));
    };
    x = add(x, std::integral_constant<int, 0xb1>{});             // quad_perm [1, 0, 3, 2]
    x = add(x, std::integral_constant<int, 0x4e>{});             // quad_perm [2, 3, 0, 1]
    if (D == 128) x = add(x, std::integral_constant<int, 0x141>{});  // row_half_mirror: the other quad of the eight
    return x;
}

template <bool STREAM>
__device__ __forceinline__ u32x4 rope_load(const uint16_t* x) {
    const u32x4* const at = reinterpret_cast<const u32x4*>(x);
    return STREAM ? __builtin_nontemporal_load(at) : *at;
}
template <bool STREAM>
__device__ __forceinline__ void rope_store(uint16_t* y, const u32x4& v) {
    u32x4* const at = reinterpret_cast<u32x4*>(y);
    if (STREAM) __builtin_nontemporal_store(v, at);
    else *at = v;
}

// PER heads of a thread, one after the other, their loads first; STREAM: more data than the memory-side cache holds, which the kernel behind this
// one will not find there anyway, goes past it
template <int D, bool NORM, int PAIRS, int PER, bool STREAM>
__global__ __launch_bounds__(256) void norm_rope_kernel(const RopeParams p) {
    constexpr int L = D / 16, ROWS = 256 / L;  // lanes of a row; tokens of a workgroup
    const int j = threadIdx.x % L;
    const long long tok = (long long)blockIdx.x * ROWS + threadIdx.x / L;
    const bool live = tok < p.tokens;
    const int t = (int)(live ? tok : p.tokens - 1), b = t / p.N, n = t - b * p.N;
    // chunks of eight features: the two halves of eight pairs, or any two; lanes next to each other have chunks next to each other
    const int pairs8 = PAIRS == PAIRS_NONE ? 0 : p.rot / 16;
    int ca = j, cb = j + L;
    if (PAIRS == PAIRS_HALF) {
        ca = j < pairs8 ? j : j + pairs8;
        cb = j < pairs8 ? j + pairs8 : j + L;
    }
    float cs[8], sn[8];  // of the pairs in a chunk of each, or of the eight pairs
    // what is not rotated is not multiplied either: 0 times an infinity beside it would be a NaN
    const bool turn_a = PAIRS == PAIRS_HALF ? j < pairs8 : ca < 2 * pairs8, turn_b = PAIRS == PAIRS_HALF ? turn_a : cb < 2 * pairs8;
    if (PAIRS != PAIRS_NONE) {
        const int pos = (int)min(max((long long)n + (p.first_pos ? p.first_pos[b] : p.first), 0LL), (long long)p.n_pos - 1);
        const float* const c = p.cos_sin + (size_t)pos * p.rot;
#pragma unroll
        for (int e4 = 0; e4 < 2; ++e4) {
            const int at = !(e4 ? turn_b : turn_a) ? 0 : PAIRS == PAIRS_HALF ? 8 * j + 4 * e4 : 4 * (e4 ? cb : ca);
            const f32x4 x = *reinterpret_cast<const f32x4*>(c + at), y = *reinterpret_cast<const f32x4*>(c + p.rot / 2 + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                cs[4 * e4 + e] = x[e];
                sn[4 * e4 + e] = y[e];
            }
        }
    }
    const int h0 = blockIdx.y * PER;
    u32x4 ra[PER], rb[PER];
    auto side = [&](int hh) { return hh < p.Hq ? 0 : hh < p.Hq + p.Hkv ? 1 : 2; };  // (the same in all lanes)
    auto head = [&](int hh, int kind) { return kind == 0 ? hh : kind == 1 ? hh - p.Hq : hh - p.Hq - p.Hkv; };
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int hh = min(h0 + u, p.heads - 1), kind = side(hh);
        const uint16_t* const x = p.X[kind] + b * p.sb[kind] + n * p.sn[kind] + head(hh, kind) * p.sh[kind];
        ra[u] = rope_load<STREAM>(x + 8 * ca);
        rb[u] = rope_load<STREAM>(x + 8 * cb);
    }
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int hh = h0 + u, kind = side(hh);
        if (hh >= p.heads) break;
        uint16_t* const y = p.Y[kind] + (((size_t)b * (kind == 0 ? p.Hq : p.Hkv) + head(hh, kind)) * p.N + n) * D;
        if (kind < 2) {
            float a[8], c[8];
            unpack_bf16(ra[u], a);
            unpack_bf16(rb[u], c);
            if (NORM) {
                float ss = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) ss += a[e] * a[e] + c[e] * c[e];
                const float r = 1.f / sqrtf(row_sum<D>(ss) * (1.f / D) + p.eps);
                const uint16_t* const w = p.W[kind];
                float wa[8], wb[8];
                if (w) {
                    unpack_bf16(*reinterpret_cast<const u32x4*>(w + 8 * ca), wa);
                    unpack_bf16(*reinterpret_cast<const u32x4*>(w + 8 * cb), wb);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    a[e] *= w ? r * wa[e] : r;
                    c[e] *= w ? r * wb[e] : r;
                }
            }
            if (PAIRS == PAIRS_HALF && turn_a) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float za = a[e], zb = c[e];
                    a[e] = za * cs[e] - zb * sn[e];
                    c[e] = zb * cs[e] + za * sn[e];
                }
            }
            auto next = [&](float* z, const float* co, const float* si) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float z0 = z[2 * e], z1 = z[2 * e + 1];
                    z[2 * e] = z0 * co[e] - z1 * si[e];
                    z[2 * e + 1] = z1 * co[e] + z0 * si[e];
                }
            };
            if (PAIRS == PAIRS_NEXT && turn_a) next(a, cs, sn);
            if (PAIRS == PAIRS_NEXT && turn_b) next(c, cs + 4, sn + 4);
            ra[u] = pack_bf16x8(a);
            rb[u] = pack_bf16x8(c);
        }
        if (live) {
            rope_store<STREAM>(y + 8 * ca, ra[u]);
            rope_store<STREAM>(y + 8 * cb, rb[u]);
        }
    }
}

}  // namespace
