// The 8-bit key/value cache: its layout, the kernel that writes rows into it and the one that reads them back.
#pragma once
#include "common.hpp"

namespace {

// ---------------------------------------------------------------------------------------------
// A block is 64 tokens of one KV head, keys and values apart: 64 * D E4M3 codes that stand for code * 2^e, and a byte e + 127.
// The codes lie as the decode kernel's lanes want them, so that every load of a wave is 1 KiB in one piece:
//   keys    [D / 64][64 keys][64 features]
//   values  [D features][64 places], key 16 t + 4 g + r at place 16 g + 4 t + r: the 16 places of g are the keys whose weights lane group g
//           of the score tile holds (see kv8_decode.hpp)
// The exponent is the smallest e >= kExpMin with max |x| <= 448 * 2^e over the block's finite elements.  Powers of two make x 2^-e exact, so
// a code is one rounding of the element, and a block that has to take a larger exponent when a row comes to it is coded again exactly but for
// codes that fall below 2^-6 (E4M3's subnormals).  From kExpMin on every value of the cache is a normal number in bf16.
constexpr int kExpMin = -117;
__device__ __forceinline__ int kv8_place(int key) { return (key & 12) << 2 | (key >> 4) << 2 | (key & 3); }

// E4M3, nearest even, infinities to +-448; a NaN stays one (the conversion itself gives NaN above 448)
__device__ __forceinline__ float kv8_clamp(float y) {
    const float v = fminf(fmaxf(y, -448.f), 448.f);
    return y != y ? y : v;
}
__device__ __forceinline__ uint32_t kv8_codes4(const float* y) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(kv8_clamp(y[0]), kv8_clamp(y[1]), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(kv8_clamp(y[2]), kv8_clamp(y[3]), w, true);
}
// four codes -> their values times f
__device__ __forceinline__ void kv8_values4(uint32_t w, float f, float* y) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    y[0] = lo[0] * f; y[1] = lo[1] * f; y[2] = hi[0] * f; y[3] = hi[1] * f;
}
// smallest e >= kExpMin with a <= 448 * 2^e, a given by its bits (448 = 1.75 * 2^8)
__device__ __forceinline__ int kv8_exponent(uint32_t bits) {
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(e, kExpMin);
}

struct Kv8Append {
    const uint16_t* X[2];  // new rows of keys and values [B, Hkv, n_in, D] with strides (elements)
    long long sb[2], sh[2], sn[2];
    uint8_t* C[2];         // codes
    uint8_t* S[2];         // exponents [B, Hkv, T]
    const int* old_lens;   // [B], or null: old_len, new_len for all
    const int* new_lens;
    int old_len, new_len, n_in, n_cap, T, Hkv;
};

__device__ __forceinline__ uint32_t wave_umax(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xf, 0xf, false));  // row_ror:1, 2, 4, 8
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xf, 0xf, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xf, 0xf, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, false));
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)max(b[0], b[1]));
}

// One workgroup per block that new rows may reach, KV head, keys or values.
template <int D>
__global__ __launch_bounds__(256) void kv8_append_kernel(const Kv8Append p) {
    constexpr int CH = D / 8, NC = BN * CH / 256;  // runs of eight features of a row; of a thread
    __shared__ uint32_t wmax[4];
    const int side = blockIdx.y & 1, h = blockIdx.y >> 1, b = blockIdx.z;
    const int o = min(max(p.old_lens ? p.old_lens[b] : p.old_len, 0), p.n_cap);
    const int n = min(min(p.new_lens ? p.new_lens[b] : p.new_len, p.n_cap), o + p.n_in);
    const int tile = o / BN + blockIdx.x, key0 = tile * BN;
    if (o >= n || key0 >= n) return;
    const int k0 = max(o - key0, 0), k1 = min(n - key0, BN);  // the block's new rows
    const size_t blk = ((size_t)b * p.Hkv + h) * p.T + tile;
    uint8_t* const C = p.C[side] + blk * (BN * D);
    const uint16_t* const x = p.X[side] + b * p.sb[side] + h * p.sh[side] + (long long)(key0 - o) * p.sn[side];
    const int e_old = (int)p.S[side][blk] - 127;
    u32x4 r[NC];
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = i * 256 + threadIdx.x, key = c / CH, f = c % CH * 8;
        r[i] = u32x4{0, 0, 0, 0};
        if (key >= k0 && key < k1) r[i] = *reinterpret_cast<const u32x4*>(x + key * p.sn[side] + f);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t lo = r[i][e] << 16 & 0x7fffffffu, hi = r[i][e] & 0x7fff0000u;
            a = max(a, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
        }
    }
    a = wave_umax(a);
    if ((threadIdx.x & 63) == 0) wmax[threadIdx.x >> 6] = a;
    __syncthreads();
    int e = kv8_exponent(max(max(wmax[0], wmax[1]), max(wmax[2], wmax[3])));
    const bool again = k0 > 0 && e > e_old;
    if (k0 > 0) e = max(e, e_old);
    const float f_new = ldexpf(1.f, -e), f_old = ldexpf(1.f, e_old - e);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = i * 256 + threadIdx.x, key = c / CH, f = c % CH * 8;
        const bool fresh = key >= k0 && key < k1;
        if (!fresh && !(again && key < k0)) continue;
        uint8_t* const at = side == 0 ? C + f / 64 * (64 * BN) + key * 64 + f % 64 : C + f * BN + kv8_place(key);
        float y[8];
        if (fresh) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                y[2 * q] = __uint_as_float(r[i][q] << 16) * f_new;
                y[2 * q + 1] = __uint_as_float(r[i][q] & 0xffff0000u) * f_new;
            }
        } else {
            u32x2 w = {0, 0};
            if (side == 0) w = *reinterpret_cast<const u32x2*>(at);
            else
                for (int q = 0; q < 8; ++q) w[q / 4] |= (uint32_t)at[q * BN] << 8 * (q % 4);
            kv8_values4(w[0], f_old, y);
            kv8_values4(w[1], f_old, y + 4);
        }
        const u32x2 w = {kv8_codes4(y), kv8_codes4(y + 4)};
        if (side == 0) *reinterpret_cast<u32x2*>(at) = w;
        else
            for (int q = 0; q < 8; ++q) at[q * BN] = (uint8_t)(w[q / 4] >> 8 * (q % 4));
    }
    if (threadIdx.x == 0) p.S[side][blk] = (uint8_t)(e + 127);
}

struct Kv8Read {
    const uint8_t* C[2];
    const uint8_t* S[2];
    uint16_t* Y[2];       // [B, Hkv, n, D]
    const int* seq_lens;  // [B], or null: seq_len for all
    int seq_len, n, n_cap, T, Hkv;
};

// One workgroup per block, KV head, keys or values; rows past the sequence's end are zeros.
template <int D>
__global__ __launch_bounds__(256) void kv8_read_kernel(const Kv8Read p) {
    constexpr int CH = D / 8, NC = BN * CH / 256;
    const int side = blockIdx.y & 1, h = blockIdx.y >> 1, b = blockIdx.z;
    const int len = min(max(p.seq_lens ? p.seq_lens[b] : p.seq_len, 0), p.n_cap), key0 = blockIdx.x * BN;
    const size_t blk = ((size_t)b * p.Hkv + h) * p.T + blockIdx.x;
    const uint8_t* const C = p.C[side] + blk * (BN * D);
    const float f = key0 < len ? ldexpf(1.f, (int)p.S[side][blk] - 127) : 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = i * 256 + threadIdx.x, key = c / CH, ft = c % CH * 8;
        if (key0 + key >= p.n) continue;
        u32x4 r = {0, 0, 0, 0};
        if (key0 + key < len) {
            const uint8_t* const at = side == 0 ? C + ft / 64 * (64 * BN) + key * 64 + ft % 64 : C + ft * BN + kv8_place(key);
            u32x2 w = {0, 0};
            if (side == 0) w = *reinterpret_cast<const u32x2*>(at);
            else
                for (int q = 0; q < 8; ++q) w[q / 4] |= (uint32_t)at[q * BN] << 8 * (q % 4);
            float y[8];
            kv8_values4(w[0], f, y);
            kv8_values4(w[1], f, y + 4);
#pragma unroll
            for (int q = 0; q < 4; ++q) r[q] = pack_bf16(y[2 * q], y[2 * q + 1]);
        }
        *reinterpret_cast<u32x4*>(p.Y[side] + (((size_t)b * p.Hkv + h) * p.n + key0 + key) * D + ft) = r;
    }
}

}  // namespace
