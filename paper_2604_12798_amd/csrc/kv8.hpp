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

typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
typedef __attribute__((ext_vector_type(2))) short s16x2;
// Codes of four bf16 elements, two to a dword, of a block with scale 2^e: v_cvt_scalef32_pk_fp8_bf16 divides by the scale and rounds to nearest even, as
// computed in 64 bits for every finite bf16 at thirteen exponents from -117 to 120.  NaN gives NaN, and so does an infinity: kv8_infinities has the bits that make
// +-448 of its code.
__device__ __forceinline__ uint32_t kv8_codes4(uint32_t x01, uint32_t x23, float scale) {
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, x01), scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, x23), scale, true);
    return __builtin_bit_cast(uint32_t, w);
}
__device__ __forceinline__ uint32_t kv8_infinities(uint32_t x01, uint32_t x23) {
    auto is = [](uint32_t x) { return (x & 0x7fff) == 0x7f80 ? 1u : 0u; };
    return is(x01) | is(x01 >> 16) << 8 | is(x23) << 16 | is(x23 >> 16) << 24;
}
// Elements 2 j and 2 j + 1 (HI) of two rows, the first in the low half.
template <bool HI>
__device__ __forceinline__ uint32_t kv8_pair(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, HI ? 0x07060302u : 0x05040100u); }
// The bits of the largest magnitude among bf16 elements, NaN and infinities above all others; and among the finite ones.
template <int N>
__device__ __forceinline__ uint32_t kv8_largest(const u32x4 (&r)[N]) {
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, r[i][q] & 0x7fff7fffu));
    return max((uint32_t)m[0], (uint32_t)m[1]);
}
template <int N>
__device__ __forceinline__ uint32_t kv8_largest_finite(const u32x4 (&r)[N]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t lo = r[i][q] & 0x7fff, hi = r[i][q] >> 16 & 0x7fff;
            m = max(m, max(lo < 0x7f80 ? lo : 0u, hi < 0x7f80 ? hi : 0u));
        }
    return m;
}
// codes 0 and 1 (HI: 2 and 3) of four -> bf16 values times a power of two
template <typename HI>
__device__ __forceinline__ uint32_t kv8_bf16x2(uint32_t w, float scale, HI) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI::value));
}
// The same four codes for a larger scale, f times the old one (a power of two): through bf16, which holds the values between exactly.
__device__ __forceinline__ uint32_t kv8_again4(uint32_t w, float f) {
    return kv8_codes4(kv8_bf16x2(w, f, std::false_type{}), kv8_bf16x2(w, f, std::true_type{}), 1.f);
}
// ... f for exponents e_old < e: what is below 2^-40 of its old value has a code of 0 anyway
__device__ __forceinline__ float kv8_smaller(int e_old, int e) { return ldexpf(1.f, max(e_old - e, -40)); }
// smallest e >= kExpMin with a <= 448 * 2^e, a given by its bits in bf16 (448 = 1.75 * 2^8)
__device__ __forceinline__ int kv8_exponent(uint32_t bits) {
    const int e = (int)(bits >> 7) - 127 - 8 + ((bits & 0x7f) > 0x60 ? 1 : 0);
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

// A workgroup of 2 D threads per block that new rows may reach, KV head, keys or values.  Of keys a thread has two runs of 16 features (16 bytes of codes);
// of values eight features of four neighbouring keys, whose codes are a dword of each feature's row, so that nothing has to be transposed.  Where all tokens of
// the block are new, and of many, 16 lanes with values cover 64 bytes of a feature's row; of up to 16 tokens 16 lanes (d = 128) cover all features of four, and
// with keys the waves come one after the other, so that those behind the last have nothing to do (d = 128, us, all lanes spread / this: 1512 blocks with 10 new
// tokens 15.7 / 12.3, 656 with 3 10.0 / 7.3, 624 with 44 9.5 / 11.9).  A thread is alone with its bytes of the cache; those of a dword that it does not write it
// puts back.
template <int D>
__global__ __launch_bounds__(2 * D) void kv8_append_kernel(const Kv8Append p) {
    __shared__ uint32_t wmax[D / 32];
    __shared__ int was;
    const int side = blockIdx.y & 1, h = blockIdx.y >> 1, b = blockIdx.z;
    const int o = min(max(p.old_lens ? p.old_lens[b] : p.old_len, 0), p.n_cap);
    const int end = min(max(p.new_lens ? p.new_lens[b] : p.new_len, 0), p.n_cap), n = end - o > p.n_in ? o + p.n_in : end;
    const int tile = o / BN + blockIdx.x;
    if (o >= n || tile > (n - 1) / BN) return;
    const int key0 = tile * BN;
    const int k0 = max(o - key0, 0), k1 = min(n - key0, BN);  // the block's new rows
    const size_t blk = ((size_t)b * p.Hkv + h) * p.T + tile;
    uint8_t* const C = p.C[side] + blk * (BN * D);
    const uint16_t* const x = p.X[side] + b * p.sb[side] + h * p.sh[side] + (long long)(key0 - o) * p.sn[side];
    // (one thread reads the old exponent and writes the new one, whoever else may be late)
    if (threadIdx.x == 0) was = (int)p.S[side][blk] - 127;
    auto body = [&](auto side_c, auto whole_c) __attribute__((always_inline)) {
        constexpr bool V = decltype(side_c)::value, WHOLE = decltype(whole_c)::value;  // WHOLE: every token of the block is new
        const int base = WHOLE ? 0 : V ? k0 & ~3 : k0;  // the first thread's key
        const int kk = base + threadIdx.x / (D / 16), kf = threadIdx.x % (D / 16) * 16;  // keys: features kf to kf + 15 of keys kk and kk + 32
        const bool few = !WHOLE && k1 - base <= 16;  // (no more than the first wave's at d = 128)
        const int vk = few ? base + threadIdx.x / (D / 8) * 4 : threadIdx.x % 16 * 4, vf = few ? threadIdx.x % (D / 8) * 8 : threadIdx.x / 16 * 8;
        uint32_t* const at4 = reinterpret_cast<uint32_t*>(C + vf * BN);  // values: features vf to vf + 7 of keys vk to vk + 3
        const int place = kv8_place(vk & (BN - 1)) / 4;
        uint32_t w4[8];
        u32x4 r[4];
        uint32_t a = 0;
        bool odd = false;  // the wave has infinities or NaN
        // (the lane of a wave's first key decides whether the wave has any; no load sits behind a branch of its own)
        const bool any = WHOLE || (V && !few) || __builtin_amdgcn_readfirstlane(V ? vk : kk) < k1;
        if (any) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = V ? vk + i : kk + 32 * (i >> 1), f = V ? vf : kf + 8 * (i & 1);
                r[i] = *reinterpret_cast<const u32x4*>(x + (WHOLE ? key : min(max(key, k0), k1 - 1)) * p.sn[V] + f);
            }
            if (V && !WHOLE)
#pragma unroll
                for (int q = 0; q < 8; ++q) w4[q] = at4[q * (BN / 4) + place];
            a = wave_umax(kv8_largest(r));  // (a new row that is read again does not change it)
            odd = a >= 0x7f80;
            if (odd) a = wave_umax(kv8_largest_finite(r));
        }
        if ((threadIdx.x & 63) == 0) wmax[threadIdx.x >> 6] = a;
        __syncthreads();
        a = wmax[0];
#pragma unroll
        for (int w = 1; w < D / 32; ++w) a = max(a, wmax[w]);
        int e = kv8_exponent(a);
        const int e_old = was;
        const bool again = !WHOLE && k0 > 0 && e > e_old;
        if (!WHOLE && k0 > 0) e = max(e, e_old);
        const float scale = ldexpf(1.f, e), f_old = kv8_smaller(e_old, e);
        if (threadIdx.x == 0) p.S[V][blk] = (uint8_t)(e + 127);
        if (any && !V) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int key = kk + 32 * u;
                if (!WHOLE && key >= k1) continue;
                u32x4 w;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t x0 = r[2 * u + (q >> 1)][2 * (q & 1)], x1 = r[2 * u + (q >> 1)][2 * (q & 1) + 1];
                    w[q] = kv8_codes4(x0, x1, scale);
                    if (odd) w[q] &= ~kv8_infinities(x0, x1);
                }
                *reinterpret_cast<u32x4*>(C + kf / 64 * (64 * BN) + key * 64 + kf % 64) = w;
            }
        } else if (any && (WHOLE || (vk < k1 && vk + 4 > k0))) {
            uint32_t put = 0, old = 0;  // bytes of new keys, of those before
            if (!WHOLE)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (vk + i < k0) old |= 0xffu << 8 * i;
                    else if (vk + i < k1) put |= 0xffu << 8 * i;
                }
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int j = q >> 1;
                const uint32_t x01 = q & 1 ? kv8_pair<true>(r[0][j], r[1][j]) : kv8_pair<false>(r[0][j], r[1][j]);
                const uint32_t x23 = q & 1 ? kv8_pair<true>(r[2][j], r[3][j]) : kv8_pair<false>(r[2][j], r[3][j]);
                uint32_t w = kv8_codes4(x01, x23, scale);
                if (odd) w &= ~kv8_infinities(x01, x23);
                if (!WHOLE) {
                    if (again) w4[q] = (w4[q] & ~old) | (kv8_again4(w4[q], f_old) & old);
                    w = (w4[q] & ~put) | (w & put);
                }
                w4[q] = w;
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) at4[q * (BN / 4) + place] = w4[q];
        }
        if (again) {  // the tokens before, but for those in a dword with a new one
            const int end = V ? k0 & ~3 : k0;
            for (int i = threadIdx.x; i < D * BN / 16; i += 2 * D) {
                if (!V) {
                    if ((i >> 2) % BN >= end) continue;
                    u32x4* const at = reinterpret_cast<u32x4*>(C) + i;
                    u32x4 w = *at;
#pragma unroll
                    for (int t = 0; t < 4; ++t) w[t] = kv8_again4(w[t], f_old);
                    *at = w;
                } else {
                    const int f = i / 4, g = i % 4;  // 16 bytes: the keys 16 t + 4 g + (0..3)
                    uint32_t* const at = reinterpret_cast<uint32_t*>(C) + f * (BN / 4) + 4 * g;
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        if (16 * t + 4 * g >= end) continue;
                        at[t] = kv8_again4(at[t], f_old);
                    }
                }
            }
        }
    };
    using std::true_type, std::false_type;
    const bool whole = k0 == 0 && k1 == BN;
    if (side == 0 && whole) body(false_type{}, true_type{});
    else if (side == 0) body(false_type{}, false_type{});
    else if (whole) body(true_type{}, true_type{});
    else body(true_type{}, false_type{});
}

// One new row for each sequence (a decode step): D / 8 lanes hold a row of keys or of values, so a wave has 512 / D rows, of KV heads next to each other, and
// nothing waits for another wave.  A block that is coded again is done by the whole wave, before the rows are written.
// (Against a workgroup for each block, 8 KV heads, d = 128, us: 1 sequence 5.6 / 3.0, 16 5.2 / 4.2, 64 7.6 / 3.8; 128 of 16, d = 64, 12.6 / 4.9.)
template <int D>
__global__ __launch_bounds__(64) void kv8_append_one_kernel(const Kv8Append p, int rows) {
    constexpr int G = D / 8;
    const int lane = threadIdx.x, j = lane % G, f = 8 * j;
    const int at = blockIdx.x * (64 / G) + lane / G, u = min(at, rows - 1), side = u & 1, bh = u >> 1, b = bh / p.Hkv, h = bh - b * p.Hkv;
    const int o = min(max(p.old_lens ? p.old_lens[b] : p.old_len, 0), p.n_cap);
    const bool fresh = at < rows && o < min(p.new_lens ? p.new_lens[b] : p.new_len, p.n_cap);
    const int tile = min(o / BN, p.T - 1), k = o % BN;
    const size_t blk = (size_t)bh * p.T + tile;
    uint8_t* const C = p.C[side] + blk * (BN * D);
    const u32x4 r[1] = {*reinterpret_cast<const u32x4*>(p.X[side] + b * p.sb[side] + h * p.sh[side] + f)};
    const int e_old = (int)p.S[side][blk] - 127;
    uint32_t a = kv8_largest(r);
    const bool odd = __builtin_amdgcn_ballot_w64(a >= 0x7f80) != 0;  // the wave has infinities or NaN
    if (odd) a = kv8_largest_finite(r);
    auto most = [](uint32_t x, auto ctrl) { return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xf, 0xf, false)); };
    using std::integral_constant;
    a = most(a, integral_constant<int, 0xb1>{});   // quad_perm [1, 0, 3, 2], [2, 3, 0, 1], row_half_mirror, row_mirror: over 2, 4, 8, 16 lanes
    a = most(a, integral_constant<int, 0x4e>{});
    a = most(a, integral_constant<int, 0x141>{});
    if (D == 128) a = most(a, integral_constant<int, 0x140>{});
    int e = kv8_exponent(a);
    const bool again = fresh && k > 0 && e > e_old;
    if (k > 0) e = max(e, e_old);
    uint64_t todo = __builtin_amdgcn_ballot_w64(again && j == 0);
    if (todo) {
        do {
            const int l = __builtin_ctzll(todo);
            todo &= todo - 1;
            const int side1 = __builtin_amdgcn_readlane(side, l), k1 = __builtin_amdgcn_readlane(k, l);
            const uint64_t blk1 = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)blk, l) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(blk >> 32), l) << 32;
            const float f_old = kv8_smaller(__builtin_amdgcn_readlane(e_old, l), __builtin_amdgcn_readlane(e, l));
            u32x4* const c = reinterpret_cast<u32x4*>(p.C[side1] + blk1 * (BN * D));
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {  // 16 bytes of a key, or 16 keys of a feature
                const int n = 64 * i + lane;
                if (side1 == 0 && (n >> 2) % BN >= k1) continue;
                u32x4 w = c[n];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int left = side1 == 0 ? 4 : k1 - (16 * t + 4 * (n & 3));  // old keys of the dword
                    const uint32_t put = left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << 8 * left) - 1;
                    w[t] = (w[t] & ~put) | (kv8_again4(w[t], f_old) & put);
                }
                c[n] = w;
            }
        } while (todo);
        __threadfence_block();  // (a row's bytes lie among those that were put back)
    }
    if (!fresh) return;
    const float scale = ldexpf(1.f, e);
    uint32_t w[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        w[q] = kv8_codes4(r[0][2 * q], r[0][2 * q + 1], scale);
        if (odd) w[q] &= ~kv8_infinities(r[0][2 * q], r[0][2 * q + 1]);
    }
    if (side == 0) {
        *reinterpret_cast<u32x2*>(C + f / 64 * (64 * BN) + k * 64 + f % 64) = u32x2{w[0], w[1]};
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q) C[(f + q) * BN + kv8_place(k)] = (uint8_t)(w[q >> 2] >> 8 * (q & 3));
    }
    if (j == 0) p.S[side][blk] = (uint8_t)(e + 127);
}

struct Kv8Read {
    const uint8_t* C[2];
    const uint8_t* S[2];
    uint16_t* Y[2];       // [B, Hkv, n, D]
    const int* seq_lens;  // [B], or null: seq_len for all
    int seq_len, n, n_cap, T, Hkv;
};

// A workgroup per block, KV head, keys or values, with the threads' shares as in kv8_append_kernel; rows past the sequence's end are zeros.
template <int D>
__global__ __launch_bounds__(2 * D) void kv8_read_kernel(const Kv8Read p) {
    const int side = blockIdx.y & 1, h = blockIdx.y >> 1, b = blockIdx.z;
    const int len = min(max(p.seq_lens ? p.seq_lens[b] : p.seq_len, 0), p.n_cap), key0 = blockIdx.x * BN;
    const int live = min(len - key0, BN), rows = min(p.n - key0, BN);  // keys that there are; rows to write
    const size_t blk = ((size_t)b * p.Hkv + h) * p.T + blockIdx.x;
    const uint8_t* const C = p.C[side] + blk * (BN * D);
    const float f = live > 0 ? ldexpf(1.f, (int)p.S[side][blk] - 127) : 0.f;
    uint16_t* const y = p.Y[side] + (((size_t)b * p.Hkv + h) * p.n + key0) * D;
    if (side == 0) {
        const int kk = threadIdx.x / (D / 16), kf = threadIdx.x % (D / 16) * 16;
        u32x4 w[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            w[u] = u32x4{0, 0, 0, 0};
            if (kk + 32 * u < live) w[u] = *reinterpret_cast<const u32x4*>(C + kf / 64 * (64 * BN) + (kk + 32 * u) * 64 + kf % 64);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (kk + 32 * u >= rows) continue;
            u32x4 v[2];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                v[q >> 1][2 * (q & 1)] = kv8_bf16x2(w[u][q], f, std::false_type{});
                v[q >> 1][2 * (q & 1) + 1] = kv8_bf16x2(w[u][q], f, std::true_type{});
            }
            u32x4* const at = reinterpret_cast<u32x4*>(y + (size_t)(kk + 32 * u) * D + kf);
            at[0] = v[0];
            at[1] = v[1];
        }
    } else {
        const int vk = threadIdx.x % 16 * 4, vf = threadIdx.x / 16 * 8;
        uint32_t w[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) w[q] = 0;
        if (vk < live) {
            const uint32_t* const at = reinterpret_cast<const uint32_t*>(C + vf * BN + kv8_place(vk));
#pragma unroll
            for (int q = 0; q < 8; ++q) w[q] = at[q * (BN / 4)];
        }
        uint32_t v[2][8];  // features of keys 0 and 1, 2 and 3
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            v[0][q] = kv8_bf16x2(w[q], f, std::false_type{});
            v[1][q] = kv8_bf16x2(w[q], f, std::true_type{});
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (vk + i >= rows) continue;
            u32x4 o = {0, 0, 0, 0};
            if (vk + i < live)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    o[q] = __builtin_amdgcn_perm(v[i >> 1][2 * q + 1], v[i >> 1][2 * q], i & 1 ? 0x07060302u : 0x05040100u);
            *reinterpret_cast<u32x4*>(y + (size_t)(vk + i) * D + vf) = o;
        }
    }
}

}  // namespace
