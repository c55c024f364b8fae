// Attention of each sequence's newest tokens over the 8-bit cache.
#pragma once
#include "decode.hpp"
#include "kv8.hpp"

namespace {

// ---------------------------------------------------------------------------------------------
// The rows of a KV head, its query heads' n_q newest tokens (at most 32), are the columns of the score tile, 16 to a tile (RT tiles):
//   S^T [64 keys, rows] = K Q^T            v_mfma_f32_16x16x32_bf16, keys 16 at a time
//   O^T [D, rows] += V^T P^T               the same, features 16 at a time
// K and V go from memory to registers as codes and are converted there (v_cvt_scalef32_pk_bf16_fp8, the block's power of two inside it: exact).
// In the accumulators lane (row, g) of a score tile holds keys 16 t + 4 g + r, r = 0..3, of the four key groups t: as the B operand of P V that is
// what lane group g needs, if the A operand has the same keys in the same order, which is how the cache lays out V.  So neither K, V nor P
// passes through LDS; only the waves' results meet there.  A wave requests a tile's keys when those of the one before are converted and its
// values likewise, so that 8 to 16 KiB (D = 128) are on their way to each wave all the time.
// Token t of the n_q sees keys < len - n_q + 1 + t.  What lies behind a sequence's end is neither a key (its scores are -inf) nor a value (its
// codes are cleared: 0 * NaN).  A NaN in the value of a key that only some of the tokens see would reach the others through weights of zero: it is
// cleared, too, and the sums of those who see it are set.
// The product with V takes weights in bf16.  Up to eight rows leave half of a tile's columns free (HALVES): column c + 8 has the same row as c, and of each weight
// c takes the upper 16 bits, c + 8 what they leave; their sums are added where the waves meet.  So a weight is held to 2^-14 for 34 more vector instructions a
// tile of 250 (us: 2048 keys of 32 heads over 8 6.35 / 6.5, 4 x 32768 48.1 / 48.3, 128 heads of 100 to 2048 keys, d = 64, 9.35 / 9.55).  With more
// rows the columns are taken, and a weight is rounded to bf16, 2^-8 of it at most, as in the bf16 decode: a second half would need a
// tile of its own (16 rows 14.9 us, as 32 columns 16.2), and where the rows come in groups a half more products.  The sum that divides has the unrounded weights in fp32.
// More than 32 rows (GROUPED: a prompt in pieces) are cut into groups of as many tokens as give 32, each with a workgroup of its own for each range; its last
// token's keys take the place of the sequence's.  The KV heads come first in the grid, so that eights of them have an XCD each, in whose L2 their groups find the
// tiles (groups first: 64 of 16384 tokens of 32 heads over 8 47 us, 33 now; 8 x 64 of 4096 81, 49), and the loads are not non-temporal.  Their vector
// instructions are what bounds them, since every wave converts its tiles for 32 rows only: D = 128, the last 1024 of 16384 tokens 288 us (924 TFLOP/s), the vector unit
// busy 75 % of the time and the matrix unit 44 %, two fifths of that together; 256 of them 89 us, 70 and 39 %; all of 2 x 16384 4.74 ms (928 TFLOP/s).
// Partial sums of ranges and their merge: decode.hpp, a row for a head.
struct Kv8Decode {
    DecodeParams d;  // Hq, g: rows for heads (query heads times new tokens); K, V not used
    const uint8_t* K8;
    const uint8_t* V8;
    const uint8_t* KS;
    const uint8_t* VS;
    int T, n_q;
    int g, tokens, groups;  // GROUPED: query heads per KV head; tokens of a workgroup (their rows at most 32); groups of so many
};

// eight codes -> bf16 values
__device__ __forceinline__ bf16x8 kv8_bf16x8(uint32_t w0, uint32_t w1, float scale) {
    using std::true_type, std::false_type;
    return __builtin_bit_cast(bf16x8, u32x4{kv8_bf16x2(w0, scale, false_type{}), kv8_bf16x2(w0, scale, true_type{}),
                                            kv8_bf16x2(w1, scale, false_type{}), kv8_bf16x2(w1, scale, true_type{})});
}
__device__ __forceinline__ float kg_max(float x) {  // over the four lanes of a row
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return xhalf_max(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
}
__device__ __forceinline__ float kg_sum(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return xhalf_sum(__uint_as_float(a[0]) + __uint_as_float(a[1]));
}
// A block's codes: bytes 1024 u + off of it, u = 0..NI - 1; with `bytes` = 0 zeros, and no access.
template <int NI, bool NT>
__device__ __forceinline__ void kv8_request(const uint8_t* base, int bytes, uint32_t off, u32x4* r) {
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
#pragma unroll
    for (int u = 0; u < NI; ++u) r[u] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, off, u * 1024, NT ? 2 : 0));
}

template <int D, int RT, int W, int LENS, bool GROUPED = false, bool HALVES = false>
__global__ __launch_bounds__(64 * W, RT == 1 ? 3 : 2) void kv8_decode_kernel(const Kv8Decode P) {
    const DecodeParams& p = P.d;
    constexpr int S = D / 64, DT = D / 16, NI = D / 16, BYTES = BN * D;
    constexpr int OROW = D + 4, WS = 16 * RT * OROW + 32 * RT;  // floats of a row, of a wave's part of the exchange
    __shared__ __attribute__((aligned(16))) float ex[W * WS];
    const int lane = threadIdx.x & 63, ql = lane & 15, kg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hkv = GROUPED ? blockIdx.x : LENS == LENS_FIXED ? blockIdx.y : blockIdx.z;
    int b = GROUPED || LENS == LENS_FIXED ? blockIdx.z : blockIdx.y, r = GROUPED ? blockIdx.y / P.groups : blockIdx.x, nb = p.n_splits;
    const int tok0 = GROUPED ? (blockIdx.y - r * P.groups) * P.tokens : 0;  // the first of its tokens
    const int ntok = GROUPED ? min(P.tokens, P.n_q - tok0) : P.n_q, rows = GROUPED ? P.g * ntok : p.g;
    // of a column's row among the entry's
    auto row_of = [&](int col) { return GROUPED ? (hkv * P.g + col / ntok) * P.n_q + tok0 + col % ntok : hkv * rows + col; };
    const int w = b * p.n_splits + r;  // range of the batch's list
    if (LENS == LENS_DEALT) {
        const Ranges rg = varlen_find(p, lane, w, 0);
        if (rg.b < 0) return;  // (the same in all waves of the workgroup)
        b = rg.b; r = w - rg.first; nb = rg.nb;
        if (r == 0 && hkv == 0 && tok0 == 0 && threadIdx.x == 0) {  // (every entry has a range)
            p.dealt[2 * b] = rg.first;
            p.dealt[2 * b + 1] = nb;
        }
    }
    const size_t slot = (size_t)w * p.Hq;
    const int all = LENS == LENS_ONE ? p.n_keys : __builtin_amdgcn_readfirstlane(min(max(p.seq_lens[b], 0), p.n_cap));
    const int len = GROUPED ? max(all - P.n_q + tok0 + ntok, 0) : all;  // keys that the last of its tokens sees
    const int Tc = (len + BN - 1) / BN, per = (Tc + nb - 1) / nb;
    const int r0 = r * per, r1 = min(Tc, r0 + per);
    const size_t bh = (size_t)b * p.Hkv + hkv;
    const uint8_t* const K8 = P.K8 + bh * P.T * BYTES;
    const uint8_t* const V8 = P.V8 + bh * P.T * BYTES;
    const uint8_t* const KS = P.KS + bh * P.T;
    const uint8_t* const VS = P.VS + bh * P.T;
    const uint32_t off = ql * 64 + kg * 16;
    bf16x8 qf[RT][2 * S];
    int sees[RT];  // keys that the lane's rows see
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = min(HALVES ? ql & 7 : 16 * rt + ql, rows - 1);
        const uint16_t* const q = p.Q + ((size_t)b * p.Hq + row_of(row)) * D;
#pragma unroll
        for (int s = 0; s < 2 * S; ++s) qf[rt][s] = *reinterpret_cast<const bf16x8*>(q + 64 * (s >> 1) + 16 * kg + 8 * (s & 1));
        sees[rt] = len - ntok + 1 + row % ntok;
    }
    const int all_see = len - ntok + 1;  // keys below are seen by every row
    f32x4 ot[RT][DT];
    float m2[RT], lsum[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m2[rt] = -INFINITY;
        lsum[rt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) ot[rt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    static_assert(!HALVES || RT == 1, "two columns of one tile for each row");
    const uint32_t upper = ql >= 8 ? 0xffff0000u : 0u;  // HALVES: what a column leaves out of a weight
    u32x4 rk[NI], rv[NI];
    int sk = 0, sv = 0;
    auto want = [&](int t) { return t < r1 ? BYTES : 0; };
    auto request_k = [&](int t) __attribute__((always_inline)) {
        sk = KS[min(t, r1 - 1)];
        kv8_request<NI, !GROUPED>(K8 + (size_t)t * BYTES, want(t), off, rk);
    };
    auto request_v = [&](int t) __attribute__((always_inline)) {
        sv = VS[min(t, r1 - 1)];
        kv8_request<NI, !GROUPED>(V8 + (size_t)t * BYTES, want(t), off, rv);
    };
    // tile t; EDGE: some row does not see all of it (there are two such tiles at most, so a wave has one at most, as its last)
    static_assert(W >= 2, "the two tiles that some rows see in part are the last of two waves");
    auto body = [&](int t, auto edge_c) __attribute__((always_inline)) {
        constexpr bool EDGE = decltype(edge_c)::value;
        f32x4 st[RT][4];
        const float ks = ldexpf(1.f, sk - 127);
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) st[rt][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const u32x4 x = rk[4 * s + kt];
                const bf16x8 k0 = kv8_bf16x8(x[0], x[1], ks), k1 = kv8_bf16x8(x[2], x[3], ks);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    st[rt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf[rt][2 * s], st[rt][kt], 0, 0, 0);
                    st[rt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf[rt][2 * s + 1], st[rt][kt], 0, 0, 0);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);  // (requests go out where they are written)
        if (!EDGE) request_k(t + W);
        __builtin_amdgcn_sched_barrier(0);
        const int key0 = t * BN;
        if (EDGE) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) st[rt][kt][e] = key0 + 16 * kt + 4 * kg + e < sees[rt] ? st[rt][kt][e] : -INFINITY;
        }
        bf16x8 pf[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float mx = -INFINITY;
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                for (int e = 0; e < 4; ++e) mx = fmaxf(mx, st[rt][kt][e]);
            const float m_new = fmaxf(m2[rt], kg_max(mx) * p.c);
            const float msub = finite_max(m_new);
            if (__builtin_amdgcn_ballot_w64(m_new != m2[rt]) != 0) {
                const float alpha = __builtin_amdgcn_exp2f(m2[rt] - msub);
                lsum[rt] *= alpha;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) ot[rt][dt] *= alpha;
                m2[rt] = m_new;
            }
            uint32_t pk[8];
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
                float e4[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    e4[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[rt][kt][e], p.c, -msub));
                    lsum[rt] += e4[e];
                }
                if (HALVES) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) e4[e] -= __uint_as_float(__float_as_uint(e4[e]) & upper);
                    pk[2 * kt] = kv8_pair<true>(__float_as_uint(e4[0]), __float_as_uint(e4[1]));
                    pk[2 * kt + 1] = kv8_pair<true>(__float_as_uint(e4[2]), __float_as_uint(e4[3]));
                } else {
                    pk[2 * kt] = pack_bf16(e4[0], e4[1]);
                    pk[2 * kt + 1] = pack_bf16(e4[2], e4[3]);
                }
            }
            pf[rt][0] = __builtin_bit_cast(bf16x8, u32x4{pk[0], pk[1], pk[2], pk[3]});
            pf[rt][1] = __builtin_bit_cast(bf16x8, u32x4{pk[4], pk[5], pk[6], pk[7]});
        }
        // from 2^120 on the largest codes would be infinities in bf16, and a NaN where the weight is 0 (a draft that the row does not see): the weights take
        // 2^16 of the scale, which is exact.  (In the exponentials, without a branch, it costs 32 rows at d = 64 4 %, 11.6 / 12.1 us; so nothing.)
        const int ve = __builtin_amdgcn_readfirstlane(sv) - 127;
        const bool top = ve > 119;
        const float vs = ldexpf(1.f, top ? ve - 16 : ve);
        if (__builtin_expect(top, 0)) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    u32x4 w = __builtin_bit_cast(u32x4, pf[rt][i]);
#pragma unroll
                    for (int q = 0; q < 4; ++q) w[q] = pack_bf16(__uint_as_float(w[q] << 16) * 65536.f, __uint_as_float(w[q] & 0xffff0000u) * 65536.f);
                    pf[rt][i] = __builtin_bit_cast(bf16x8, w);
                }
        }
        // the keys of the lane's bytes below `end`: dword kt holds keys 16 kt + 4 kg + (0..3)
        auto seen_bytes = [&](int kt, int end) {
            const int left = end - (key0 + 16 * kt + 4 * kg);
            return left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << 8 * left) - 1;
        };
        auto nans = [](uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; };  // the top bits of the bytes that are NaN
        if (EDGE) {
            uint32_t in[4], some[4], nan = 0;  // bytes of keys before the end; of keys that some rows see and others not
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
                in[kt] = seen_bytes(kt, len);
                some[kt] = in[kt] & ~seen_bytes(kt, all_see);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    rv[dt][kt] &= in[kt];
                    nan |= nans(rv[dt][kt]) & some[kt];
                }
            }
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(nan != 0) != 0, 0)) {
                // the NaNs of those keys leave the tile; their sums are set to NaN in the rows that see one, which a product of ones counts
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    uint32_t one[4];
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt) {
                        const uint32_t n = (nans(rv[dt][kt]) & some[kt]) >> 7;
                        one[kt] = n * 0x38;  // (the code of 1)
                        rv[dt][kt] &= ~(n * 0xff);
                    }
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        uint32_t see[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int k = key0 + 16 * (i >> 1) + 4 * kg + 2 * (i & 1);
                            see[i] = (k < sees[rt] ? 0x3f80u : 0u) | (k + 1 < sees[rt] ? 0x3f800000u : 0u);
                        }
                        f32x4 count = {0.f, 0.f, 0.f, 0.f};
                        count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kv8_bf16x8(one[0], one[1], 1.f), __builtin_bit_cast(bf16x8, u32x4{see[0], see[1], see[2], see[3]}), count, 0, 0, 0);
                        count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kv8_bf16x8(one[2], one[3], 1.f), __builtin_bit_cast(bf16x8, u32x4{see[4], see[5], see[6], see[7]}), count, 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 4; ++e) ot[rt][dt][e] = count[e] > 0.f ? __builtin_nanf("") : ot[rt][dt][e];
                    }
                }
            }
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            const bf16x8 v0 = kv8_bf16x8(rv[dt][0], rv[dt][1], vs), v1 = kv8_bf16x8(rv[dt][2], rv[dt][3], vs);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                ot[rt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, pf[rt][0], ot[rt][dt], 0, 0, 0);
                ot[rt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, pf[rt][1], ot[rt][dt], 0, 0, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (!EDGE) request_v(t + W);
        __builtin_amdgcn_sched_barrier(0);
    };
    int t = r0 + wave;
    if (t < r1) {
        request_k(t);
        request_v(t);
        const int whole = min(r1, all_see < 0 ? 0 : all_see / BN);  // tiles below are seen whole by every row
        for (; t < whole; t += W) body(t, std::false_type{});
        if (t < r1) body(t, std::true_type{});
    }
    // the waves' sums meet in LDS
    float* const ox = ex + wave * WS;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const float l = kg_sum(lsum[rt]);
        const int row = 16 * rt + ql;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(ox + row * OROW + 16 * dt + 4 * kg) = ot[rt][dt];
        if (kg == 0) {
            ox[16 * RT * OROW + row] = m2[rt];
            ox[16 * RT * OROW + 16 * RT + row] = l;
        }
    }
    __syncthreads();
    for (int idx = threadIdx.x; idx < rows * (D / 4); idx += 64 * W) {
        const int col = idx / (D / 4), c4 = idx - col * (D / 4);
        float m = -INFINITY;
#pragma unroll
        for (int v = 0; v < W; ++v) m = fmaxf(m, ex[v * WS + 16 * RT * OROW + col]);
        const float msub = finite_max(m);
        float lt = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < W; ++v) {
            const float a = __builtin_amdgcn_exp2f(ex[v * WS + 16 * RT * OROW + col] - msub);
            lt += a * ex[v * WS + 16 * RT * OROW + 16 * RT + col];
            const float* const x = ex + v * WS + col * OROW + 4 * c4;
            if (HALVES) o += a * (*reinterpret_cast<const f32x4*>(x) + *reinterpret_cast<const f32x4*>(x + 8 * OROW));
            else o += a * *reinterpret_cast<const f32x4*>(x);
        }
        if (p.n_splits == 1) {  // the only range: this is the result
            const size_t row = (size_t)b * p.Hq + row_of(col);
            const float inv = lt == 0.f ? 0.f : 1.f / lt;
            *reinterpret_cast<u32x2*>(p.O + row * D + 4 * c4) = u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
            if (p.LSE && c4 == 0) p.LSE[row] = lt == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(lt)) * kLn2;
        } else {
            const size_t row = slot + row_of(col);
            *reinterpret_cast<f32x4*>(p.opart + row * D + 4 * c4) = o;
            if (c4 == 0) {
                p.pm[row] = m;
                p.lpart[row] = lt;
            }
        }
    }
}

}  // namespace
