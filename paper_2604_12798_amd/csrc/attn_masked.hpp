// Attention of whole prompts in which each row sees a run of keys of its own, with scores that may be capped or get a bias by distance.
#pragma once
#include "masked_pv.hpp"
#include "scores.hpp"

namespace {

// ---------------------------------------------------------------------------------------------
// Row i sees the keys [lo, hi) of its entry in `ranges` (all without one), and with `causal` none behind itself.  A workgroup has 32 RW rows of a head and
// goes over the steps of 32 KQ keys from the last key that any of its rows sees to the first (the keys next to a row come first, so that a bias leaves the max where
// they put it: from the first to the last the max moved in nearly every step, 4 x 16 heads of 4096, d = 64, 293 us, 221 the other way).  Wave (rw, kq) multiplies the
// 32 keys of group kq with rows 32 rw .. 32 rw + 31, and leaves out the steps at either end that none of its own rows sees.
//
// A score's log2 weight is A + F v.  Without a cap v is what the matrix unit gives and F = c; with one v = 1 / (1 + e^(2 s / cap)), F = -2 cap2 and A = cap2 (see
// Scores).  A bias -slope |i - j| is linear in the key's place in the step on either side of the row: that part goes into v, and the rest is the
// step's A, so that up to 62 slopes are rounded and cancel.  Of the step across the rows, the one with the nearest keys, the distances are taken one by one: they go into v, and
// A is 0.
//
// Iteration s of a wave: Q.K^T of its step s + 1 and P.V of its step s - 1, a product of each in turn, with the softmax of step s dealt out between them, and the
// fragments of the products read a ring ahead.  The max is a reference, the row's max when it last moved plus kMaskedKeep; it moves when a score passes it.
// (So the weight of that max is a power of two, which bf16 holds: a row that sees one key gets its value unchanged.  Rounded up to a whole number, outputs of rows of few keys
// were up to 5 times further off, of long rows 1.4 times where they are 1.3 now, both against outputs rounded once.)
// Weights are rounded to bf16 for the product with V, once more when the max moves between the two: the matrix unit takes 16 bits, and halves as in decode would be twice the products.
// The relative error of whole outputs is 1.16 to 1.38 times that of a form in 32 bits whose outputs are rounded once (0.0019 to 0.0022 / 0.0016 to 0.0017).
// Nothing in an iteration but the masks is conditional: with the three parts behind conditions of their own the compiler held the accumulators twice, and spilled.
//
// RW = 4, KQ = 1: 128 rows.  RW = 2, KQ = 2: 64 rows and half as many steps, for fewer items than the units hold workgroups of the first kind (32 heads over 8, causal, d = 128,
// N = 777 21.9 / 16.5 us, 1024 25.9 / 19.8, 1500 37.3 / 34; 2048, where they are as many, 50.7 / 56).
//
// What bounds it.  d = 128: the matrix unit has 512 cycles of a step and wave, the vector unit 413 (890 with a cap: two exponentials, a reciprocal and five
// other instructions a score), and two waves share a SIMD: a step takes 850 (1140) cycles, at the 1.8 GHz that the power leaves.  Whether the fragments come a ring of 4 or
// of 8 ahead, products in turn or one kind after the other, scheduled here or by the compiler, moves it by 1 %.  32 heads over 8, N = 8192, causal: 502 us, 1095 TFLOP/s (the
// best kernel of Alg. 1 470, the baseline 506, a large matrix product 1256), with a cap 643.  d = 64: the vector unit, three waves a SIMD: 4 x 16 heads of 4096 166 us
// (190 for Alg. 1 on that card), with a bias 182.
// One after the other, tile by tile (K and V of 64 keys in two buffers, ascending, an exact max in each), the first form: 538 us, with a cap 666; d = 64 198, with a bias
// 240; 32 heads, N = 777 21.6, with a cap 25.8.
constexpr float kMaskedKeep = 8.f;

struct MaskedParams {
    Params a;          // Q, K, V, O, LSE, sizes, items, c
    Scores s;
    const int2* ranges;
    int together, heads8;  // KV heads of an XCD whose blocks are taken together; KV heads of an XCD, or 0
};

// The order of the items.  Eights of KV heads have an XCD each, whose L2 then holds their keys, and a list: `together` of its KV heads at a time, late (long) blocks of
// all of them first, so that no long item starts when the others have ended, but no more heads than fill the XCD twice.  (One head after the other, 4 x 16 heads of 4096, d = 64:
// the eight heads of an XCD are 256 items in 96 places; the last head's longest starts in the last third and ends 1.35 times the mean, all together 1.1.)
// Other numbers of KV heads: late blocks of all heads first.
__device__ __forceinline__ Item masked_item(const MaskedParams& P, int id) {
    const Params& p = P.a;
    if (!P.heads8) return item_of(p, id);
    const int y = id >> 3, per = P.together * p.g * p.Tr, part = y / per;
    const int k = min(P.together, P.heads8 - part * P.together);  // KV heads of this part of the list
    const int rem = y - part * per, t = rem / (k * p.g), r = rem - t * k * p.g, j = r / p.g;
    const int kv = (part * P.together + j) * 8 + (id & 7);
    return {kv * p.g + r - j * p.g, kv, p.Tr - 1 - t};
}

template <typename F>
__device__ __forceinline__ int wave_fold(int x, F f) {
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x121, 0xf, 0xf, false));  // row_ror:1, 2, 4, 8
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x122, 0xf, 0xf, false));
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x124, 0xf, 0xf, false));
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, false));
    const auto a = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)x, false, false);
    x = f((int)a[0], (int)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap((uint32_t)x, (uint32_t)x, false, false);
    return __builtin_amdgcn_readfirstlane(f((int)b[0], (int)b[1]));
}

__device__ __forceinline__ void request1_at(const u32x4& rsrc, uint32_t at, uint32_t o0, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(o0), "s"(rsrc), "s"(__builtin_amdgcn_readfirstlane(at))
                 : "memory", "m0");
}

enum class Side { left, across, right };  // of a wave's keys of a step: all at or before its rows, both, all at or behind them

template <int D, int RW, int KQ>
struct Masked {
    static constexpr int KT = 32 * KQ;                 // keys of a step
    static constexpr int SLOT = KT * Tile<D>::ROWB;    // of K or V
    static constexpr int S = KQ == 1 ? 4 : 2;          // slots of each
    static constexpr int LI = SLOT / 4096;             // load instructions of a wave and slot
    static constexpr bool AHEAD = S == 4;              // slots are there a step early, and a step's first fragments are read in the one before
    static constexpr int R = D == 128 ? 8 : 4;         // fragments under way
    static constexpr int LDS_BYTES = 2 * S * SLOT;
    static_assert(RW * KQ == 4, "four waves");
    static_assert(KQ == 1 || 4 * (D * 64 + 256) <= LDS_BYTES, "the partial sums have to fit the slots' memory");
};

template <int D, int RW, int KQ, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void attn_masked_kernel(const MaskedParams P) {
    const Params& p = P.a;
    using T = Tile<D>;
    using F = Masked<D, RW, KQ>;
    constexpr int BM = 32 * RW, KK = D / 16, DB = D / 32, KT = F::KT, S = F::S, LI = F::LI, RPI = 1024 / T::ROWB;
    __shared__ __attribute__((aligned(16))) uint8_t smem[F::LDS_BYTES];  // K[S], V[S]
    __shared__ uint64_t bad[4];  // keys of a slot with values that are not finite, by the wave that found them
    uint8_t* const Vs = smem + S * F::SLOT;
    const int tid = threadIdx.x, lane = tid & 63, ql = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rw = wave % RW, kq = wave / RW;
    const auto [head, kv, i] = masked_item(P, blockIdx.x);
    const int N = p.N, row0 = i * BM, b = kv / p.Hkv;
    const int qrow0 = row0 + 32 * rw, qrow = qrow0 + ql, qrow_c = min(qrow, N - 1);
    // the keys [x, y) that a row sees; one that sees none has [0, 0)
    auto range_of = [&](int r) {
        int2 k = {0, N};
        if (P.ranges) {
            k = P.ranges[(size_t)b * N + r];
            k.x = max(k.x, 0);
            k.y = min(k.y, N);
        }
        if (p.causal) k.y = min(k.y, r + 1);
        return k.x < k.y ? k : int2{0, 0};
    };
    const auto lesser = [](int x, int y) { return min(x, y); };
    const auto larger = [](int x, int y) { return max(x, y); };
    const int far = 0x7fffffff;
    // of the wave: the first and the last key that any row sees, and what all rows see; of the workgroup
    int2 own;
    bf16x8 qf[KK];
    int any_lo, any_hi, all_lo, all_hi, wg_lo, wg_hi, wg_all_lo, wg_all_hi;
    {
        own = range_of(qrow_c);
        const int2 r0 = range_of(min(row0 + lane, N - 1)), r1 = BM == 128 ? range_of(min(row0 + 64 + lane, N - 1)) : r0;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(p.Q + ((size_t)head * N + qrow_c) * D + 16 * kk + 8 * hh);
        any_lo = wave_fold(own.x < own.y ? own.x : far, lesser);
        any_hi = wave_fold(own.y, larger);
        all_lo = wave_fold(own.x, larger);
        all_hi = wave_fold(own.y, lesser);
        wg_lo = wave_fold(min(r0.x < r0.y ? r0.x : far, r1.x < r1.y ? r1.x : far), lesser);
        wg_hi = wave_fold(max(r0.y, r1.y), larger);
        wg_all_lo = wave_fold(max(r0.x, r1.x), larger);
        wg_all_hi = wave_fold(min(r0.y, r1.y), lesser);
    }
    // Blocks of KT keys [b_lo, b_hi): a step each, the last block first.  Steps of the wave: [o_lo, o_hi)
    const int b_lo = wg_lo < wg_hi ? wg_lo / KT : 0, b_hi = wg_lo < wg_hi ? (wg_hi + KT - 1) / KT : 0, steps = b_hi - b_lo;
    const int o_lo = any_hi > 32 * kq ? b_hi - (any_hi - 32 * kq + KT - 1) / KT : steps;
    const int o_hi = any_lo < any_hi ? b_hi - max((any_lo - 32 * kq - 31 + KT - 1) / KT, b_lo) : 0;

    // ---- requests: a wave moves LI adjacent pieces (1 KiB of whole rows) of a slot, by buffer loads whose buffer is the head's keys: rows past the end
    // of the sequence are out of its range and LDS gets zeros, as for steps before the first one and past the last
    const int r_own = RPI * LI * wave + lane / T::CH, cp = lane % T::CH;
    uint32_t offK[LI];
#pragma unroll
    for (int u = 0; u < LI; ++u) offK[u] = (uint32_t)(r_own * T::ROWB + ((cp ^ T::k_mix(r_own + RPI * u)) << 4));
    const uint32_t offV = (uint32_t)(r_own * T::ROWB + ((cp ^ T::v_mix(r_own)) << 4));  // (the same for all pieces)
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr(smem) + wave * LI * 1024);
    const uint32_t bytes = (uint32_t)N * T::ROWB;  // (launched for fewer than 2^31)
    const u32x4 rsrcK = tile_buffer((uint64_t)(uintptr_t)(p.K + (size_t)kv * N * D), bytes), rsrcV = tile_buffer((uint64_t)(uintptr_t)(p.V + (size_t)kv * N * D), bytes);
    auto request = [&](const u32x4& rsrc, int s, int slot, bool is_v, bool there) __attribute__((always_inline)) {
        const uint32_t at = there || (uint32_t)s < (uint32_t)steps ? (uint32_t)(b_hi - 1 - s) * F::SLOT : bytes, to = lds0 + slot * F::SLOT;
        if constexpr (LI == 4) request4_at(rsrc, at, is_v ? offV : offK[0], is_v ? offV : offK[1], is_v ? offV : offK[2], is_v ? offV : offK[3], to);
        else if constexpr (LI == 2) request2_at(rsrc, at, is_v ? offV : offK[0], is_v ? offV : offK[1], to);
        else request1_at(rsrc, at, is_v ? offV : offK[0], to);
    };
    f32x16 ot[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) ot[db] = f32x16{0};
    float m2 = -INFINITY, lsum = 0.f;

    if (steps > 0) {  // (the same in all waves)
        // slot of step s: s mod S.  The first iteration takes the last slot of V for that of the step before it: zeros
#pragma unroll
        for (int e = 0; e < S - 1; ++e) request(rsrcK, e, e, false, false);
#pragma unroll
        for (int e = 0; e < S - 3; ++e) request(rsrcV, e, S + e, true, false);
#pragma unroll
        for (int u = 0; u < LI; ++u) *reinterpret_cast<u32x4*>(Vs + (S - 1) * F::SLOT + (wave * LI + u) * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
        const float slope2 = BIAS ? P.s.slopes[head % p.Hq] * kLog2e : 0.f;
        const float fac = CAP ? -2.f * P.s.cap2 : p.c;
        const float lin = BIAS ? slope2 / fac : 0.f;  // the bias of a key's distance, in units of v
        wait_vm0_and_sync();
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) asm volatile("" : "+v"(qf[kk]));  // (waited for here, not in the steps)

        uint32_t ka[KK], va[DB];
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) ka[kk] = lds_addr(smem) + (T::k_base(ql, hh) ^ (kk << 5)) + 32 * kq * T::ROWB;
#pragma unroll
        for (int db = 0; db < DB; ++db) va[db] = lds_addr(Vs) + (T::v_base(lane, hh) ^ (db << 6)) + 32 * kq * T::ROWB;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) asm volatile("" : "+v"(ka[kk]));  // (sums of a scalar and a vector that the compiler would add up again for each load)
#pragma unroll
        for (int db = 0; db < DB; ++db) asm volatile("" : "+v"(va[db]));
        auto ld_k = [&](uint32_t slot, int kk) __attribute__((always_inline)) { return *(lds_frag)(ka[kk] + slot); };
        auto ld_v = [&](uint32_t slot, int f) __attribute__((always_inline)) {
            const uint32_t a = va[f % DB] + (slot + 16 * (f / DB) * T::ROWB);
            const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(a));
            const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(a + 8 * T::ROWB));
            const u32x2 a0 = __builtin_bit_cast(u32x2, v0), a1 = __builtin_bit_cast(u32x2, v1);
            return __builtin_bit_cast(bf16x8, u32x4{a0[0], a0[1], a1[0], a1[1]});
        };
        auto pf = [&](const uint32_t* pk, int c) __attribute__((always_inline)) {
            return __builtin_bit_cast(bf16x8, u32x4{pk[4 * c], pk[4 * c + 1], pk[4 * c + 2], pk[4 * c + 3]});
        };
        // (all in steps, worked out once) Sides of a bias: the wave's keys of step s all at or before all of its rows; all at or behind all of them.
        // Steps that all rows of the wave see whole, and all rows of the workgroup
        const int l_lo = b_hi - (qrow0 >= 32 * kq + 31 ? (qrow0 - 32 * kq - 31) / KT + 1 : 0), r_hi = b_hi - (max(qrow0 + 31 - 32 * kq, 0) + KT - 1) / KT;
        const int w_lo = b_hi - (all_hi >= 32 * kq + 32 ? (all_hi - 32 * kq - 32) / KT + 1 : 0), w_hi = b_hi - (max(all_lo - 32 * kq, 0) + KT - 1) / KT;
        const int f_lo = b_hi - wg_all_hi / KT, f_hi = b_hi - (wg_all_lo + KT - 1) / KT;
        const uint32_t w_many = max(w_hi - w_lo, 0), f_many = max(f_hi - f_lo, 0);
        auto side_of = [&](int s) { return !BIAS || s >= l_lo ? Side::left : s < r_hi ? Side::right : Side::across; };
        auto whole = [&](int s) { return (uint32_t)(s - w_lo) < w_many; };
        auto first_key = [&](int s) { return (b_hi - 1 - s) * KT + 32 * kq; };  // of the wave

        // A bias's part that is linear in the key's place, as one more product, of the places 0 .. 31 (exact in bf16) with the slope in three pieces of bf16: sixteen
        // multiply-adds of a step less.  It comes behind those of Q.K^T, which would be rounded at its size otherwise.
        bf16x4 places, pieces;
        if (BIAS && !CAP) {
            float rest = lin;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                places[e] = (__bf16)(hh == 0 && e < 3 ? (float)ql : 0.f);
                pieces[e] = (__bf16)(hh == 0 && e < 3 ? rest : 0.f);
                rest -= (float)pieces[e];
            }
        }
        auto slant = [&](const f32x16& st, Side side) __attribute__((always_inline)) -> f32x16 {
            if (!BIAS || CAP) return st;
            u32x2 b = __builtin_bit_cast(u32x2, pieces);
#pragma unroll
            for (int e = 0; e < 2; ++e) b[e] = side == Side::left ? b[e] : side == Side::right ? b[e] ^ 0x80008000u : 0u;
            return __builtin_amdgcn_mfma_f32_32x32x8bf16_1k(__builtin_bit_cast(s16x4, places), __builtin_bit_cast(s16x4, b), st, 0, 0, 0);
        };
        // the softmax of a step, in parts: pairs of scores to v (CAP), the max, pairs of v to weights
        float add = -INFINITY;  // A - the max
        auto offset = [&](int s, Side side) __attribute__((always_inline)) {  // A
            const int away = qrow - first_key(s) - (CAP ? 4 * hh : 0);
            const float base = BIAS ? (side == Side::left ? -slope2 : side == Side::right ? slope2 : 0.f) * (float)away : 0.f;
            return CAP ? P.s.cap2 + base : base;
        };
        auto part_a = [&](f32x16& st, Side side, int q) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 2 * q; e < 2 * q + 2; ++e) {
                st[e] = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(st[e] * P.s.capk));
                if (BIAS) st[e] = __builtin_fmaf(side == Side::left ? lin : side == Side::right ? -lin : 0.f, (float)(8 * (e >> 2) + (e & 3)), st[e]);
            }
        };
        // Products of po that have been started are in ot, those to come take the changed po: the max may move between any two of them.  po is rounded
        // twice then, but at 2^-8 of the row's new max at most.  (Each row by itself: what the others see changes none of its bits.)
        auto part_m = [&](const f32x16& st, uint32_t* po, int s, Side side) __attribute__((always_inline)) {
            float x = st[0];
#pragma unroll
            for (int q = 0; q < 7; ++q) x = CAP ? fminf(fminf(x, st[1 + 2 * q]), st[2 + 2 * q]) : fmaxf(fmaxf(x, st[1 + 2 * q]), st[2 + 2 * q]);
            x = CAP ? fminf(x, st[15]) : fmaxf(x, st[15]);
            const float a = offset(s, side), y = __builtin_fmaf(x, fac, a);  // (with a cap and a bias A differs between the halves)
            const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
            const float top = fmaxf(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(top > m2) != 0, 0)) {
                const float m_new = top > m2 ? top + kMaskedKeep : m2;
                const float alpha = __builtin_amdgcn_exp2f(m2 - finite_max(m_new));
                lsum *= alpha;
#pragma unroll
                for (int db = 0; db < DB; ++db) ot[db] *= alpha;
#pragma unroll
                for (int q = 0; q < 8; ++q) po[q] = pack_bf16(__uint_as_float(po[q] << 16) * alpha, __uint_as_float(po[q] & 0xffff0000u) * alpha);
                m2 = m_new;
                if (!BIAS) add = a - finite_max(m2);
            }
            if (BIAS) add = a - finite_max(m2);
        };
        auto part_b = [&](const f32x16& st, uint32_t* pk, int q) __attribute__((always_inline)) {
            const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(st[2 * q], fac, add)), e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(st[2 * q + 1], fac, add));
            lsum += e0;
            lsum += e1;
            pk[q] = pack_bf16(e0, e1);
            asm volatile("" : "+v"(pk[q]), "+v"(lsum));  // (here, between the products: the compiler sank them behind the next branch)
        };
        constexpr int R = F::R;
        static_assert(!F::AHEAD || 2 * KK % R == 0, "a step ends where the ring of fragments began");
        bf16x8 fr[R];
        // Iteration s: st, pk of step s; sn of step s + 1, po of step s - 1
        auto work = [&](int s, f32x16& st, f32x16& sn, uint32_t* pk, uint32_t* po, uint32_t slot_k, uint32_t slot_v, uint32_t next_k, uint32_t next_v, auto plain_c)
                        __attribute__((always_inline)) {
            constexpr bool A = CAP, PLAIN = decltype(plain_c)::value;
            constexpr int M = 2 * KK, H = A ? M / 2 : 0;  // products; those in front of the masks
            static_assert(KK == 2 * DB, "as many products on either side");
            auto frag = [&](int e, uint32_t sk, uint32_t sv) __attribute__((always_inline)) { return e & 1 ? ld_v(sv, e >> 1) : ld_k(sk, e >> 1); };
            auto product = [&](int e) __attribute__((always_inline)) {
                if (e & 1) {
                    const int f = e >> 1;
                    ot[f % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[e % R], pf(po, f / DB), ot[f % DB], 0, 0, 0);
                } else {
                    sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[e % R], qf[e >> 1], e == 0 ? f32x16{0} : sn, 0, 0, 0);
                    if (e == M - 2) sn = slant(sn, PLAIN ? Side::left : side_of(s + 1));
                }
                if (e + R < M) fr[e % R] = frag(e + R, slot_k, slot_v);
                else if (F::AHEAD) fr[e % R] = frag(e + R - M, next_k, next_v);
                __builtin_amdgcn_sched_barrier(0);
            };
            if (!F::AHEAD) {
#pragma unroll
                for (int e = 0; e < R; ++e) fr[e] = frag(e, slot_k, slot_v);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int e = 0; e < H; ++e) {
#pragma unroll
                for (int u = 8 * e / H; u < 8 * (e + 1) / H; ++u) part_a(st, PLAIN ? Side::left : side_of(s), u);
                product(e);
            }
            const int key0 = first_key(s) + 4 * hh;
            if (BIAS && !PLAIN && side_of(s) == Side::across) {
#pragma unroll
                for (int r = 0; r < 16; ++r) st[r] = __builtin_fmaf(-lin, __builtin_fabsf((float)(qrow - key0 - 8 * (r >> 2) - (r & 3))), st[r]);
            }
            if (!PLAIN && !whole(s)) {
                const uint32_t first = own.x - key0, many = own.y - own.x;
#pragma unroll
                for (int r = 0; r < 16; ++r) st[r] = (uint32_t)(8 * (r >> 2) + (r & 3)) - first < many ? st[r] : CAP ? INFINITY : -INFINITY;
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int e = H; e < M; ++e) {
#pragma unroll
                for (int u = 10 * (e - H) / (M - H); u < 10 * (e - H + 1) / (M - H); ++u) {
                    if (u == 0) part_m(st, po, s, PLAIN ? Side::left : side_of(s));
                    else if (u >= 2) part_b(st, pk, u - 2);
                }
                product(e);
            }
        };
        // What surrounds the work of an iteration; j = s mod S
        uint64_t keys = 0;  // of the step whose values are multiplied: those with values that are not finite
        auto iteration = [&](int s, int j, auto plain_c, auto f) __attribute__((always_inline)) {
            constexpr bool PLAIN = decltype(plain_c)::value;
            const uint32_t slot_v = (j + S - 1) % S * F::SLOT;
            // No row of the workgroup may get what is not finite among the values of a key that it does not see: those of a step that not all rows see whole
            // are cleared before the first of them is read
            const int c = F::AHEAD ? s : s - 1;
            uint64_t found = 0;
            if (!PLAIN && (uint32_t)(c - f_lo) >= f_many && (uint32_t)c < (uint32_t)steps) {
                bad[wave] = clear_not_finite<D, LI>(Vs + (F::AHEAD ? j * F::SLOT : slot_v), wave * LI, lane);
                __syncthreads();
                found = bad[0] | bad[1] | bad[2] | bad[3];
                found = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(found >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)found);
            }
            if (!F::AHEAD) keys = found;
            request(rsrcK, s + S, j % S, false, PLAIN);
            request(rsrcV, s - 2 + S, S + (j + S - 2) % S, true, PLAIN);
            f((j + 1) % S * F::SLOT, slot_v);
            if (!PLAIN && __builtin_expect(keys != 0, 0)) {
                const uint16_t* const Vg = p.V + (size_t)kv * N * D;
                // (the max may have moved behind the product: what is added is not finite, whatever it is multiplied with)
#pragma unroll 1
                for (uint64_t left_over = keys >> (32 * kq) & 0xffffffffull; left_over; left_over &= left_over - 1) {
                    const int k = first_key(s - 1) + __builtin_ctzll(left_over);  // (a key of the sequence: behind its end LDS has zeros)
                    add_not_finite<D>(Vg + (size_t)k * D, k >= own.x && k < own.y, ot, hh);
                }
            }
            if (!PLAIN) keys = found;
            // K of step s + 2 and V of step s are there, AHEAD those of the steps behind them; reads of slots that are written next are through with their products
            __builtin_amdgcn_s_waitcnt(F::AHEAD ? 0x0F70 | 2 * LI : 0x0070);
            __builtin_amdgcn_s_barrier();
        };
        // Iterations [front, o_hi] are the wave's (the slots are constants, so the first one is the first of a round); its scores of step `front` come from the
        // one before.  What is not the wave's among their steps is masked, so its weights are 0, and the values that they meet are finite: cleared, or,
        // in the first iteration of all, the slot of zeros.
        const bool any = o_lo < o_hi;
        const int front = any ? o_lo / S * S : steps + 2;
        int s = -1, j = S - 1;
        auto idle = [&](int end) __attribute__((always_inline)) {
            for (; s < end; ++s) {
                iteration(s, j, std::false_type{}, [](uint32_t, uint32_t) {});
                j = j + 1 == S ? 0 : j + 1;
            }
        };
        idle(min(front - 1, steps + 1));
        if (any) {
            f32x16 sa, sb;
            uint32_t pa[8], pb[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) pa[q] = 0;
            iteration(s, S - 1, std::false_type{}, [&](uint32_t, uint32_t) __attribute__((always_inline)) {
                sa = f32x16{0};
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) sa = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ld_k(0, kk), qf[kk], sa, 0, 0, 0);
                sa = slant(sa, side_of(front));
                __builtin_amdgcn_sched_barrier(0);
                if (F::AHEAD) {  // (of K of step front + 1, V of step front - 1)
#pragma unroll
                    for (int e = 0; e < R; ++e) fr[e] = e & 1 ? ld_v((S - 1) * F::SLOT, e >> 1) : ld_k(F::SLOT, e >> 1);
                }
            });
            ++s;
            auto step = [&](auto j_c, auto plain_c) __attribute__((always_inline)) {
                constexpr int J = decltype(j_c)::value;
                iteration(s, J, plain_c, [&](uint32_t, uint32_t) __attribute__((always_inline)) {
                    work(s, J & 1 ? sb : sa, J & 1 ? sa : sb, J & 1 ? pa : pb, J & 1 ? pb : pa, (J + 1) % S * F::SLOT, (J + S - 1) % S * F::SLOT, (J + 2) % S * F::SLOT, J * F::SLOT, plain_c);
                });
                ++s;
            };
            auto round = [&](auto plain_c) __attribute__((always_inline)) {
                step(std::integral_constant<int, 0>{}, plain_c);
                step(std::integral_constant<int, 1>{}, plain_c);
                if constexpr (S == 4) {
                    step(std::integral_constant<int, 2>{}, plain_c);
                    step(std::integral_constant<int, 3>{}, plain_c);
                }
            };
            // Whole rounds of steps with nothing special, [plain_lo, plain_hi), have a loop without a condition: all rows of the wave see them whole, on the left,
            // those of the workgroup the step whose values are read first (and the one before), and there is a step to request.  (Few rows gain nothing from it.)
            int plain_lo = max(max(w_lo, f_lo + 1), front), plain_hi = min(min(w_hi, f_hi), min(steps - S, o_hi));
            if (BIAS) plain_lo = max(plain_lo, l_lo);
            plain_lo = (plain_lo + S - 1) / S * S;
            if (KQ == 1 && plain_hi - plain_lo >= S) {
                while (s < plain_lo) round(std::false_type{});
                while (s + S <= plain_hi) round(std::true_type{});
            }
            for (;;) {
                auto one = [&](auto j_c) __attribute__((always_inline)) {  // (as a function with a result: a break behind each made the compiler spill)
                    if (s > o_hi) return false;
                    step(j_c, std::false_type{});
                    return true;
                };
                if (!one(std::integral_constant<int, 0>{})) break;
                if (!one(std::integral_constant<int, 1>{})) break;
                if constexpr (S == 4) {
                    if (!one(std::integral_constant<int, 2>{})) break;
                    if (!one(std::integral_constant<int, 3>{})) break;
                }
            }
        }
        j = s % S;
        idle(steps + 1);
        wait_vm0_and_sync();  // (the requests past the last step write zeros)
    }

    // ---- the groups add their sums, each for its share of the features
    float l = xhalf_sum(lsum);
    float m = m2, w_own = 1.f;
    if constexpr (KQ == 2) {
        float* const ex = reinterpret_cast<float*>(smem);                    // [wave][unit of 4 registers][lane][4]
        float* const xml = reinterpret_cast<float*>(smem + 4 * D * 64);      // [wave][max, l][32 rows]
        if (hh == 0) {
            xml[wave * 64 + ql] = m2;
            xml[wave * 64 + 32 + ql] = l;
        }
        // group 0 keeps the first half of the features' blocks of 32, group 1 the second
#pragma unroll
        for (int db = 0; db < DB / 2; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x16& o = kq == 0 ? ot[DB / 2 + db] : ot[db];
                *reinterpret_cast<f32x4*>(ex + ((wave * (DB / 2 * 4) + db * 4 + q) * 64 + lane) * 4) = f32x4{o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]};
            }
        __syncthreads();
        const int other = wave ^ RW;  // (wave = kq * RW + rw)
        const float mo = xml[other * 64 + ql], lo = xml[other * 64 + 32 + ql];
        m = fmaxf(m2, mo);
        const float msub = finite_max(m);
        w_own = __builtin_amdgcn_exp2f(m2 - msub);
        const float w_other = __builtin_amdgcn_exp2f(mo - msub);
        l = w_own * l + w_other * lo;
#pragma unroll
        for (int db = 0; db < DB / 2; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 x = *reinterpret_cast<const f32x4*>(ex + ((other * (DB / 2 * 4) + db * 4 + q) * 64 + lane) * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float mine = kq == 0 ? ot[db][4 * q + e] : ot[DB / 2 + db][4 * q + e];
                    ot[db][4 * q + e] = __builtin_fmaf(w_own, mine, w_other * x[e]);
                }
            }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (qrow < N && p.LSE && kq == 0 && hh == 0) p.LSE[(size_t)head * N + qrow] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
    uint16_t* const Og = p.O + ((size_t)head * N + qrow_c) * D + (KQ == 2 ? kq * (D / 2) : 0);
#pragma unroll
    for (int db = 0; db < DB / KQ; ++db)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            // the lane pair (l, l ^ 32) trades runs of four features for runs of eight, as in store_output
            const f32x16& o = ot[db];
            const int e = 8 * u;
            const uint32_t a0 = pack_bf16(o[e] * inv, o[e + 1] * inv), a1 = pack_bf16(o[e + 2] * inv, o[e + 3] * inv);
            const uint32_t b0 = pack_bf16(o[e + 4] * inv, o[e + 5] * inv), b1 = pack_bf16(o[e + 6] * inv, o[e + 7] * inv);
            const auto r0 = __builtin_amdgcn_permlane32_swap(a0, b0, false, false);
            const auto r1 = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
            if (qrow < N) *reinterpret_cast<u32x4*>(Og + 32 * db + 16 * u + 8 * hh) = u32x4{r0[0], r1[0], r0[1], r1[1]};
        }
}

}  // namespace
