// Attention of whole prompts in which each row sees a run of keys of its own, with scores that may be capped or get a bias by distance.
#pragma once
#include "masked_pv.hpp"
#include "scores.hpp"

namespace {

// ---------------------------------------------------------------------------------------------
// Row i sees the keys [lo, hi) of its entry in `ranges` (all without one), and with `causal` none behind itself.  A workgroup of four waves has 128
// rows of a head, a wave 32 of them; it goes over the tiles from the first key that any of its rows sees to the last, and a wave leaves out those that none of
// its own rows sees.  Exact running max.
struct MaskedParams {
    Params a;          // Q, K, V, O, LSE, sizes, items, c
    Scores s;
    const int2* ranges;
    float unit;        // 1 / scale: a bias in units of raw scores
};

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

template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void attn_masked_kernel(const MaskedParams P) {
    const Params& p = P.a;
    using T = Tile<D>;
    constexpr int NW = 4, BM = 32 * NW, KK = D / 16, DB = D / 32;
    constexpr int LI = T::BYTES / 1024 / NW, RPI = 1024 / T::ROWB;
    __shared__ __attribute__((aligned(16))) uint8_t smem[4 * T::BYTES];  // K[2], V[2]
    __shared__ uint64_t bad[NW];  // keys of the tile with values that are not finite, by the wave that found them
    uint8_t* const Ks = smem;
    uint8_t* const Vs = smem + 2 * T::BYTES;
    const int tid = threadIdx.x, lane = tid & 63, ql = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const auto [head, kv, i] = item_of(p, blockIdx.x);
    const int N = p.N, row0 = i * BM, b = kv / p.Hkv;
    const int qrow = row0 + 32 * wave + ql, qrow_c = min(qrow, N - 1);
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
    const int2 own = range_of(qrow_c);
    const int far = 0x7fffffff;
    // of the wave: the first and the last key that any row sees, and what all rows see
    const int any_lo = wave_fold(own.x < own.y ? own.x : far, lesser), any_hi = wave_fold(own.y, larger);
    const int all_lo = wave_fold(own.x, larger), all_hi = wave_fold(own.y, lesser);
    // of the workgroup
    int wg_lo, wg_hi, wg_all_lo, wg_all_hi;
    {
        const int2 r0 = range_of(min(row0 + lane, N - 1)), r1 = range_of(min(row0 + 64 + lane, N - 1));
        wg_lo = wave_fold(min(r0.x < r0.y ? r0.x : far, r1.x < r1.y ? r1.x : far), lesser);
        wg_hi = wave_fold(max(r0.y, r1.y), larger);
        wg_all_lo = wave_fold(max(r0.x, r1.x), larger);
        wg_all_hi = wave_fold(min(r0.y, r1.y), lesser);
    }
    // ---- requests: a wave moves LI adjacent pieces (1 KiB of whole rows) of a tile, by buffer loads whose buffer is the head's keys: rows past the end
    // of the sequence are out of its range and LDS gets zeros
    const int r_own = RPI * LI * wave + lane / T::CH, cp = lane % T::CH;
    uint32_t offK[LI];
#pragma unroll
    for (int u = 0; u < LI; ++u) offK[u] = (uint32_t)(r_own * T::ROWB + ((cp ^ T::k_mix(r_own + RPI * u)) << 4));
    const uint32_t offV = (uint32_t)(r_own * T::ROWB + ((cp ^ T::v_mix(r_own)) << 4));  // (the same for all pieces)
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr(smem) + wave * LI * 1024);
    const uint32_t bytes = (uint32_t)N * T::ROWB;  // (launched for fewer than 2^32)
    const u32x4 rsrcK = tile_buffer((uint64_t)(uintptr_t)(p.K + (size_t)kv * N * D), bytes), rsrcV = tile_buffer((uint64_t)(uintptr_t)(p.V + (size_t)kv * N * D), bytes);
    auto request = [&](int t, int buf) __attribute__((always_inline)) {
        const uint32_t at = (uint32_t)t * T::BYTES;
        if constexpr (LI == 4) {
            request4_at(rsrcK, at, offK[0], offK[1], offK[2], offK[3], lds0 + buf * T::BYTES);
            request4_at(rsrcV, at, offV, offV, offV, offV, lds0 + (2 + buf) * T::BYTES);
        } else {
            request2_at(rsrcK, at, offK[0], offK[1], lds0 + buf * T::BYTES);
            request2_at(rsrcV, at, offV, offV, lds0 + (2 + buf) * T::BYTES);
        }
    };
    const int t_lo = wg_lo / BN, t_hi = wg_lo < wg_hi ? (wg_hi + BN - 1) / BN : t_lo;
    if (t_lo < t_hi) request(t_lo, 0);
    bf16x8 qf[KK];
    {
        const uint16_t* const Qg = p.Q + ((size_t)head * N + qrow_c) * D;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(Qg + 16 * kk + 8 * hh);
    }
    const float slope2 = BIAS ? P.s.slopes[head % p.Hq] * kLog2e : 0.f;
    f32x16 ot[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) ot[db] = f32x16{0};
    float m2 = -INFINITY, lsum = 0.f;
    const float c = CAP || BIAS ? 1.f : p.c;
    // (one body with a branch around the mask: two bodies were given accumulators of their own, and spilled)
    auto tile = [&](int t, int buf, bool masked) __attribute__((always_inline)) {
        f32x16 st[2];
        uint32_t pk[16];
        __builtin_amdgcn_s_setprio(1);
        qk_tile_pipe<D>(Ks + buf * T::BYTES, qf, st, ql, hh);
        __builtin_amdgcn_s_setprio(0);
        const int key0 = t * BN + 4 * hh;
        if (CAP) cap_scores(P.s, st);
        if (BIAS) bias_scores(P.s, p.c, st, slope2, (float)(qrow - key0));
        if (masked) {
            const uint32_t first = own.x - key0, many = own.y - own.x;
#pragma unroll
            for (int e = 0; e < 32; ++e) {
                const uint32_t k = 32 * (e >> 4) + 8 * ((e & 15) >> 2) + (e & 3);
                const bool ok = k - first < many;
                st[e >> 4][e & 15] = ok ? st[e >> 4][e & 15] : -INFINITY;
            }
        }
        softmax_tile<true, false, DB, true, true>(st, pk, ot, m2, lsum, c, 0, 0, hh, 0.f);
        __builtin_amdgcn_s_setprio(1);
        pv_tile_pipe<D>(Vs + buf * T::BYTES, pk, ot, lane, hh);
        __builtin_amdgcn_s_setprio(0);
    };
    wait_vm0_and_sync();
    for (int t = t_lo; t < t_hi; ++t) {
        const int buf = (t - t_lo) & 1, k0 = t * BN;
        if (t + 1 < t_hi) request(t + 1, buf ^ 1);
        // (no row of the workgroup may get what is not finite among the values of a key that it does not see)
        const bool part = !(k0 >= wg_all_lo && k0 + BN <= wg_all_hi);
        if (part) {
            bad[wave] = clear_not_finite<D, LI>(Vs + buf * T::BYTES, wave * LI, lane);
            __syncthreads();
        }
        if (k0 < any_hi && k0 + BN > any_lo) {
            tile(t, buf, !(k0 >= all_lo && k0 + BN <= all_hi));
        }
        if (part) {
            uint64_t keys = bad[0] | bad[1] | bad[2] | bad[3];
            if (__builtin_expect(keys != 0, 0)) {
                const uint16_t* const Vg = p.V + (size_t)kv * N * D;
#pragma unroll 1
                for (; keys; keys &= keys - 1) {
                    const int k = k0 + __builtin_ctzll(keys);  // (a key of the sequence: behind its end LDS has zeros)
                    add_not_finite<D>(Vg + (size_t)k * D, k >= own.x && k < own.y, ot, hh);
                }
            }
        }
        wait_vm0_and_sync();
    }
    store_output<D>(p, ot, m2, lsum, 0, head, qrow, hh);
}

}  // namespace
