// Attention of each sequence's newest tokens over the paged cache.
#pragma once
#include "decode.hpp"
#include "kvp.hpp"
#include "masked_pv.hpp"
#include "scores.hpp"

namespace {

// ---------------------------------------------------------------------------------------------
// As decode_split_kernel: a wave takes a contiguous part of a range, tiles of 64 keys go from memory to registers one tile ahead and from there into the
// two tiles of LDS that the wave owns, and its score tile has the rows of a KV head, the query heads' n_q newest tokens, as its 32 columns.  A tile is
// four runs of 16 rows, each in a page of its own or not, with a buffer of its own: rows past the sequence's end and runs without a page are out of
// range and give zeros.  The table's entries are read by scalar loads a tile before they are needed.
// Up to 16 rows leave half of the columns free (HALVES): column c + 16 has the same row as c, and of each weight c takes the upper 16 bits, c + 16 what
// they leave; their sums are added where the waves meet.
// More than 32 rows (GROUPED: a prompt in pieces) are cut into groups of as many tokens as give 32, each with a workgroup of its own for each range.
// Each group reads the keys again, and a tile feeds one product of 32 columns: the last 1024 of 16384 tokens, 32 heads over 8, d = 128, 551 us with one range (601 with two), where the products
// alone take 212 at the rate of a large one; the last 256 145 / 53.
// What bounds it: reading the pages once, 4 x 32768 tokens of 8 KV heads, d = 128, 82 us (6.5 TB/s; 7.1 is what a read-only stream reaches), 16 of 200 to 8192 with a
// cap 45 (6.1); behind it the merge, 4.5 us, and for few keys the two launches (2048 keys 9.2 us in a graph).  In front of a tile only scalar work depends on its pages, so pages
// of 16 tokens cost no more than pages of 64.  Waves: four for each range, or one where ranges are dealt out (see the launch).
struct KvpDecode {
    DecodeParams d;  // Hq, g: rows for heads (query heads times new tokens); K, V: the pool; n_cap: M * S
    Scores s;
    const int* table;       // [B, M]
    int n_pages, M, sh_page, n_q;
    int g, tokens, groups;  // query heads per KV head; GROUPED: tokens of a workgroup (their rows at most 32); groups of so many
};

template <int D, bool NT>
__device__ __forceinline__ void kvp_to_regs(const uint16_t* pool, const KvpTile& at, int left, const uint32_t* offs, u32x4* r) {
    using T = Tile<D>;
    constexpr int NI = BN / (1024 / T::ROWB), PER = NI / 4;  // loads of a tile; of a run
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const int rows = at.there >> s & 1 ? min(max(left - 16 * s, 0), 16) : 0;
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(pool)) + at.off[s], 0, __builtin_amdgcn_readfirstlane(rows * T::ROWB), 0x00020000);
#pragma unroll
        for (int u = 0; u < PER; ++u)
            r[s * PER + u] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, offs[u], u * 1024, NT ? 2 : 0));
    }
}

template <int D, int W, int LENS, bool GROUPED, bool HALVES>
__global__ __launch_bounds__(64 * W, D == 64 ? 2 : 1) void kvp_decode_kernel(const KvpDecode P) {
    const DecodeParams& p = P.d;
    using T = Tile<D>;
    constexpr int KK = D / 16, DB = D / 32;
    constexpr int NI = BN / (1024 / T::ROWB);
    constexpr int OROW = D + 4;  // row of the exchange of partial sums, in floats: padded against bank conflicts
    static_assert(32 * OROW * 4 + 64 * 4 <= 2 * T::BYTES, "the exchange has to fit the tiles' memory");
    __shared__ __attribute__((aligned(16))) uint8_t smem[W * 2 * T::BYTES];
    const int lane = threadIdx.x & 63, ql = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint8_t* const Ks = smem + wave * 2 * T::BYTES;
    uint8_t* const Vs = Ks + T::BYTES;
    const int hkv = GROUPED ? blockIdx.x : LENS == LENS_FIXED ? blockIdx.y : blockIdx.z;
    int b = GROUPED || LENS == LENS_FIXED ? blockIdx.z : blockIdx.y, r = GROUPED ? blockIdx.y / P.groups : blockIdx.x, nb = p.n_splits;
    const int tok0 = GROUPED ? (blockIdx.y - r * P.groups) * P.tokens : 0;  // the first of its tokens
    const int ntok = GROUPED ? min(P.tokens, P.n_q - tok0) : P.n_q, rows = P.g * ntok;
    // of a column's row among the entry's
    auto row_of = [&](int col) { return (hkv * P.g + col / ntok) * P.n_q + tok0 + col % ntok; };
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
    const int all_see = max(len - ntok + 1, 0);                         // keys below are seen by every row
    const int Tc = len / BN + (len % BN != 0), per = (Tc + nb - 1) / nb;
    const int r0 = r * per, r1 = min(Tc, r0 + per);
    const int share = (max(r1 - r0, 0) + W - 1) / W;
    const int t_lo = r0 + wave * share, t_hi = min(r1, t_lo + share);
    const int t_whole = min(t_hi, all_see / BN);  // tiles below are seen whole by every row
    const KvpTable table = (KvpTable)(uintptr_t)(P.table + (size_t)b * P.M);
    auto entries = [&](int t) __attribute__((always_inline)) { return kvp_entries(table, t, P.sh_page, P.M); };
    auto place = [&](const KvpEntries& e, int t) __attribute__((always_inline)) { return kvp_tile<D>(e, t, P.sh_page, P.n_pages, p.Hkv, hkv); };
    uint32_t offk[4], offv[4];
    tile_lane_offsets<D>(false, lane, offk);
    tile_lane_offsets<D>(true, lane, offv);
    const int col = min(HALVES ? ql & 15 : ql, rows - 1);
    const int row = row_of(col);
    const int sees = len - ntok + 1 + col % ntok;  // keys that the lane's row sees; its own position is the one before
    const float slope2 = P.s.slopes ? P.s.slopes[row / P.n_q] * kLog2e : 0.f;
    bf16x8 qf[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
        qf[kk] = *reinterpret_cast<const bf16x8*>(p.Q + ((size_t)b * p.Hq + row) * D + 16 * kk + 8 * hh);
    f32x16 ot[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) ot[db] = f32x16{0};
    float m2 = -INFINITY, lsum = 0.f;
    const uint32_t upper = HALVES && ql >= 16 ? 0xffff0000u : 0u;  // what a column leaves out of a weight
    u32x4 rk[NI], rv[NI];
    KvpTile next;              // tile t + 1
    KvpEntries after;          // of tile t + 2
    uint32_t there = 0;        // runs of tile t that have a page
    // tile t.  On entry K(t) is in LDS, rv holds V(t) and, requested after it, rk holds K(t + 1) (HASK1).
    // HASV1 / HASK2: tiles t + 1 / t + 2 exist; FULL: every row sees all of tile t, but for runs without a page
    auto body = [&](int t, auto hasv1_c, auto hask1_c, auto hask2_c, auto full_c) __attribute__((always_inline)) {
        constexpr bool HASV1 = decltype(hasv1_c)::value, HASK1 = decltype(hask1_c)::value, HASK2 = decltype(hask2_c)::value;
        constexpr bool FULL = decltype(full_c)::value;
        f32x16 st[2];
        uint32_t pk[16];
        const uint32_t there_now = there;
        qk_tile_pipe<D>(Ks, qf, st, ql, hh);
        const float c = score_units(P.s, p.c);
        if (P.s.cap2 > 0.f) cap_scores(P.s, st);
        if (P.s.slopes) bias_scores(P.s, p.c, st, slope2, (float)(sees - 1 - t * BN - 4 * hh));
        if (!FULL || there_now != 15u) {
            const int rel = sees - t * BN - 4 * hh;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int k = 32 * (i >> 4) + 8 * ((i & 15) >> 2) + (i & 3);  // (+ 4 hh: the same run)
                const bool ok = k < rel && (there_now >> (k >> 4) & 1);
                st[i >> 4][i & 15] = ok ? st[i >> 4][i & 15] : -INFINITY;
            }
        }
        softmax_halves<HALVES, DB>(st, pk, ot, m2, lsum, c, upper);
        __builtin_amdgcn_sched_barrier(0);  // (requests and LDS writes go out where they are written, not where the scheduler likes them)
        regs_to_tile<D>(Vs, lane, rv);  // V(t) has landed when only K(t + 1) is still out
        if (HASV1) kvp_to_regs<D, !GROUPED>(p.V, next, len - (t + 1) * BN, offv, rv);
        __builtin_amdgcn_sched_barrier(0);
        uint64_t bad = 0;  // (with one token a row that some do not see is behind the sequence's end, and zero)
        if (!FULL && ntok > 1) bad = clear_not_finite<D, NI>(Vs, 0, lane);
        pv_tile_pipe<D>(Vs, pk, ot, lane, hh);
        if (!FULL && __builtin_expect(bad != 0, 0)) {
            const KvpTile at = place(entries(t), t);
#pragma unroll 1
            for (; bad; bad &= bad - 1) {
                const int k = __builtin_ctzll(bad), run = k >> 4;
                const uint64_t off = run == 0 ? at.off[0] : run == 1 ? at.off[1] : run == 2 ? at.off[2] : at.off[3];
                const uint8_t* const value = reinterpret_cast<const uint8_t*>(p.V) + off + (k & 15) * T::ROWB;
                add_not_finite<D>(reinterpret_cast<const uint16_t*>(value), t * BN + k < sees, ot, hh);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (HASK1) {
            regs_to_tile<D>(Ks, lane, rk);  // K(t + 1) has landed when only V(t + 1) is still out
            there = next.there;
        }
        if (HASK2) {
            next = place(after, t + 2);
            kvp_to_regs<D, !GROUPED>(p.K, next, len - (t + 2) * BN, offk, rk);
            after = entries(t + 3);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    using Y = std::true_type;
    using N_ = std::false_type;
    if (t_lo < t_hi) {
        int t = t_lo;
        const KvpTile first = place(entries(t), t);
        after = entries(t + 1);
        there = first.there;
        kvp_to_regs<D, !GROUPED>(p.K, first, len - t * BN, offk, rk);
        kvp_to_regs<D, !GROUPED>(p.V, first, len - t * BN, offv, rv);
        __builtin_amdgcn_sched_barrier(0);
        regs_to_tile<D>(Ks, lane, rk);
        next = place(after, t + 1);
        after = entries(t + 2);
        __builtin_amdgcn_sched_barrier(0);
        if (t + 2 < t_whole) {  // (the request for K(t + 1) is not behind a branch of its own: the compiler's wait counts stay exact)
            kvp_to_regs<D, !GROUPED>(p.K, next, len - (t + 1) * BN, offk, rk);
            do {  // tiles t + 1 and t + 2 are whole and inside the range
                body(t, Y{}, Y{}, Y{}, Y{});
                ++t;
            } while (t + 2 < t_whole);
        } else if (t + 1 < t_hi) {
            kvp_to_regs<D, !GROUPED>(p.K, next, len - (t + 1) * BN, offk, rk);
        }
        while (t + 2 < t_hi) body(t++, Y{}, Y{}, Y{}, N_{});  // (two at most: t_hi <= t_whole + 2)
        if (t + 1 < t_hi) body(t++, Y{}, Y{}, N_{}, N_{});
        body(t, N_{}, N_{}, N_{}, N_{});
    }
    // the waves' sums meet in LDS (in the tiles' memory; each wave writes its own part, behind its own last reads)
    float* const ox = reinterpret_cast<float*>(Ks);
    const float l = xhalf_sum(lsum);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
            *reinterpret_cast<f32x4*>(ox + ql * OROW + 32 * db + 8 * q4 + 4 * hh) =
                f32x4{ot[db][4 * q4], ot[db][4 * q4 + 1], ot[db][4 * q4 + 2], ot[db][4 * q4 + 3]};
    if (hh == 0) {
        ox[32 * OROW + ql] = m2;
        ox[32 * OROW + 32 + ql] = l;
    }
    __syncthreads();
    for (int idx = threadIdx.x; idx < rows * (D / 4); idx += 64 * W) {
        const int cx = idx / (D / 4), c4 = idx - cx * (D / 4);
        const float* const x0 = reinterpret_cast<const float*>(smem);
        constexpr int WS = 2 * T::BYTES / 4;  // floats from one wave's part to the next
        float m = -INFINITY;
#pragma unroll
        for (int v = 0; v < W; ++v) m = fmaxf(m, x0[v * WS + 32 * OROW + cx]);
        const float msub = finite_max(m);
        float lt = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < W; ++v) {
            const float a = __builtin_amdgcn_exp2f(x0[v * WS + 32 * OROW + cx] - msub);
            lt += a * x0[v * WS + 32 * OROW + 32 + cx];
            const float* const x = x0 + v * WS + cx * OROW + 4 * c4;
            f32x4 y = *reinterpret_cast<const f32x4*>(x);
            if (HALVES) {  // (an infinite value times a lower half of 0 is no NaN of the row)
                const f32x4 z = *reinterpret_cast<const f32x4*>(x + 16 * OROW);
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = __builtin_fabsf(y[e]) == INFINITY ? y[e] : y[e] + z[e];
            }
            o += a * y;
        }
        const int rw = row_of(cx);
        if (p.n_splits == 1) {  // the only range: this is the result
            const size_t at = (size_t)b * p.Hq + rw;
            const float inv = lt == 0.f ? 0.f : 1.f / lt;
            *reinterpret_cast<u32x2*>(p.O + at * D + 4 * c4) = u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
            if (p.LSE && c4 == 0) p.LSE[at] = lt == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(lt)) * kLn2;
        } else {
            *reinterpret_cast<f32x4*>(p.opart + (slot + rw) * D + 4 * c4) = o;
            if (c4 == 0) {
                p.pm[slot + rw] = m;
                p.lpart[slot + rw] = lt;
            }
        }
    }
}

}  // namespace
