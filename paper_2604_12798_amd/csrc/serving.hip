// C ABI of the serving operators around the 8-bit cache (declared in vfa.h): argument checks, kernel selection and launches.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <math.h>

#include "vfa.h"

#include "common.hpp"
#include "host.hpp"
#include "norm_rope.hpp"
#include "kv8.hpp"
#include "kv8_decode.hpp"

namespace {

inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
int launched() { return hipGetLastError() == hipSuccess ? VFA_OK : VFA_ERR_HIP; }

// What the cache's entry points have in common; *done: there is nothing to do.
int check_cache8(const void* K8, const void* V8, const void* KS, const void* VS, int B, int Hkv, int n_cap, int d, bool* done) {
    *done = false;
    if (B < 0 || Hkv <= 0 || n_cap < 0 || d <= 0) return VFA_ERR_INVALID_ARG;
    if ((d != 64 && d != 128) || n_cap % BN != 0) return VFA_ERR_UNSUPPORTED;
    if (B == 0) { *done = true; return VFA_OK; }
    if (n_cap > 0 && (!K8 || !V8 || !KS || !VS || !aligned16(K8) || !aligned16(V8))) return VFA_ERR_INVALID_ARG;
    if (2LL * Hkv > 65535 || (long long)B * Hkv > 65535) return VFA_ERR_UNSUPPORTED;
    return VFA_OK;
}

// Strides of rows that are read 16 bytes at a time
bool whole_runs(long long a, long long b, long long c) { return ((a | b | c) & 7) == 0; }

template <typename F>
void with_d(int d, F f) {
    if (d == 128) f(std::integral_constant<int, 128>{});
    else f(std::integral_constant<int, 64>{});
}

}  // namespace

extern "C" {

int vfa_qk_norm_rope_fwd(const void* Xq, const void* Xk, const void* Xv, void* Q, void* K, void* V, int B, int N, int Hq, int Hkv, int d,
                         long long q_sb, long long q_sn, long long q_sh, long long k_sb, long long k_sn, long long k_sh, long long v_sb,
                         long long v_sn, long long v_sh, int norm, const void* q_weight, const void* k_weight, float eps,
                         const float* cos_sin, int n_pos, int rot_dim, int interleaved, const int* first_pos, int first, void* stream) {
    if (B < 0 || N < 0 || Hq <= 0 || Hkv <= 0 || d <= 0 || rot_dim < 0) return VFA_ERR_INVALID_ARG;
    if ((norm != 0 && norm != 1) || (interleaved != 0 && interleaved != 1)) return VFA_ERR_INVALID_ARG;
    if (d != 64 && d != 128) return VFA_ERR_UNSUPPORTED;
    if (rot_dim > d || rot_dim % 16 != 0) return VFA_ERR_INVALID_ARG;
    if (norm ? !(eps >= 0.f) || !isfinite(eps) : q_weight || k_weight) return VFA_ERR_INVALID_ARG;
    if (rot_dim > 0 && (!cos_sin || !aligned16(cos_sin) || n_pos <= 0 || !aligned4(first_pos))) return VFA_ERR_INVALID_ARG;
    if (B == 0 || N == 0) return VFA_OK;
    if (!Xq || !Xk || !Q || !K || !Xv != !V) return VFA_ERR_INVALID_ARG;
    if (!aligned16(Xq) || !aligned16(Xk) || !aligned16(Xv) || !aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(q_weight) ||
        !aligned16(k_weight))
        return VFA_ERR_INVALID_ARG;
    if (!whole_runs(q_sb, q_sn, q_sh) || !whole_runs(k_sb, k_sn, k_sh) || (V && !whole_runs(v_sb, v_sn, v_sh))) return VFA_ERR_INVALID_ARG;
    RopeParams p{};
    p.X[0] = (const uint16_t*)Xq; p.X[1] = (const uint16_t*)Xk; p.X[2] = (const uint16_t*)Xv;
    p.Y[0] = (uint16_t*)Q; p.Y[1] = (uint16_t*)K; p.Y[2] = (uint16_t*)V;
    p.sb[0] = q_sb; p.sn[0] = q_sn; p.sh[0] = q_sh;
    p.sb[1] = k_sb; p.sn[1] = k_sn; p.sh[1] = k_sh;
    p.sb[2] = v_sb; p.sn[2] = v_sn; p.sh[2] = v_sh;
    p.W[0] = (const uint16_t*)q_weight; p.W[1] = (const uint16_t*)k_weight;
    p.cos_sin = cos_sin; p.first_pos = first_pos; p.first = first; p.n_pos = n_pos; p.rot = rot_dim;
    const long long heads = (long long)Hq + Hkv + (V ? Hkv : 0), tokens = (long long)B * N;
    if (tokens > 0x7fffffffLL || heads > 0x7fffffffLL) return VFA_ERR_UNSUPPORTED;
    p.N = N; p.tokens = (int)tokens; p.Hq = Hq; p.Hkv = Hkv; p.heads = (int)heads; p.eps = eps;
    const int rows = 256 / (d / 16);
    const long long wgs = (tokens + rows - 1) / rows;
    // Heads of a thread: four, or one where that gives fewer than two workgroups for each compute unit (16 x 1 tokens of 48 heads: 6.3 / 4.2 us).
    // Loads and stores past the caches from 256 MiB on (d = 128, us: 2 x 16384 tokens of 48 heads 178 / 164, 2 x 6240 of 80, neighbouring pairs, 110 / 98;
    // below 3 x 777 of 24, d = 64, 14 MiB, 5.7 / 6.2), if each covers whole lines of 128 bytes; in parts, a line is fetched twice (7 x 2495 of 96, d = 64, 101 / 128;
    // 2 x 6240 of 80, half of the features rotated, 112 / 131)
    const int n_cu = cu_count() > 0 ? cu_count() : 256;
    const bool few = wgs * ((heads + 3) / 4) < 2 * n_cu;
    const long long ys = few ? heads : (heads + 3) / 4;
    if (ys > 65535 || wgs * ys > kMaxWorkgroups256) return VFA_ERR_UNSUPPORTED;
    const bool stream_past = tokens * heads * d >= 1LL << 26 && d == 128 && (interleaved || rot_dim % 128 == 0);
    const dim3 grid((unsigned)wgs, (unsigned)ys);
    hipStream_t s = (hipStream_t)stream;
    (void)hipGetLastError();
    with_d(d, [&](auto d_c) {
        constexpr int D = decltype(d_c)::value;
        auto launch = [&](auto norm_c, auto per_c, auto past_c) {
            constexpr bool NORM = decltype(norm_c)::value, PAST = decltype(past_c)::value;
            constexpr int PER = decltype(per_c)::value;
            if (rot_dim == 0) norm_rope_kernel<D, NORM, PAIRS_NONE, PER, PAST><<<grid, 256, 0, s>>>(p);
            else if (interleaved) norm_rope_kernel<D, NORM, PAIRS_NEXT, PER, PAST><<<grid, 256, 0, s>>>(p);
            else norm_rope_kernel<D, NORM, PAIRS_HALF, PER, PAST><<<grid, 256, 0, s>>>(p);
        };
        auto sized = [&](auto norm_c) {
            using std::integral_constant;
            if (few) launch(norm_c, integral_constant<int, 1>{}, std::false_type{});
            else if (!stream_past) launch(norm_c, integral_constant<int, 4>{}, std::false_type{});
            else if constexpr (D == 128) launch(norm_c, integral_constant<int, 4>{}, std::true_type{});
        };
        if (norm) sized(std::true_type{});
        else sized(std::false_type{});
    });
    return launched();
}

int vfa_kv8_append(const void* K, const void* V, void* K8, void* V8, void* KS, void* VS, int B, int Hkv, int n_cap, int n_in, int d,
                   long long k_sb, long long k_sh, long long k_sn, long long v_sb, long long v_sh, long long v_sn, const int* old_lens,
                   const int* new_lens, int n_old, int n_new, void* stream) {
    bool done;
    const int rc = check_cache8(K8, V8, KS, VS, B, Hkv, n_cap, d, &done);
    if (rc != VFA_OK || n_in < 0) return rc != VFA_OK ? rc : VFA_ERR_INVALID_ARG;
    if (!old_lens != !new_lens || !aligned4(old_lens) || !aligned4(new_lens)) return VFA_ERR_INVALID_ARG;
    if (!old_lens && (n_old < 0 || n_old > n_new || n_new > n_cap || n_new - n_old > n_in)) return VFA_ERR_INVALID_ARG;
    if (done || n_cap == 0 || n_in == 0 || (!old_lens && n_old == n_new)) return VFA_OK;
    if (!K || !V || !aligned16(K) || !aligned16(V) || !whole_runs(k_sb, k_sh, k_sn) || !whole_runs(v_sb, v_sh, v_sn)) return VFA_ERR_INVALID_ARG;
    Kv8Append p{};
    p.X[0] = (const uint16_t*)K; p.X[1] = (const uint16_t*)V;
    p.sb[0] = k_sb; p.sh[0] = k_sh; p.sn[0] = k_sn;
    p.sb[1] = v_sb; p.sh[1] = v_sh; p.sn[1] = v_sn;
    p.C[0] = (uint8_t*)K8; p.C[1] = (uint8_t*)V8; p.S[0] = (uint8_t*)KS; p.S[1] = (uint8_t*)VS;
    p.old_lens = old_lens; p.new_lens = new_lens; p.old_len = n_old; p.new_len = n_new;
    p.n_in = n_in; p.n_cap = n_cap; p.T = n_cap / BN; p.Hkv = Hkv;
    (void)hipGetLastError();
    if (n_in == 1) {
        const int rows = 2 * B * Hkv, each = 512 / d;
        with_d(d, [&](auto d_c) {
            kv8_append_one_kernel<decltype(d_c)::value><<<(unsigned)ceil_div(rows, each), 64, 0, (hipStream_t)stream>>>(p, rows);
        });
        return launched();
    }
    // blocks that the rows can reach, wherever they begin
    const int most = n_in < n_cap ? n_in : n_cap;
    const long long tiles = old_lens ? (most + BN - 2LL) / BN + 1 : (n_new - 1) / BN - n_old / BN + 1;
    if (tiles * 2 * Hkv * B > kMaxWorkgroups256) return VFA_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)tiles, (unsigned)(2 * Hkv), (unsigned)B);
    with_d(d, [&](auto d_c) { kv8_append_kernel<decltype(d_c)::value><<<grid, 2 * d, 0, (hipStream_t)stream>>>(p); });
    return launched();
}

int vfa_kv8_read(const void* K8, const void* V8, const void* KS, const void* VS, void* K, void* V, int B, int Hkv, int n_cap, int n, int d,
                 const int* seq_lens, int seq_len, void* stream) {
    bool done;
    const int rc = check_cache8(K8, V8, KS, VS, B, Hkv, n_cap, d, &done);
    if (rc != VFA_OK || n < 0 || n > n_cap || !aligned4(seq_lens)) return rc != VFA_OK ? rc : VFA_ERR_INVALID_ARG;
    if (done || n == 0) return VFA_OK;
    if (!K || !V || !aligned16(K) || !aligned16(V)) return VFA_ERR_INVALID_ARG;
    Kv8Read p{};
    p.C[0] = (const uint8_t*)K8; p.C[1] = (const uint8_t*)V8; p.S[0] = (const uint8_t*)KS; p.S[1] = (const uint8_t*)VS;
    p.Y[0] = (uint16_t*)K; p.Y[1] = (uint16_t*)V;
    p.seq_lens = seq_lens; p.seq_len = seq_len; p.n = n; p.n_cap = n_cap; p.T = n_cap / BN; p.Hkv = Hkv;
    const long long tiles = ceil_div(n, BN);
    if (tiles * 2 * Hkv * B > kMaxWorkgroups256) return VFA_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)tiles, (unsigned)(2 * Hkv), (unsigned)B);
    (void)hipGetLastError();
    with_d(d, [&](auto d_c) { kv8_read_kernel<decltype(d_c)::value><<<grid, 2 * d, 0, (hipStream_t)stream>>>(p); });
    return launched();
}

// One range for each KV head, which is one launch and no partial sums, where there are few keys, and more of them the more units the heads fill; the limits lie
// where the two meet (us, one range / the best number of ranges; d = 128: 8 heads of 768 keys 6.1 / 6.8, of 1024 7.0 / 6.5, of 1536 10.2 / 7.2; 128 of 1536
// 12.2 / 12.8, of 200 to 2048 14.1 / 13.1; 256 of 100 to 1024 10.2 / 13.5, of 200 to 4096 28.5 / 28.8, to 5120 36.1 / 33.9; d = 64: 16 of 1024 5.2 / 6.5, of
// 2048 9.9 / 6.7; 128 of 100 to 2048 8.6 / 10.0, to 2560 10.2 / 10.5, to 3200 12.0 / 11.2; 256 of 100 to 2048 10.0 / 12.8, to 6208 23.1 / 23.8, to 8192
// 29.7 / 27.9; 288 of 300 to 6144 26.0 / 26.6, to 6175 26.9 / 26.2, to 8192 34.6 / 31.9).
// Else as many workgroups as there are compute units where all are equally long: a unit has 64 KiB on their way to it in either case, and fewer
// partial sums (32 heads of 32768 keys, d = 128: 8 ranges 45.0, 12 46.8, 16 49.5, 24 45.7; 128 of 4224: 1 27.0, 2 26.0, 3 27.0, 6 25.8; d = 64, 128 of
// 32768: 1 119, 2 80, 3 85, 6 83).  Where lengths differ and ranges are dealt out, as many as the units hold at a time, three each, so that what a range is
// longer than the mean weighs less (128 heads of 200 to 8192 keys: 2 ranges 30.2, 4 29.0, 6 27.8, 8 29.9; 512 of 200 to 2048: 1 29.1, 2 33.2; more fit
// in at d = 64, 288 heads of 300 to 6175 keys: 2 30.1, 3 28.3, 4 26.2), but one where
// more than 16 rows make more of the merge (32 heads of 500 to 8192 keys, 32 rows each: 4 ranges 18.1, 8 16.1, 16 19.4, 24 22.5; 20 rows: 16.7, 14.5, 16.5,
// 21.2; 64 heads, 24 rows, d = 64: 2 18.6, 4 13.7, 8 14.7, 16 20.0).
int vfa_kv8_decode_splits(int B, int Hq, int Hkv, int n_q, int d, int n_keys, int varlen) {
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || n_q <= 0 || n_keys <= 0 || (long long)B * Hkv > 65535) return 1;
    const int n_cu = cu_count() > 0 ? cu_count() : 256, all = n_keys / BN + (n_keys % BN != 0);  // (n_keys + 63 may not fit)
    const long long rows = (long long)(Hq / Hkv) * n_q;
    const int g = Hq / Hkv, tokens = rows <= 32 ? n_q : g < 32 ? 32 / g : 1;
    const long long heads = (long long)B * Hkv * (((long long)n_q + tokens - 1) / tokens);  // (with more than 32 rows, groups of them)
    const int most = heads >= n_cu ? (d == 64 ? 96 : 64) : 2 * heads >= n_cu ? (d == 64 ? 40 : 28) : d == 64 ? 16 : 12;
    if (all <= most) return 1;
    // more than 32 rows: two workgroups for each compute unit (32 heads over 8, 64 of 16384 tokens: 1 range 80 us, 2 48, 4 32, 8 32; 256: 1 90, 2 93, 4 101)
    if (rows > 32) return (int)max(1LL, min(2LL * n_cu / heads, (all + 3) / 4LL));
    const bool dealt = varlen && B > 1 && rows <= 16;
    long long n = (dealt ? 3LL * n_cu + (d == 64 ? heads - 1 : 0) : (long long)n_cu) / heads;
    // no range without a tile for each of its waves, and two if there are enough for the units (64 heads of 2000 keys: 4 ranges 11.2, 8 12.3)
    if (dealt) n = min(n, max((all + 7) / 8LL, (n_cu + heads - 1) / heads));
    return (int)max(1LL, min(n, (all + 3) / 4LL));
}

size_t vfa_kv8_decode_workspace_bytes(int B, int Hq, int n_q, int d, int n_splits) {
    if (B <= 0 || Hq <= 0 || n_q <= 0 || d <= 0 || n_splits <= 0) return 0;
    const size_t bytes = (size_t)B * Hq * n_q * n_splits * (2 + (size_t)d) * sizeof(float) + 2 * sizeof(int) * (size_t)B;
    return (bytes + 255) & ~(size_t)255;
}

int vfa_kv8_decode_fwd(const void* Q, const void* K8, const void* V8, const void* KS, const void* VS, void* O, float* LSE, int B, int Hq,
                       int Hkv, int n_cap, int n_q, int d, const int* seq_lens, int n_keys, int n_splits, float softmax_scale,
                       void* workspace, size_t workspace_bytes, void* stream) {
    bool done;
    const int rc = check_cache8(K8, V8, KS, VS, B, Hkv, n_cap, d, &done);
    if (rc != VFA_OK) return rc;
    if (Hq <= 0 || Hq % Hkv != 0 || n_q < 0 || n_splits < 1 || n_splits > 4096 || !isfinite(softmax_scale)) return VFA_ERR_INVALID_ARG;
    if (!aligned4(seq_lens) || (!seq_lens && (n_keys < 0 || n_keys > n_cap))) return VFA_ERR_INVALID_ARG;
    const int g = Hq / Hkv;
    if (g > 32) return VFA_ERR_UNSUPPORTED;
    const long long rows = (long long)g * n_q;
    if (done || n_q == 0) return VFA_OK;
    if (!Q || !O || !aligned16(Q) || !aligned16(O) || !aligned4(LSE)) return VFA_ERR_INVALID_ARG;
    const bool grouped = rows > 32;
    const int tokens = grouped ? 32 / g : n_q;
    const long long groups = ((long long)n_q + tokens - 1) / tokens, out_rows = (long long)B * Hq * n_q;
    if (grouped && groups * n_splits > 65535) return VFA_ERR_UNSUPPORTED;
    const long long wgs = (long long)B * Hkv * n_splits * groups;
    if (out_rows > 0x7fffffffLL || wgs > kMaxWorkgroups256 || (n_splits > 1 && out_rows > kMaxWorkgroups256)) return VFA_ERR_UNSUPPORTED;
    if (n_splits > 1 && (!workspace || !aligned16(workspace) || workspace_bytes < vfa_kv8_decode_workspace_bytes(B, Hq, n_q, d, n_splits)))
        return VFA_ERR_INVALID_ARG;
    if (n_cap == 0) n_splits = 1;  // (no keys, so no ranges to deal out)
    Kv8Decode P{};
    DecodeParams& p = P.d;
    P.K8 = (const uint8_t*)K8; P.V8 = (const uint8_t*)V8; P.KS = (const uint8_t*)KS; P.VS = (const uint8_t*)VS;
    P.T = n_cap / BN; P.n_q = n_q; P.g = g; P.tokens = tokens; P.groups = (int)groups;
    p.Q = (const uint16_t*)Q; p.O = (uint16_t*)O; p.LSE = LSE;
    p.B = B; p.Hq = Hq * n_q; p.Hkv = Hkv; p.n_cap = n_cap; p.n_keys = seq_lens ? n_cap : n_keys; p.seq_lens = seq_lens; p.n_splits = n_splits;
    p.g = (int)rows;
    p.c = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)d)) * kLog2e;
    const size_t slots = (size_t)B * Hq * n_q * n_splits;
    p.opart = (float*)workspace; p.pm = p.opart + slots * d; p.lpart = p.pm + slots; p.dealt = (int*)(p.lpart + slots);
    hipStream_t s = (hipStream_t)stream;
    const int n_cu = cu_count() > 0 ? cu_count() : 256;
    (void)hipGetLastError();
    const bool dealt = seq_lens && n_splits > 1 && B > 1 && (B <= 64 || (B <= DEAL_MAX_B && (long long)B * Hkv * n_splits <= 8LL * n_cu && ceil_div(n_cap, BN) > 2 * n_splits));
    with_d(d, [&](auto d_c) {
        constexpr int D = decltype(d_c)::value;
        // Waves of a workgroup: four have 64 KiB on their way at d = 128, which is what a compute unit gets at a time (one workgroup of 8 waves
        // takes as long for 2048 keys as one of 4, 13 us); d = 64 has half as much in a wave, and one long range eight waves (32 heads of 2048 keys
        // 9.9 / 8.2 us, 128 of 32768 119 / 94)
        const bool wide = D == 64 && n_splits == 1 && p.n_keys > 1024 && !grouped;
        auto launch = [&](auto rt_c, auto w_c, auto halves_c) {
            constexpr int RT = decltype(rt_c)::value, W = decltype(w_c)::value;
            constexpr bool HALVES = decltype(halves_c)::value;
            const dim3 grid((unsigned)n_splits, (unsigned)B, (unsigned)Hkv);
            if constexpr (W == 4) {  // (one range is not dealt out)
                if (dealt) {
                    kv8_decode_kernel<D, RT, W, LENS_DEALT, false, HALVES><<<grid, 64 * W, 0, s>>>(P);
                    return;
                }
            }
            if (!seq_lens) kv8_decode_kernel<D, RT, W, LENS_ONE, false, HALVES><<<grid, 64 * W, 0, s>>>(P);
            else kv8_decode_kernel<D, RT, W, LENS_FIXED, false, HALVES><<<dim3((unsigned)n_splits, (unsigned)Hkv, (unsigned)B), 64 * W, 0, s>>>(P);
        };
        using std::integral_constant;
        auto sized = [&](auto w_c) {
            if (rows <= 8) launch(integral_constant<int, 1>{}, w_c, std::true_type{});
            else if (rows <= 16) launch(integral_constant<int, 1>{}, w_c, std::false_type{});
            else launch(integral_constant<int, 2>{}, w_c, std::false_type{});
        };
        if (grouped) {
            const dim3 grid((unsigned)Hkv, (unsigned)(groups * n_splits), (unsigned)B);
            if (!seq_lens) kv8_decode_kernel<D, 2, 4, LENS_ONE, true><<<grid, 256, 0, s>>>(P);
            else if (dealt) kv8_decode_kernel<D, 2, 4, LENS_DEALT, true><<<grid, 256, 0, s>>>(P);
            else kv8_decode_kernel<D, 2, 4, LENS_FIXED, true><<<grid, 256, 0, s>>>(P);
        } else if (wide) {
            if constexpr (D == 64) sized(integral_constant<int, 8>{});
        } else {
            sized(integral_constant<int, 4>{});
        }
        if (n_splits == 1) return;
        const dim3 grid((unsigned)p.Hq, (unsigned)B);
        if (dealt) decode_merge_kernel<D, SLOTS_TABLE, true><<<grid, 256, 0, s>>>(p);
        else decode_merge_kernel<D, SLOTS_FIXED, true><<<grid, 256, 0, s>>>(p);
    });
    return launched();
}

}  // extern "C"
