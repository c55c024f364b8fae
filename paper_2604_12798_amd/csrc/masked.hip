// C ABI of the paged cache and of masked, capped or biased attention (declared in vfa.h): argument checks, kernel selection and launches.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <math.h>

#include "vfa.h"

#include "common.hpp"
#include "host.hpp"
#include "kvp.hpp"
#include "kvp_decode.hpp"
#include "row_ranges.hpp"
#include "attn_masked.hpp"

namespace {

inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline bool aligned8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }
int launched() { return hipGetLastError() == hipSuccess ? VFA_OK : VFA_ERR_HIP; }

// What the paged cache's entry points have in common; *done: there is nothing to do.
int check_pages(const void* K, const void* V, int n_pages, const int* table, int M, int B, int Hkv, int page, int d, bool* done) {
    *done = false;
    if (B < 0 || Hkv <= 0 || n_pages < 0 || M < 0 || page <= 0 || d <= 0) return VFA_ERR_INVALID_ARG;
    if ((d != 64 && d != 128) || page < 16 || (page & (page - 1)) != 0) return VFA_ERR_UNSUPPORTED;
    if ((long long)M * page > 1LL << 30) return VFA_ERR_UNSUPPORTED;
    if (B == 0) { *done = true; return VFA_OK; }
    if (n_pages > 0 && (!K || !V || !aligned16(K) || !aligned16(V))) return VFA_ERR_INVALID_ARG;
    if (M > 0 && (!table || !aligned4(table))) return VFA_ERR_INVALID_ARG;
    if (2LL * Hkv > 65535 || (long long)B * Hkv > 65535) return VFA_ERR_UNSUPPORTED;
    return VFA_OK;
}

int log2_of(int page) {
    int s = 0;
    while ((1 << s) < page) ++s;
    return s;
}

// Strides of rows that are read 16 bytes at a time
bool whole_runs(long long a, long long b, long long c) { return ((a | b | c) & 7) == 0; }

// cap: 0 = none, else 0.001 to 1000 (see Scores)
bool cap_ok(float cap) { return cap == 0.f || (cap >= 0.001f && cap <= 1000.f); }
// A slope over the least stays far from the end of fp32; with more than the largest, scores of ordinary rows pass 2^28, where the difference to a rounded max
// may be an exponent that gives infinity
bool scale_ok(float scale) { return scale <= 0.f || (scale >= 0x1p-64f && scale <= 0x1p16f); }
Scores scores_of(const float* slopes, float cap, float scale) { return Scores{slopes, cap * kLog2e, cap > 0.f ? 2.f * kLog2e * scale / cap : 0.f}; }

// Whether the ranges of a batch of sequences of up to `tiles` tiles are dealt out by length (see varlen_find, which also says why not): they are counted in an int, and pages may be
// shared or missing, so that the memory that tokens would take does not bound them.
constexpr int DEAL_FREELY_B = 64;
constexpr long long kDealtPerUnit = 8;
bool deals(int B, int Hkv, int n_splits, int tiles, int n_cu) {
    if (n_splits <= 1 || B <= 1 || (long long)B * ((long long)tiles + n_splits) > 0x7fffffffLL) return false;
    return B <= DEAL_FREELY_B || (B <= DEAL_MAX_B && (long long)B * Hkv * n_splits <= kDealtPerUnit * n_cu && tiles > 2 * n_splits);
}

template <typename F>
void with_d(int d, F f) {
    if (d == 128) f(std::integral_constant<int, 128>{});
    else f(std::integral_constant<int, 64>{});
}

}  // namespace

extern "C" {

int vfa_kvp_append(const void* K, const void* V, void* KP, void* VP, const int* table, int B, int Hkv, int n_pages, int page, int max_pages,
                   int n_in, int d, long long k_sb, long long k_sh, long long k_sn, long long v_sb, long long v_sh, long long v_sn,
                   const int* old_lens, const int* new_lens, int n_old, int n_new, void* stream) {
    bool done;
    const int rc = check_pages(KP, VP, n_pages, table, max_pages, B, Hkv, page, d, &done);
    if (rc != VFA_OK || n_in < 0) return rc != VFA_OK ? rc : VFA_ERR_INVALID_ARG;
    if (!old_lens != !new_lens || !aligned4(old_lens) || !aligned4(new_lens)) return VFA_ERR_INVALID_ARG;
    const int cap = max_pages * page;
    if (!old_lens && (n_old < 0 || n_old > n_new || n_new > cap || n_new - n_old > n_in)) return VFA_ERR_INVALID_ARG;
    if (done || cap == 0 || n_pages == 0 || n_in == 0 || (!old_lens && n_old == n_new)) return VFA_OK;
    if (!K || !V || !aligned16(K) || !aligned16(V) || !whole_runs(k_sb, k_sh, k_sn) || !whole_runs(v_sb, v_sh, v_sn)) return VFA_ERR_INVALID_ARG;
    KvpAppend p{};
    p.X[0] = (const uint16_t*)K; p.X[1] = (const uint16_t*)V;
    p.sb[0] = k_sb; p.sh[0] = k_sh; p.sn[0] = k_sn;
    p.sb[1] = v_sb; p.sh[1] = v_sh; p.sn[1] = v_sn;
    p.Y[0] = (uint16_t*)KP; p.Y[1] = (uint16_t*)VP;
    p.table = table; p.old_lens = old_lens; p.new_lens = new_lens; p.old_len = n_old; p.new_len = n_new;
    p.n_in = n_in; p.n_pages = n_pages; p.M = max_pages; p.Hkv = Hkv; p.sh_page = log2_of(page);
    hipStream_t s = (hipStream_t)stream;
    (void)hipGetLastError();
    const int rows = 2 * B * Hkv;
    if (n_in == 1) {
        with_d(d, [&](auto d_c) { kvp_append_kernel<decltype(d_c)::value, true><<<(unsigned)ceil_div(rows, 512 / d), 64, 0, s>>>(p, rows); });
        return launched();
    }
    const int most = min(n_in, cap), each = 4 * 2048 / d;
    const long long groups = ((long long)(old_lens ? most : n_new - n_old) + each - 1) / each;
    if (groups * 2 * Hkv * B > kMaxWorkgroups256) return VFA_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)groups, (unsigned)(2 * Hkv), (unsigned)B);
    with_d(d, [&](auto d_c) { kvp_append_kernel<decltype(d_c)::value, false><<<grid, 256, 0, s>>>(p, rows); });
    return launched();
}

// Two tiles a range at least (8 heads of 2048 keys, d = 128: 8 ranges 10.3 us, 16 9.4; of 600 1 12.1, 3 9.9, 4 9.8), one range where there are few.  Equal lengths:
// as many ranges as compute units, whose workgroups of four waves have a unit each at d = 128 and half of one at d = 64 (32 heads of 32768 keys 4 ranges 96, 6 83, 8
// 85, 16 87, 32 92; 128 of 4096: 1 55, 2 46, 4 50; 256 of 1000: 1 25.8, 2 30.6; 8 of 8000: 16 14.1, 32 11.8, 48 17.1; d = 64: 16 of 2048 8 8.7, 16 8.1).  Rounded down: 136 heads
// of 1024 keys 1 range 17, 2 25, of 4096 52 / 68 (3: 53), of 16384 198 / 233 (3: 179); 192 of them 20 / 27, 66 / 75, 249 / 252; 248 of them 23 / 30, 83 / 88, 325 / 315.
// Lengths of their own, dealt out to workgroups of one wave: as many as the units hold (128 heads of 200 to 8192 keys, d = 128: 4 ranges 55, 6 51, 8 49.5, 12 55, 16 56; with
// four waves each 2 55, 4 54.6, 8 64.5; 64 of 500 to 16384: 8 49.9, 16 48.4, 24 55.8; d = 64, 128 of 300 to 8192: 8 28, 16 26.9, 24 29.6), and above 64 sequences as many as are
// dealt at all (100 heads of 1000 keys 7 ranges 16.8 dealt, 8 27 of four waves each; 80 of 1500 11 17.4, 12 28).
// More than one and a half heads for each unit keep them busy with one range each if lengths are even, and wait for the longest if they are not.  Which they are is not known here, the
// capacity is.  Even from 200 up to it / one of it and the others 200, 64 x 8 heads, d = 128: of 2048 1 range 48 / 33, 2 56 / 21, 4 58 / 24; of 4096 86 / 51, 97 / 21, 94 / 24; of 8192 166 / 87,
// 182 / 23, 175 / 27; of 16384 324 / 160, 349 / 28, 341 / 34 (of 8192 50 x 8 136 / 86, 162 / 22, 145 / 25; 70 x 8 199 / 92, 209 / 25, three 203 / 28, four, not dealt, 199 / 68; d = 64, 64 x 8
// 94 / 50, 97 / 16, 92 / 16).  So one up to 4096 keys, which one unit reads in 40 us (20 at d = 64), above that up to four while there are no
// more than 1024 heads (64 x 32 of 8192 695 / 136, two 735 / 73; d = 64 321 / 70, 371 / 40) and they are dealt.
// More than 256 sequences are not dealt, but take more than one range above 2048 keys too (300 heads of 100 to 1000 keys 1 range 18, 3 31; of 4000 58 / 63, all of 4000 121 / 108; one of
// 32768 and the others 200 288 / 115; 512 of 200 to 8192 168, 2 173, one of 8192 and the others 200 84 / 61).
int vfa_kvp_decode_splits(int B, int Hq, int Hkv, int n_q, int d, int n_keys, int varlen) {
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || n_q <= 0 || n_keys <= 0 || (long long)B * Hkv > 65535) return 1;
    const int n_cu = cu_count() > 0 ? cu_count() : 256, all = n_keys / BN + (n_keys % BN != 0);  // (n_keys + 63 may not fit)
    const long long rows = (long long)(Hq / Hkv) * n_q;
    const int g = Hq / Hkv, tokens = rows <= 32 ? n_q : g < 32 ? 32 / g : 1;
    const long long heads = (long long)B * Hkv * (((long long)n_q + tokens - 1) / tokens);  // (with more than 32 rows, groups of them)
    if (all <= (d == 64 ? 8 : 5)) return 1;
    const long long units = (long long)n_cu * (d == 64 ? 2 : 1);
    auto bounded = [&](long long n) { return (int)max(1LL, min(n, min((all + 1LL) / 2, 4096LL))); };
    if (!varlen || B == 1 || rows > 32) return bounded(units / heads);
    const bool busy = 2 * heads > 3LL * n_cu;
    if (busy && all <= 4096 / BN) return 1;
    const int n = bounded(max(4 * units / heads, busy ? min(4LL, kDealtPerUnit * n_cu / heads) : 1));
    const int dealt = B <= DEAL_FREELY_B ? n : (int)min((long long)n, min(kDealtPerUnit * n_cu / heads, (all - 1LL) / 2));
    if (deals(B, Hkv, dealt, all, n_cu)) return dealt;
    return bounded((all > 2048 / BN ? 4 : 1) * units / heads);
}

size_t vfa_kvp_decode_workspace_bytes(int B, int Hq, int n_q, int d, int n_splits) {
    if (B <= 0 || Hq <= 0 || n_q <= 0 || d <= 0 || n_splits <= 0) return 0;
    const size_t bytes = (size_t)B * Hq * n_q * n_splits * (2 + (size_t)d) * sizeof(float) + 2 * sizeof(int) * (size_t)B;
    return (bytes + 255) & ~(size_t)255;
}

int vfa_kvp_decode_fwd(const void* Q, const void* KP, const void* VP, const int* table, void* O, float* LSE, int B, int Hq, int Hkv, int n_pages,
                       int page, int max_pages, int n_q, int d, const int* seq_lens, int n_keys, int n_splits, float softmax_scale,
                       float score_cap, const float* slopes, void* workspace, size_t workspace_bytes, void* stream) {
    bool done;
    const int rc = check_pages(KP, VP, n_pages, table, max_pages, B, Hkv, page, d, &done);
    if (rc != VFA_OK) return rc;
    const int n_cap = max_pages * page;
    if (Hq <= 0 || Hq % Hkv != 0 || n_q < 0 || n_splits < 1 || n_splits > 4096 || !isfinite(softmax_scale) || !scale_ok(softmax_scale) || !cap_ok(score_cap)) return VFA_ERR_INVALID_ARG;
    if (!aligned4(seq_lens) || !aligned4(slopes) || (!seq_lens && (n_keys < 0 || n_keys > n_cap))) return VFA_ERR_INVALID_ARG;
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
    if (out_rows > 0x7fffffffLL || wgs > kMaxWorkgroups256 / 2 || (n_splits > 1 && out_rows > kMaxWorkgroups256)) return VFA_ERR_UNSUPPORTED;
    if (n_splits > 1 && (!workspace || !aligned16(workspace) || workspace_bytes < vfa_kvp_decode_workspace_bytes(B, Hq, n_q, d, n_splits)))
        return VFA_ERR_INVALID_ARG;
    if (n_cap == 0) n_splits = 1;  // (no keys, so no ranges to deal out)
    KvpDecode P{};
    DecodeParams& p = P.d;
    P.table = table; P.n_pages = n_pages; P.M = max_pages; P.sh_page = log2_of(page); P.n_q = n_q; P.g = g; P.tokens = tokens; P.groups = (int)groups;
    p.Q = (const uint16_t*)Q; p.K = (const uint16_t*)KP; p.V = (const uint16_t*)VP; p.O = (uint16_t*)O; p.LSE = LSE;
    p.B = B; p.Hq = Hq * n_q; p.Hkv = Hkv; p.n_cap = n_cap; p.n_keys = seq_lens ? n_cap : n_keys; p.seq_lens = seq_lens; p.n_splits = n_splits;
    p.g = (int)rows;
    const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)d);
    p.c = scale * kLog2e;
    P.s = scores_of(slopes, score_cap, scale);
    const size_t slots = (size_t)B * Hq * n_q * n_splits;
    p.opart = (float*)workspace; p.pm = p.opart + slots * d; p.lpart = p.pm + slots; p.dealt = (int*)(p.lpart + slots);
    hipStream_t s = (hipStream_t)stream;
    const int n_cu = cu_count() > 0 ? cu_count() : 256;
    (void)hipGetLastError();
    const bool dealt = seq_lens && deals(B, Hkv, n_splits, ceil_div(n_cap, BN), n_cu);
    with_d(d, [&](auto d_c) {
        constexpr int D = decltype(d_c)::value;
        // (dealt out, there are enough ranges for one wave each)
        auto launch = [&](auto halves_c) {
            constexpr bool HALVES = decltype(halves_c)::value;
            const dim3 grid((unsigned)n_splits, (unsigned)B, (unsigned)Hkv);
            if (!seq_lens) kvp_decode_kernel<D, 4, LENS_ONE, false, HALVES><<<grid, 256, 0, s>>>(P);
            else if (dealt) kvp_decode_kernel<D, 1, LENS_DEALT, false, HALVES><<<grid, 64, 0, s>>>(P);
            else kvp_decode_kernel<D, 4, LENS_FIXED, false, HALVES><<<dim3((unsigned)n_splits, (unsigned)Hkv, (unsigned)B), 256, 0, s>>>(P);
        };
        if (grouped) {
            const dim3 grid((unsigned)Hkv, (unsigned)(groups * n_splits), (unsigned)B);
            if (!seq_lens) kvp_decode_kernel<D, 4, LENS_ONE, true, false><<<grid, 256, 0, s>>>(P);
            else if (dealt) kvp_decode_kernel<D, 4, LENS_DEALT, true, false><<<grid, 256, 0, s>>>(P);
            else kvp_decode_kernel<D, 4, LENS_FIXED, true, false><<<grid, 256, 0, s>>>(P);
        } else if (rows <= 16) {
            launch(std::true_type{});
        } else {
            launch(std::false_type{});
        }
        if (n_splits == 1) return;
        const dim3 grid((unsigned)p.Hq, (unsigned)B);
        if (dealt) decode_merge_kernel<D, SLOTS_TABLE, true><<<grid, 256, 0, s>>>(p);
        else decode_merge_kernel<D, SLOTS_FIXED, true><<<grid, 256, 0, s>>>(p);
    });
    return launched();
}

int vfa_row_ranges(const int* doc_offsets, const int* prefix_lens, int* ranges, int B, int N, int n_docs, int causal, void* stream) {
    if (B < 0 || N < 0 || n_docs < 0 || (causal != 0 && causal != 1)) return VFA_ERR_INVALID_ARG;
    if (!aligned4(doc_offsets) || !aligned4(prefix_lens) || !aligned8(ranges)) return VFA_ERR_INVALID_ARG;
    if (B == 0 || N == 0) return VFA_OK;
    if (!doc_offsets || !ranges) return VFA_ERR_INVALID_ARG;
    const long long groups = ((long long)N + 255) / 256;
    if (B > 65535 || n_docs == 0x7fffffff || groups * B > kMaxWorkgroups256) return VFA_ERR_UNSUPPORTED;
    if (!causal) prefix_lens = nullptr;  // (not read: all of a document is seen as it is)
    const RowRanges p{doc_offsets, prefix_lens, reinterpret_cast<int2*>(ranges), N, n_docs, causal};
    (void)hipGetLastError();
    row_ranges_kernel<<<dim3((unsigned)groups, (unsigned)B), 256, 0, (hipStream_t)stream>>>(p);
    return launched();
}

int vfa_masked_attn_fwd(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq, int Hkv, int N, int d, int causal,
                        const int* ranges, float softmax_scale, float score_cap, const float* slopes, void* stream) {
    if (B < 0 || Hq <= 0 || Hkv <= 0 || N < 0 || d <= 0 || Hq % Hkv != 0 || (causal != 0 && causal != 1)) return VFA_ERR_INVALID_ARG;
    if (!isfinite(softmax_scale) || !scale_ok(softmax_scale) || !cap_ok(score_cap)) return VFA_ERR_INVALID_ARG;
    if (d != 64 && d != 128) return VFA_ERR_UNSUPPORTED;
    if (!aligned8(ranges) || !aligned4(slopes) || !aligned4(LSE)) return VFA_ERR_INVALID_ARG;
    if (B == 0 || N == 0) return VFA_OK;
    if (!Q || !K || !V || !O || !aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O)) return VFA_ERR_INVALID_ARG;
    const int n_cu = cu_count() > 0 ? cu_count() : 256;
    const long long heads = (long long)B * Hq;
    const int places = (d == 64 ? 3 : 2) * n_cu;  // workgroups that the units hold
    const bool split = heads * (((long long)N + 127) / 128) < places;
    const long long rows = split ? 64 : 128, blocks = ((long long)N + rows - 1) / rows;
    if ((long long)N * 2 * d > 0x7fffffffLL || heads > 0x7fffffffLL / blocks || heads * blocks > kMaxWorkgroups256) return VFA_ERR_UNSUPPORTED;
    MaskedParams P{};
    Params& p = P.a;
    p.Q = (const uint16_t*)Q; p.K = (const uint16_t*)K; p.V = (const uint16_t*)V; p.O = (uint16_t*)O; p.LSE = LSE;
    p.B = B; p.Hq = Hq; p.Hkv = Hkv; p.N = N; p.Tr = (int)blocks; p.Tc = ceil_div(N, BN); p.causal = causal;
    set_items(p, false);
    const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)d);
    p.c = scale * kLog2e;
    P.s = scores_of(slopes, score_cap, scale);
    P.ranges = reinterpret_cast<const int2*>(ranges);
    if ((B * Hkv) % 8 == 0) {
        P.heads8 = B * Hkv / 8;
        const int parts = (int)max(1LL, heads * blocks / (2 * places));
        P.together = ceil_div(P.heads8, parts);
    }
    const unsigned grid = (unsigned)(heads * blocks);
    (void)hipGetLastError();
    with_d(d, [&](auto d_c) {
        constexpr int D = decltype(d_c)::value;
        hipStream_t s = (hipStream_t)stream;
        auto launch = [&](auto cap_c, auto bias_c) {
            constexpr bool CAP = decltype(cap_c)::value, BIAS = decltype(bias_c)::value;
            if (split) attn_masked_kernel<D, 2, 2, CAP, BIAS><<<grid, 256, 0, s>>>(P);
            else attn_masked_kernel<D, 4, 1, CAP, BIAS><<<grid, 256, 0, s>>>(P);
        };
        using std::false_type, std::true_type;
        if (score_cap > 0.f && slopes) launch(true_type{}, true_type{});
        else if (score_cap > 0.f) launch(true_type{}, false_type{});
        else if (slopes) launch(false_type{}, true_type{});
        else launch(false_type{}, false_type{});
    });
    return launched();
}

}  // extern "C"
