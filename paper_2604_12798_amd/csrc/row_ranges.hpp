// The keys that each row of a packed batch sees.
#pragma once
#include "common.hpp"

namespace {

// ---------------------------------------------------------------------------------------------
// Document k of an entry is [o_k, o_(k+1)); its row i sees the keys from o_k to its end, or, causal, to itself or to the end of the document's prefix, whichever
// is later.  A row's document is the last one that begins at or before it (a search among the offsets, which go through LDS 1024 at a time);
// rows outside of all of them see nothing.  (16384 rows of 24 documents 2.5 us, 64 x 2048 of one 2.6: a launch and a load; the search is eight reads of LDS.)
struct RowRanges {
    const int* offsets;  // [B, n_docs + 1]
    const int* prefix;   // [B, n_docs] or null
    int2* out;           // [B, N]
    int N, n_docs, causal;
};

__global__ __launch_bounds__(256) void row_ranges_kernel(const RowRanges p) {
    constexpr int CHUNK = 1024;
    __shared__ int o[CHUNK];
    const int b = blockIdx.y, tid = threadIdx.x, n = p.n_docs + 1;
    const long long i = (long long)blockIdx.x * 256 + tid;
    const int* const off = p.offsets + (size_t)b * n;
    auto clamped = [&](int x) { return min(max(x, 0), p.N); };
    int at = 0;  // offsets at or before the row
    for (int c0 = 0; c0 < n; c0 += CHUNK) {
        const int have = min(CHUNK, n - c0);
        __syncthreads();
        for (int k = tid; k < have; k += 256) o[k] = clamped(off[c0 + k]);
        __syncthreads();
        int lo = 0, hi = have;  // offsets [0, lo) are at or before the row, those from hi on behind it
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (o[mid] <= i) lo = mid + 1;
            else hi = mid;
        }
        at += lo;
    }
    if (i >= p.N) return;
    int2 r = {0, 0};
    if (at > 0 && at < n) {  // (at = n: behind the last document)
        const int from = clamped(off[at - 1]), to = clamped(off[at]);
        const int reach = p.prefix ? (int)min((long long)from + p.prefix[(size_t)b * p.n_docs + at - 1], (long long)to) : from;
        r = int2{from, p.causal ? max((int)i + 1, reach) : to};
    }
    p.out[(size_t)b * p.N + i] = r;
}

}  // namespace
