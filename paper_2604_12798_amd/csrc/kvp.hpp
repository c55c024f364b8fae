// The paged cache: pages of bf16 rows found through a table, writing new rows, and where a tile of keys lies.
#pragma once
#include "common.hpp"

namespace {

// ---------------------------------------------------------------------------------------------
// A pool is K, V [n_pages, Hkv, S, D] (S a power of two, 16 or more).  Token n of sequence b lies in page table[b, n / S], row n % S.  An entry
// outside [0, n_pages) is a hole: nothing is written to it and nobody sees its tokens, so that a table may hold anything behind a
// sequence's end, and pages whose tokens are not needed any more can be given back.
struct KvpAppend {
    const uint16_t* X[2];    // new rows of K, V [B, Hkv, n_in, D] with strides (elements)
    long long sb[2], sh[2], sn[2];
    uint16_t* Y[2];          // the pool
    const int* table;        // [B, M]
    const int* old_lens;     // [B] or null
    const int* new_lens;
    int old_len, new_len, n_in, n_pages, M, Hkv, sh_page;  // S = 1 << sh_page
};

// Sixteen bytes of a row are a thread's: loads and the table's entry, which depend on the old length, first, then the stores.  A row of the pool has
// neighbours in its page, so 16 tokens of a head (D = 128) are 4 KiB next to each other on either side.  Memory bounds it: 2 x 16384 tokens of 8 KV heads, 268 MB, 45 us in the kernel
// (58.8 with inputs that come from memory, a copy of as many bytes 53); 16 x 1 tokens 3 us, a launch and three loads that depend on each other.  ONE: a single new row for each sequence, a wave for
// 512 / D of the batch's rows; else 64 lanes x 4 waves take 4 x U x 512 / D tokens of one head.
template <int D, bool ONE>
__global__ __launch_bounds__(ONE ? 64 : 256) void kvp_append_kernel(const KvpAppend p, int rows) {
    constexpr int L = D / 8, U = ONE ? 1 : 4, T = (ONE ? 64 : 256) / L;  // lanes of a row; rounds; rows of a round
    const int c = threadIdx.x % L, r = threadIdx.x / L;
    int b, kv, h, n0;
    if (ONE) {
        const int row = blockIdx.x * T + r;
        if (row >= rows) return;
        h = row % p.Hkv;
        kv = row / p.Hkv & 1;
        b = row / (2 * p.Hkv);
        n0 = 0;
    } else {
        b = blockIdx.z;
        kv = blockIdx.y >= p.Hkv;
        h = blockIdx.y - (kv ? p.Hkv : 0);
        n0 = blockIdx.x * (T * U) + r;
    }
    const long long cap = (long long)p.M << p.sh_page;
    const long long from = p.old_lens ? min(max((long long)p.old_lens[b], 0LL), cap) : p.old_len;
    const long long to = min(p.new_lens ? min((long long)p.new_lens[b], cap) : p.new_len, from + p.n_in);
    const uint16_t* const x = (kv ? p.X[1] : p.X[0]) + b * p.sb[kv] + h * p.sh[kv] + 8 * c;
    uint16_t* const y = kv ? p.Y[1] : p.Y[0];
    u32x4 v[U];
    int page[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = n0 + u * T;
        const bool live = from + i < to;
        page[u] = -1;
        if (live) {
            v[u] = *reinterpret_cast<const u32x4*>(x + (long long)i * p.sn[kv]);
            page[u] = p.table[(size_t)b * p.M + ((from + i) >> p.sh_page)];
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if ((unsigned)page[u] >= (unsigned)p.n_pages) continue;
        const int row = (int)(from + n0 + u * T) & ((1 << p.sh_page) - 1);
        *reinterpret_cast<u32x4*>(y + ((((size_t)page[u] * p.Hkv + h) << p.sh_page) + row) * D + 8 * c) = v[u];
    }
}

// Where a tile of 64 keys lies: its four runs of 16 rows, which no page's end cuts.
struct KvpTile {
    uint64_t off[4];  // bytes from the pool's start
    uint32_t there;   // bit s: run s has a page
};
// The table's entries of a sequence, by scalar loads
typedef const __attribute__((address_space(4))) int* KvpTable;
struct KvpEntries {
    int e[4];
};
__device__ __forceinline__ KvpEntries kvp_entries(KvpTable table, int t, int sh_page, int M) {
    KvpEntries r;
#pragma unroll
    for (int s = 0; s < 4; ++s) r.e[s] = table[min((t * BN + 16 * s) >> sh_page, M - 1)];
    return r;
}
template <int D>
__device__ __forceinline__ KvpTile kvp_tile(const KvpEntries& en, int t, int sh_page, int n_pages, int Hkv, int hkv) {
    KvpTile r;
    r.there = 0;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const bool there = (uint32_t)en.e[s] < (uint32_t)n_pages;
        const uint32_t row = (t * BN + 16 * s) & ((1 << sh_page) - 1);
        r.there |= there ? 1u << s : 0u;
        r.off[s] = there ? ((((uint64_t)(uint32_t)en.e[s] * (uint32_t)Hkv + (uint32_t)hkv) << sh_page) + row) * (2 * D) : 0;
    }
    return r;
}

}  // namespace
