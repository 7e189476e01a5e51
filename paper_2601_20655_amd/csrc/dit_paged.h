// The paged key/value cache: what the kernels that append to it and attend over it are told, and how they find a token's
// request and a key's row.
#pragma once
#include "dit_attn_device.h"

namespace dit {

// n / d for 0 <= n < 2^31 as one high product: with l = ceil(log2 d), m = ceil(2^(31 + l) / d) < 2^32 (for d = 2^l it is
// 2^31), and n m / 2^(31 + l) exceeds n / d by less than n / 2^31 / d.
struct FastDiv {
    uint32_t d, mul;
    int shift;
};
inline FastDiv fast_div(uint32_t d) {
    int l = 0;
    while ((1ull << l) < d) ++l;
    return {d, (uint32_t)(((1ull << (31 + l)) + d - 1) / d), l};
}
__device__ __forceinline__ uint32_t div_by(uint32_t n, const FastDiv& f) { return __umulhi(2u * n, f.mul) >> f.shift; }

// Pages [n_pages][page_size] x heads of D channels; K and V alike.  Strides in units of 16 bytes: a 32-bit number of them
// reaches every row of a cache of up to 64 GiB.
struct PageArgs {
    const int32_t* table;    // [n_requests, max_pages]
    const int32_t* q_start;  // [n_requests + 1]
    const int32_t* kv_len;   // [n_requests]
    int n_requests, max_pages, n_pages;
    uint32_t page16, token16, head16;
    FastDiv page;  // page_size
    int runs;      // 16 tokens from a multiple of 16 on lie in one page, their rows within 2^31 bytes
};

// Tokens of a request that attend: those that are there, that its table has room for, and that a few tiles past the last one still
// have numbers for in 31 bits.
constexpr int kMostKeys = 0x7fff0000;
__device__ __forceinline__ int keys_of(const PageArgs& p, int r) {
    const int64_t room = (int64_t)p.max_pages * p.page.d, most = room < kMostKeys ? room : kMostKeys;
    int n = p.kv_len[r];
    n = n < 0 ? 0 : n;
    return n < most ? n : (int)most;
}

// Request of new token t: the last r with q_start[r] <= t, by the wavefront together, 64 entries at a time; -1: of none.
__device__ __forceinline__ int request_of(const PageArgs& p, int t, int lane) {
    // the answer is among entries lo .. lo + n - 1, or lo is 0 and there is none (unsigned: n is 2^31 at the most)
    const uint32_t entries = (uint32_t)p.n_requests + 1;
    uint32_t lo = 0, n = entries;
    while (true) {
        const uint32_t step = (n + 63) >> 6, mine = (uint32_t)lane * step;
        const uint64_t b = __ballot(mine < n && p.q_start[lo + mine < entries ? lo + mine : entries - 1] <= t);
        if (b == 0) return -1;
        const uint32_t last = 63 - __builtin_clzll(b);
        lo += last * step;
        n = n - last * step < step ? n - last * step : step;
        if (step == 1) break;
    }
    return lo + 1 < entries ? (int)lo : -1;
}

// ---- rows normalised and rotated, to rows or to pages (dit_paged_rows.hip) ----
constexpr int kMostPairs = 64;  // head_dim 128
struct RowTensor {
    const void* x;
    void* y;
    const float* gamma;  // nullable [H D]
    int H;
    int64_t sx_t, sx_h, sy_t, sy_h;
};
struct RowsArgs {
    RowTensor q, k, v;  // H = 0: none.  v: neither normalised nor rotated
    const int32_t* pos;  // nullable [N, 3]
    int N, t0;           // tokens; the first one of this launch
    int x_f32;
    int y_type;          // dit_dtype of the rows of q (and of k where it is no cache)
    int norm;            // 0; 1: over a head; 2: over the token's heads
    float eps;
    int cached;          // k and v go to pages
    int cache_f16;
    PageArgs pages;
    void *k_cache, *v_cache;
    int hd[3];                // pairs per axis
    double turn[kMostPairs];  // turns per unit of position, of every pair
};
hipError_t launch_rows(const RowsArgs& a, int D, hipStream_t s);
// A token's wavefronts (one has four heads at least) are no more than those of a launch of 2^32 work items.
bool rows_heads_fit(int H, int Hk, int Hv);
bool rows_fit(int H, int Hk, int Hv, int D);  // the heads of a token, where the mean is over all of them

// ---- attention over pages (dit_attn_paged.hip) ----
struct PagedAttnArgs {
    const void* q;
    const uint8_t *k_cache, *v_cache;
    void* out;
    float* lse;  // nullable [H, N]
    PageArgs pages;
    int N, H, Hk, G;  // G = H / Hk; N H + n_requests Hk < 2^30: so are all units' numbers
    FastDiv group;    // G
    int64_t sq_t, sq_h, so_t, so_h;
    int q_type, out_type;  // dit_dtype
    int frame, window;
    FastDiv frame_div;  // with a frame
    float scale, scale_log2;  // of the scores; times log2(e)
    // work: tiles of query rows (row = new token * G + head within the group), the keys of a tile in pieces where there are
    // few tiles; requests of fewer than rows_lo or more than rows_hi rows are another launch's
    int rows_lo, rows_hi;
    int pieces;      // work units wanted, per key head; 0: every tile whole
    int pieces_each; // of a tile, as far as the host knows (the joining launch's size goes by it)
    int least;       // key tiles of a piece, at least
    int part_cap;    // tiles' pieces per key head that part_o, part_ml have room for
    float* part_o;   // [Hk][piece][row][D] unnormalised
    float2* part_ml; // [Hk][piece][row]: maximum of the products, sum
};
struct PagedPlan {
    bool few, big;
    int few_qb, few_waves;        // 16-row blocks of a few-row tile; wavefronts of its workgroup
    int big_qb, big_waves;        // 16-row blocks of a wavefront, wavefronts of a many-row tile's workgroup
    int few_units, big_units;     // workgroups
    int few_pieces, big_pieces;   // units wanted per key head; 0: every tile whole
    int few_each, big_each;       // of a tile, as far as is known
    int few_cap, big_cap;
    size_t few_bytes, big_bytes;  // of workspace
};
// How a call is laid over the chip (no device is touched; the host tests read it).  max_q, max_kv: 0 = not known.
PagedPlan plan_paged(int N, int R, int H, int Hk, int D, int64_t max_keys, int max_q, int runs);
hipError_t launch_attn_paged(const PagedAttnArgs& a, const PagedPlan& plan, int D, int op, uint8_t* workspace, hipStream_t s);

}  // namespace dit
