// Attention of chunks of new tokens over a paged key/value cache (gfx950).
//
// For query token i of a request's `new` ones, at place p = kv_len - new + i:
//     out = softmax(scale q K^T over the keys first(p) .. past(p) - 1 whose pages are there) V.
// Rows: the query heads that share a key head are rows of one tile (row = token * G + head in the group), so that each tile
// of keys is read once for all of them.
//
// Scores: S^T(key, row) = K Q^T on v_mfma_f32_16x16x32, 16 keys x 16 rows a block: a lane (i = lane % 16, g = lane / 16) holds
// row i's scores of keys 4g .. 4g+3 of each block.  The rounded probabilities of blocks 2m and 2m + 1 are, as they lie, the
// lane's B operand of O^T += V^T P^T over 32 keys; the matching A operand, eight keys of one channel, comes out of LDS rows of
// V by two transposing reads (ds_read_b64_tr_b16: four rows x 16 channels a group of 16 lanes).  So K and V go from the
// pages to LDS as the rows they are (global_load_lds, 16 bytes a lane), and P never moves between lanes.
#include "dit_paged.h"

#include "../../include/dit_attn.h"
#include "dit_attn_fwd_pipe16.h"

namespace dit {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* ltr_t;

constexpr int kWaitLoads = 0x0f70;  // s_waitcnt vmcnt(0), the other counters at their most
constexpr float kNoScore = -0x1.fffffep127f;  // running maximum of a row that has none (finite: its difference to itself is 0)

// Probabilities are formed times 2^bits, which the division by their sum takes out again (lse and nothing else has to know).  fp16 holds
// numbers from 2^-24 up to 2^16, so that of a row with a large one many small ones would be lost: with as many bits as the kernel's largest
// probability leaves (1 with few rows, 2^8 where a maximum is raised late) those down to 2^-39 or 2^-31 of the row's largest keep
// all or some of theirs, and a smaller one is off by 2^-40 or 2^-32.  bf16 has fp32's range.
template <int OP>
constexpr int prob_bits(bool few) { return OP == OP_F16 ? (few ? 15 : 7) : 0; }

// ---- rows of K and V in LDS ----
// A wavefront-wide load brings 1 KiB: 4 rows of 128 channels or 8 of 64, in lane order.  So that a fragment's read takes each
// bank once, a row's 16-byte pieces lie in an order of the row's own (the order is in which piece a lane fetches), and each
// KiB a little past the one before it: K fragments read one piece of 16 rows, V fragments two neighbouring pieces of 8
// rows (twice).  Orders that exchange pieces among four neighbours (K) or pairs among four (V) leave the rest of a fragment's place to the
// instruction's own offset: one address register for all of K's fragments, four for V's.
template <int D>
struct Rows {
    static constexpr int RB = 2 * D;            // bytes of a row
    static constexpr int PPR = RB / 16;         // pieces of a row
    static constexpr int RPL = 1024 / RB;       // rows of a load
    static constexpr int KG = 1024 + 64, VG = D == 128 ? 1024 + 128 : 1024;  // from a load's rows to the next one's
    static constexpr int k_bytes(int rows) { return rows / RPL * KG; }
    static constexpr int v_bytes(int rows) { return rows / RPL * VG; }
    // which piece the lane with place `slot` of row `row` (of a load's) fetches
    static __device__ __forceinline__ int k_piece(int row, int slot) { return slot ^ (D == 128 ? row & 3 : (row >> 1) & 3); }
    static __device__ __forceinline__ int v_piece(int row, int slot) { return slot ^ (D == 128 ? (row & 3) << 1 : ((row >> 1) & 3) << 1); }
    // where piece `piece` of row `row` lies
    static __device__ __forceinline__ int k_at(int row, int piece) { return row / RPL * KG + row % RPL * RB + 16 * k_piece(row % RPL, piece); }
    static __device__ __forceinline__ int v_at(int row, int piece) { return row / RPL * VG + row % RPL * RB + 16 * v_piece(row % RPL, piece); }
};

// Operand of 16 keys (rows key0 .. +15), channels 32 ks .. +31: the lane's key i, channels 8g .. +7.  k_lane: where the lane
// reads row 0's, ks = 0.
template <int D>
__device__ __forceinline__ int k_lane(int i, int g) { return Rows<D>::k_at(i, g); }
template <int D>
__device__ __forceinline__ u32x4 k_fragment_at(const uint8_t* k, int key0, int ks) {
    return *reinterpret_cast<const u32x4*>(k + key0 / Rows<D>::RPL * Rows<D>::KG + 64 * ks);
}
template <int D>
__device__ __forceinline__ u32x4 k_fragment(const uint8_t* k, int key0, int ks, int i, int g) {
    return k_fragment_at<D>(k + k_lane<D>(i, g), key0, ks);
}
// Operand of 16 channels (16 cb .. +15) and 32 keys (rows key0 .. +31): the lane's channel i, keys 4g .. +3 and 16 + 4g .. +3.
// v_lane: where the lane reads row 0's, of the blocks cb % 4 = c.
template <int D>
__device__ __forceinline__ int v_lane(int c, int i, int g) {
    return Rows<D>::v_at(4 * g + (i >> 2), 2 * c + ((i & 3) >> 1)) + 8 * (i & 1);
}
template <int D>
__device__ __forceinline__ u32x4 v_fragment_at(uint8_t* v, int key0, int cb) {
    uint2 h[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        uint8_t* const p = v + (key0 + 16 * b) / Rows<D>::RPL * Rows<D>::VG + (cb >> 2) * 128;
        h[b] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((ltr_t)p));
    }
    return mk4(h[0].x, h[0].y, h[1].x, h[1].y);
}
template <int D>
__device__ __forceinline__ u32x4 v_fragment(uint8_t* v, int key0, int cb, int i, int g) {
    return v_fragment_at<D>(v + v_lane<D>(cb & 3, i, g), key0, cb);
}

// 16 bytes a lane from base + off (bytes, of the lane) to LDS, lane l's 16 l behind `to`.  (As the instruction and not by the
// compiler's built-in function: for a transposing read behind that one the compiler waits until every such load has landed, as it
// cannot tell whether the read is of what the load writes.  Whoever reads waits for kWaitLoads first.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // m0 is never kept, which is what the warning is about
__device__ __forceinline__ void load_to_lds(const uint8_t* base, uint32_t off, uint8_t* to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :
                 : "s"((uint32_t)(uintptr_t)(lptr_t)to), "v"(off), "s"(base)
                 : "memory", "m0");
}
__device__ __forceinline__ void load_to_lds(const uint8_t* from, uint8_t* to) {  // the lane's own address
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :
                 : "s"((uint32_t)(uintptr_t)(lptr_t)to), "v"(from)
                 : "memory", "m0");
}
#pragma clang diagnostic pop

// ---- which work ----
struct Unit {
    int r;             // request
    int q0, new_;      // its first new token, their number
    int keys;          // its keys
    int tile;          // of query rows
    int piece, pieces; // of its keys
    int slot;          // of the piece, among the key head's
};

// A request as the wavefronts see it.
struct Load {
    int tiles, key_tiles;
};
template <int BQ>
__device__ __forceinline__ Load load_of(const PagedAttnArgs& a, int r, bool live, int& q0, int& n, int& keys) {
    q0 = n = keys = 0;
    if (live) {
        const int s0 = a.pages.q_start[r], s1 = a.pages.q_start[r + 1];
        q0 = s0 < 0 ? 0 : s0 < a.N ? s0 : a.N;
        n = s1 < q0 ? 0 : (s1 < a.N ? s1 : a.N) - q0;
        keys = keys_of(a.pages, r);
    }
    const int64_t rows = (int64_t)n * a.G;
    Load l;
    l.tiles = rows < a.rows_lo || rows > a.rows_hi ? 0 : (int)((rows + BQ - 1) / BQ);
    int64_t most = keys;
    if (a.window) {  // tokens of one tile see no more than this
        const int64_t w = (int64_t)a.window * a.frame + BQ + a.frame;
        most = w < most ? w : most;
    }
    l.key_tiles = (int)((most + kBK - 1) / kBK);
    return l;
}

// Sums of the lanes up to each: within rows of 16 lanes, then row to row (a lane that has no neighbour there adds 0).
template <class T>
__device__ __forceinline__ T scan_add(T x) {
#define DIT_ADD_LANE(ctrl, rows, zero) \
    x += __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl, rows, 0xf, zero))
    DIT_ADD_LANE(0x111, 0xf, true);   // row_shr:1
    DIT_ADD_LANE(0x112, 0xf, true);   // row_shr:2
    DIT_ADD_LANE(0x114, 0xf, true);   // row_shr:4
    DIT_ADD_LANE(0x118, 0xf, true);   // row_shr:8
    DIT_ADD_LANE(0x142, 0xa, false);  // row_bcast:15, to rows 1 and 3
    DIT_ADD_LANE(0x143, 0xc, false);  // row_bcast:31, to rows 2 and 3
#undef DIT_ADD_LANE
    return x;
}

__device__ __forceinline__ int pieces_of(int key_tiles, int c) { return key_tiles <= c ? 1 : (key_tiles + c - 1) / c; }

// What the wavefront's lanes know of 64 requests.
template <int BQ>
struct Requests {
    int q0, n, keys;
    Load l;
    __device__ __forceinline__ void read(const PagedAttnArgs& a, int r0, int lane) {
        l = load_of<BQ>(a, r0 + lane, r0 + lane < a.pages.n_requests, q0, n, keys);
    }
};
template <class T>
__device__ __forceinline__ T sum_of_lanes(T x) {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, scan_add(x)), 63));
}

// The key head's units: `c` key tiles of a piece, at most, units in all, tiles in all.  c is such that all tiles' keys make no
// more than a.pieces units, where there are not more tiles than that already.
struct Units {
    int c, units, tiles;
};
template <int BQ>
__device__ __forceinline__ Units count_units(const PagedAttnArgs& a, const Requests<BQ>& first, int lane) {
    auto total = [&](auto&& of) {
        auto all = of(first);
        if (a.pages.n_requests == 1)
            return __builtin_bit_cast(decltype(all), __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, all)));
        for (int r0 = 64; r0 < a.pages.n_requests; r0 += 64) {
            Requests<BQ> r;
            r.read(a, r0, lane);
            all += of(r);
        }
        return sum_of_lanes(all);
    };
    Units u;
    u.tiles = u.units = total([](const Requests<BQ>& r) { return r.l.tiles; });
    u.c = 0x7fffffff;
    if (!a.pieces || u.tiles >= a.pieces) return u;
    const float keys = total([](const Requests<BQ>& r) { return (float)r.l.tiles * (float)r.l.key_tiles; });
    float c = ceilf(keys / (float)a.pieces);
    c = c < (float)a.least ? (float)a.least : c;
    for (int k = 0; k < 4; ++k) {
        u.c = c < 1e9f ? (int)c : 1000000000;
        u.units = total([&](const Requests<BQ>& r) { return r.l.tiles * pieces_of(r.l.key_tiles, u.c); });
        if (u.units <= a.pieces) break;
        c = ceilf(c * ((float)u.units / (float)a.pieces));
    }
    u.c = __builtin_amdgcn_readfirstlane(u.c);
    return u;
}

// Unit u of a key head's (WHOLE: tile u of its tiles, whatever their pieces): false if there are not so many.
template <int BQ, bool WHOLE>
__device__ __forceinline__ bool find_unit(const PagedAttnArgs& a, const Requests<BQ>& first, int c, int u, int lane, Unit* out) {
    if (a.pages.n_requests == 1) {
        auto of = [&](int x) { return __builtin_amdgcn_readfirstlane(x); };
        const int tiles = of(first.l.tiles), pieces = of(pieces_of(first.l.key_tiles, c));
        if (u >= (WHOLE ? tiles : tiles * pieces)) return false;
        out->r = 0;
        out->q0 = of(first.q0);
        out->new_ = of(first.n);
        out->keys = of(first.keys);
        out->pieces = pieces;
        out->piece = WHOLE || pieces == 1 ? 0 : u / tiles;
        out->tile = u - out->piece * tiles;
        out->slot = u;
        return true;
    }
    int units_before = 0, slots_before = 0;
    for (int r0 = 0; r0 < a.pages.n_requests; r0 += 64) {
        Requests<BQ> r = first;
        if (r0) r.read(a, r0, lane);
        const int pieces = pieces_of(r.l.key_tiles, c);
        const int slots = r.l.tiles * pieces, units = WHOLE ? r.l.tiles : slots;
        const int upto = scan_add(units), slots_upto = WHOLE ? scan_add(slots) : upto;
        const uint64_t b = __ballot(u - units_before < upto);
        if (b) {
            const int at = __builtin_ctzll(b);
            auto of = [&](int x) { return __builtin_amdgcn_readlane(x, at); };
            out->r = r0 + at;
            out->q0 = of(r.q0);
            out->new_ = of(r.n);
            out->keys = of(r.keys);
            out->pieces = of(pieces);
            const int in = u - units_before - (of(upto) - of(units)), tiles = of(r.l.tiles);
            if ((uint32_t)in >= (uint32_t)of(units)) return false;  // (counts that make no sense, of more units than 31 bits hold)
            // pieces of the same keys next to each other
            out->piece = WHOLE ? 0 : in / tiles;
            out->tile = WHOLE ? in : in - out->piece * tiles;
            out->slot = slots_before + of(slots_upto) - of(slots) + in;
            return true;
        }
        units_before += __builtin_amdgcn_readlane(upto, 63);
        slots_before += __builtin_amdgcn_readlane(slots_upto, 63);
    }
    return false;
}

// The n-th of a workgroup's units: workgroups go round the eight XCDs, each of which gets a run of neighbouring units, that
// is of the same head's keys.  -1: none left.
__device__ __forceinline__ int nth_unit(int total, int n) {
    const uint32_t run = ((uint32_t)total + 7) / 8, at = (blockIdx.x >> 3) + (uint32_t)n * (gridDim.x >> 3);
    if (at >= run) return -1;
    const uint32_t u = (blockIdx.x & 7) * run + at;
    return u < (uint32_t)total ? (int)u : -1;
}

// Keys [first, past) that the token at place p sees of `keys`.
__device__ __forceinline__ void seen_by(const PagedAttnArgs& a, int64_t p, int keys, int& first, int& past) {
    first = 0;
    past = keys;
    if (a.frame) {
        const int64_t f = p >= 0 ? (int64_t)div_by((uint32_t)p, a.frame_div) : -1;
        const int64_t end = (f + 1) * a.frame;
        past = end < keys ? (int)end : keys;
        if (a.window) {
            const int64_t begin = (f - a.window + 1) * a.frame;
            first = begin < 0 ? 0 : begin < keys ? (int)begin : keys;
        }
    }
}

// ---- keys' rows ----
// Lane l's key of a tile: its row's place in the cache in units of 16 bytes, and whether there is one.
struct KeyRow {
    uint32_t off16;
    bool there;
};
__device__ __forceinline__ int entry_of(const PageArgs& p, const int32_t* table, int key, int keys) {  // keys > 0
    const int n = key < 0 ? 0 : key < keys ? key : keys - 1;
    return table[div_by((uint32_t)n, p.page)];
}
__device__ __forceinline__ KeyRow row_of(const PageArgs& p, int entry, int key, int keys) {
    const int n = key < 0 ? 0 : key < keys ? key : keys - 1;
    const uint32_t in = (uint32_t)n - div_by((uint32_t)n, p.page) * p.page.d;
    KeyRow k;
    k.there = (uint32_t)key < (uint32_t)keys && entry >= 0 && entry < p.n_pages;
    k.off16 = (uint32_t)entry * p.page16 + in * p.token16;
    return k;
}

// ---- query rows ----
// Rounded to the cache's type where theirs is another: a product of the matrix cores has two operands of one 16-bit type, and a second part
// (what the rounding leaves) would double the scores' products.
__device__ __forceinline__ u32x4 load_q(const void* q, int64_t off, int type, int op) {
    if (type == (op == OP_F16 ? DIT_F16 : DIT_BF16)) return *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(q) + off);
    float x[8];
    if (type == DIT_F16) {
        const f16x8 h = *reinterpret_cast<const f16x8*>(static_cast<const uint16_t*>(q) + off);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)h[e];
    } else {
        load8(q, off, type == DIT_F32, x);
    }
    return op == OP_F16 ? pack8<OP_F16>(x) : pack8<OP_BF16>(x);
}

__device__ __forceinline__ void store4(void* out, int64_t off, int type, f32x4 v) {
    if (type == DIT_F32) *reinterpret_cast<f32x4*>(static_cast<float*>(out) + off) = v;
    else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + off) = make_uint2(pack2<OP_BF16>(v[0], v[1]), pack2<OP_BF16>(v[2], v[3]));
}

// The probabilities of a tile in which some keys are masked for some rows, times rows of V of which some hold an infinity or a
// NaN: 0 times those is no 0, so the masked ones are left out one by one, on the vector ALU.  (Rare: such values in such a
// tile only.)  keep: bit b of the lane's mask = its row sees key 16 (b / 4) + 4 g + b % 4 of the 32.
template <int D, int OP, class Acc>
__device__ __forceinline__ void pv_one_by_one(const uint8_t* v, const uint32_t (&P)[4], uint32_t keep, Acc&& O, int i, int g) {
#pragma unroll 1
    for (int key = 0; key < 32; ++key) {
        // the lane that holds row i's probability of this key, and where
        const int b = 4 * (key >> 4) + (key & 3), from = ((key & 15) >> 2) * 16 + i;
        uint32_t pair = P[0];
#pragma unroll
        for (int w = 1; w < 4; ++w) pair = w == (b >> 1) ? P[w] : pair;
        pair = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * from, (int)pair);
        const uint32_t k = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * from, (int)keep);
        const uint32_t bits = (b & 1) ? pair >> 16 : pair & 0xffffu;
        const float p = OP == OP_F16 ? (float)__builtin_bit_cast(f16x2, bits)[0] : __uint_as_float(bits << 16);
        const bool ok = (k >> b) & 1;
#pragma unroll
        for (int cb = 0; cb < D / 16; ++cb) {
            const uint2 raw = *reinterpret_cast<const uint2*>(v + Rows<D>::v_at(key, 2 * cb + (g >> 1)) + 8 * (g & 1));
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint32_t u = r < 2 ? raw.x : raw.y;
                const float x = OP == OP_F16 ? (float)__builtin_bit_cast(f16x2, u)[r & 1] : (r & 1) ? bf16_hi(u) : bf16_lo(u);
                O(cb, r, [&](float o) { return ok ? fmaf(p, x, o) : o; });
            }
        }
    }
}
// Whether a pair of 16-bit numbers holds an infinity or a NaN.
template <int OP>
__device__ __forceinline__ bool pair_not_finite(uint32_t u) {
    constexpr uint32_t e = OP == OP_F16 ? 0x7c00u : 0x7f80u;
    return (u & e) == e || ((u >> 16) & e) == e;
}

// One wavefront's rows: 16 QB of them, and what it has of their softmax.
template <int D, int QB>
struct RowState {
    f32x4 O[QB][D / 16];
    float m[QB], l[QB];  // of the lane's row i; l: the lane's own keys
    int first[QB], past[QB];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int q = 0; q < QB; ++q) {
            m[q] = kNoScore;
            l[q] = 0.f;
#pragma unroll
            for (int cb = 0; cb < D / 16; ++cb) O[q][cb] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
};

// 32 keys: scores, softmax, O += P V.  P is rounded to the cache's type, V's, as the matrix cores take it (what a second part of P
// would cost is as many products again); its sums are of the unrounded ones.  kf(f), vf(cb): their fragments.  MASKED: `there` (bit
// = the key's page is there) and the rows' ranges leave some out, and vt is where V's rows lie in LDS.
template <int D, int OP, int QB, bool MASKED, class KF, class VF>
__device__ __forceinline__ void block_step(RowState<D, QB>& st, const u32x4 (&Q)[QB][D / 32], KF&& kf, VF&& vf, const uint8_t* vt,
                                           int key0, uint32_t there, float scale_log2, int i, int g) {
    constexpr int NKS = D / 32, NCB = D / 16;
    f32x4 S[QB][2];
    uint32_t keep[QB];
#pragma unroll
    for (int f = 0; f < 2 * NKS; ++f) {
        const u32x4 k = kf(f);
#pragma unroll
        for (int q = 0; q < QB; ++q) {
            const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
            S[q][f & 1] = mfma16<OP>(k, Q[q][f >> 1], f < 2 ? zero : S[q][f & 1]);
        }
    }
#pragma unroll
    for (int q = 0; q < QB; ++q) {
        if constexpr (MASKED) {
            keep[q] = 0;
            const uint32_t mine = there >> (4 * g);
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int key = key0 + 16 * b + 4 * g + r;
                    const bool ok = ((mine >> (16 * b + r)) & 1) && key >= st.first[q] && key < st.past[q];
                    keep[q] |= (ok ? 1u : 0u) << (4 * b + r);
                    S[q][b][r] = ok ? S[q][b][r] : -INFINITY;
                }
        }
    }
    uint32_t P[QB][4];
#pragma unroll
    for (int q = 0; q < QB; ++q) {
        float mx = S[q][0][0];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) mx = fmaxf(mx, S[q][b][r]);
        mx = fmaxf(max_across_rows16(mx), st.m[q]);
        if (__any(mx > st.m[q])) {
            const float alpha = __builtin_amdgcn_exp2f((st.m[q] - mx) * scale_log2);
            st.l[q] *= alpha;
#pragma unroll
            for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
                for (int r = 0; r < 4; ++r) st.O[q][cb][r] *= alpha;
            st.m[q] = mx;
        }
        // (s - m) c (+ bits) as one fma(s, c, -m c).  -m c is rounded: by 2^-13 at most below 2^12; beyond, where it would be by more
        // than an exponent holds, the difference is taken first.
        constexpr float bits = prob_bits<OP>(true);
        float off = fmaf(-mx, scale_log2, bits);
        if (__any(__builtin_fabsf(off) > 4096.0f)) {
            off = bits;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[q][b][r] -= mx;
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            float e[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                e[r] = __builtin_amdgcn_exp2f(fmaf(S[q][b][r], scale_log2, off));
                st.l[q] += e[r];
            }
            P[q][2 * b] = pack2<OP>(e[0], e[1]);
            P[q][2 * b + 1] = pack2<OP>(e[2], e[3]);
        }
    }
    if constexpr (MASKED) {
        bool bad = false;
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb) {
            const u32x4 v = vf(cb);
#pragma unroll
            for (int w = 0; w < 4; ++w) bad = bad || pair_not_finite<OP>(v[w]);
        }
        if (__any(bad)) {
#pragma unroll
            for (int q = 0; q < QB; ++q)
                pv_one_by_one<D, OP>(vt, P[q], keep[q], [&](int cb, int r, auto&& add) { st.O[q][cb][r] = add(st.O[q][cb][r]); }, i, g);
            return;
        }
    }
#pragma unroll
    for (int cb = 0; cb < NCB; ++cb) {
        const u32x4 v = vf(cb);
#pragma unroll
        for (int q = 0; q < QB; ++q) st.O[q][cb] = mfma16<OP>(v, mk4(P[q][0], P[q][1], P[q][2], P[q][3]), st.O[q][cb]);
    }
}

// Query rows of a wavefront: 16 QB from `row0` of the unit's; rows past the end are the last one again, and not stored.
struct RowPlace {
    int token, head;  // token counted from the request's first new one
    bool live;
};
__device__ __forceinline__ RowPlace place_of(const PagedAttnArgs& a, const Unit& u, int hk, int64_t row) {
    const int64_t rows = (int64_t)u.new_ * a.G;
    RowPlace p;
    p.live = row < rows;
    const uint32_t n = (uint32_t)(p.live ? row : rows - 1);
    const uint32_t t = div_by(n, a.group);
    p.token = (int)t;
    p.head = hk * a.G + (int)(n - t * a.G);
    return p;
}

template <int D, int OP, int QB>
__device__ __forceinline__ void load_rows(const PagedAttnArgs& a, const Unit& u, int hk, int64_t row0, int i, int g,
                                          u32x4 (&Q)[QB][D / 32], RowState<D, QB>& st) {
#pragma unroll
    for (int q = 0; q < QB; ++q) {
        const RowPlace p = place_of(a, u, hk, row0 + 16 * q + i);
        const int64_t off = (int64_t)(u.q0 + p.token) * a.sq_t + (int64_t)p.head * a.sq_h + 8 * g;
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) Q[q][ks] = load_q(a.q, off + 32 * ks, a.q_type, OP);
        seen_by(a, (int64_t)u.keys - u.new_ + p.token, u.keys, st.first[q], st.past[q]);
    }
}

// Channel blocks cb0 .. of row `row` out: normalised, or (a tile in pieces) as they are with their maximum (of the products, not
// scaled) and sum.  l: summed over the row's lanes.  at_tile: the row's place in its tile.  bits: as of prob_bits.
template <int N>
__device__ __forceinline__ void store_blocks(const PagedAttnArgs& a, const Unit& u, int hk, int D, int rows_of_tile, int at_tile, int64_t row,
                                             int g, int cb0, const f32x4 (&O)[N], float m, float l, int bits) {
    const RowPlace p = place_of(a, u, hk, row);
    if (!p.live) return;
    if (u.pieces > 1) {
        if (u.slot >= a.part_cap) return;
        const int64_t at = ((int64_t)hk * a.part_cap + u.slot) * rows_of_tile + at_tile;
        float* const o = a.part_o + at * D + 16 * cb0 + 4 * g;
#pragma unroll
        for (int cb = 0; cb < N; ++cb) *reinterpret_cast<f32x4*>(o + 16 * cb) = O[cb];
        if (g == 0 && cb0 == 0) a.part_ml[at] = make_float2(m, l);
        return;
    }
    const float inv = l > 0.f || l != l ? 1.0f / l : 0.f;
    const int64_t off = (int64_t)(u.q0 + p.token) * a.so_t + (int64_t)p.head * a.so_h + 16 * cb0 + 4 * g;
#pragma unroll
    for (int cb = 0; cb < N; ++cb) {
        f32x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = O[cb][r] * inv;
        store4(a.out, off + 16 * cb, a.out_type, v);
    }
    if (a.lse && g == 0 && cb0 == 0)
        a.lse[(int64_t)p.head * a.N + u.q0 + p.token] = (m * a.scale_log2 + (__builtin_amdgcn_logf(l) - (float)bits)) * 0.6931471805599453f;
}

// Key tiles of the unit: from the first key that its first token sees to the last that its last token sees, and of those its
// piece.
template <int BQ>
__device__ __forceinline__ void key_tiles_of(const PagedAttnArgs& a, const Unit& u, int& begin, int& end) {
    const int64_t rows = (int64_t)u.new_ * a.G, row0 = (int64_t)u.tile * BQ;
    const int64_t row1 = row0 + BQ < rows ? row0 + BQ - 1 : rows - 1;
    const int64_t place = (int64_t)u.keys - u.new_;
    int lo, hi, none;
    seen_by(a, place + div_by((uint32_t)row0, a.group), u.keys, lo, none);
    seen_by(a, place + div_by((uint32_t)row1, a.group), u.keys, none, hi);
    const int b = lo / kBK, e = hi > lo ? (hi + kBK - 1) / kBK : b;
    begin = b;
    end = e;
    if (u.pieces > 1) {  // (the first ones a tile longer than the rest)
        const int each = (int)((uint32_t)(e - b) / (uint32_t)u.pieces), rest = (e - b) - each * u.pieces;
        begin = b + u.piece * each + (u.piece < rest ? u.piece : rest);
        end = begin + each + (u.piece < rest ? 1 : 0);
    }
}

// ---- few rows: each wavefront of a workgroup has keys of its own ----
// 16 QB rows; the unit's keys go to the NW wavefronts 32 at a time, each of which has LDS of its own for 32 rows of K and V.
// Memory bounds it: a wavefront reads its fragments into registers as soon as the rows have landed, and asks for the next ones
// before it multiplies.  Two workgroups of 4 wavefronts a compute unit, or one of 8 (where there are few: half as many keys one
// after the other), keep up to 128 KiB on their way.  Their results are joined in LDS.  Measured, one new token a request: 40 heads with
// keys of their own x 32,760 keys 114 us = 5.9 TB/s, 32 requests of 16 to 8,190 keys x 8 key heads 104 us = 5.2 TB/s, 8 key heads x 257 keys
// 9.9 (counts, page, rows, products, join and store one after the other; 11.6 where one wavefront joined and stored).  Of 128 channels the
// 32-row form fills all 256 vector registers and spills 35 to 45 (16 rows: 181 to 200, none).
template <int D, int NW>
constexpr int few_lds() { return NW * (Rows<D>::k_bytes(32) + Rows<D>::v_bytes(32)); }

template <int D, int OP, int QB, bool RUNS, int NW>
__global__ void __launch_bounds__(64 * NW, 2) attn_paged_few_kernel(const PagedAttnArgs a) {
    using R = Rows<D>;
    constexpr int BQ = 16 * QB, KEYS = 32, RPI = R::RPL, NL = KEYS / RPI, NKF = D / 16, NCB = D / 16;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint8_t* const kt = smem + wave * (R::k_bytes(KEYS) + R::v_bytes(KEYS));
    uint8_t* const vt = kt + R::k_bytes(KEYS);
    Requests<BQ> requests;
    requests.read(a, 0, lane);
    const Units all = count_units<BQ>(a, requests, lane);
    const int per_head = all.units, total = per_head * a.Hk;
    for (int n = 0;; ++n) {
        const int id = nth_unit(total, n);
        if (id < 0) return;
        const int hk = id / per_head;
        Unit u;
        if (!find_unit<BQ, false>(a, requests, all.c, id - hk * per_head, lane, &u)) return;
        int begin, end;
        key_tiles_of<BQ>(a, u, begin, end);
        const int32_t* const table = a.pages.table + (int64_t)u.r * a.pages.max_pages;
        const uint8_t* const kc = a.k_cache + (int64_t)hk * a.pages.head16 * 16;
        const uint8_t* const vc = a.v_cache + (int64_t)hk * a.pages.head16 * 16;
        // the wavefront's blocks of 32 keys: from b on, every NW-th
        int b = 2 * begin + wave;
        const int blocks = 2 * end;
        // RUNS: lane x knows where run x % 2 (16 keys) of the wavefront's block x / 2 from `first` on begins; else lane x knows row x
        // of block `first`, and asks for the page of the next one.
        int first = b, entry = 0;
        uint32_t off16 = 0, there = 0;  // there: of the block fetched last
        uint64_t ok = 0;
        auto locate = [&](int block) {
            first = block;
            const int key = RUNS ? KEYS * (block + NW * (lane >> 1)) + 16 * (lane & 1) : KEYS * block + (lane & 31);
            if (RUNS) entry = entry_of(a.pages, table, key, u.keys);
            const KeyRow kr = row_of(a.pages, entry, key, u.keys);
            ok = __ballot(kr.there);
            off16 = kr.off16;
            if (!RUNS) entry = entry_of(a.pages, table, key + KEYS * NW, u.keys);
        };
        auto fetch = [&](int block) {
            if (!RUNS || block - first >= 32 * NW) locate(block);
            const int at = RUNS ? (block - first) / NW * 2 : 0;
            const int left = u.keys - KEYS * block;
            there = RUNS ? ((uint32_t)(ok >> at) & 1 ? 0xffffu : 0u) | ((uint32_t)(ok >> at) & 2 ? 0xffff0000u : 0u) : (uint32_t)ok;
            there = left >= KEYS ? there : left <= 0 ? 0u : there & ((1u << left) - 1);
            const int in = lane / R::PPR, slot = lane % R::PPR;
            const uint32_t kp = 16 * R::k_piece(in, slot), vp = 16 * R::v_piece(in, slot);
            const bool whole = there == 0xffffffffu;
            if constexpr (RUNS) {
                const uint32_t row = 16 * a.pages.token16;
#pragma unroll
                for (int run = 0; run < 2; ++run) {
                    const uint64_t from = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)off16, at + run) * 16;
#pragma unroll
                    for (int x = 0; x < NL / 2; ++x) {
                        const int p = run * (NL / 2) + x;
                        if (whole || ((there >> (p * RPI + in)) & 1)) {
                            load_to_lds(kc + from + x * RPI * row, in * row + kp, kt + p * R::KG);
                            load_to_lds(vc + from + x * RPI * row, in * row + vp, vt + p * R::VG);
                        } else {
                            *reinterpret_cast<u32x4*>(kt + p * R::KG + 16 * lane) = mk4(0, 0, 0, 0);
                            *reinterpret_cast<u32x4*>(vt + p * R::VG + 16 * lane) = mk4(0, 0, 0, 0);
                        }
                    }
                }
            } else {
                uint32_t at_row[NL];
#pragma unroll
                for (int p = 0; p < NL; ++p) at_row[p] = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (p * RPI + in), (int)off16);
#pragma unroll
                for (int p = 0; p < NL; ++p) {
                    if (whole || ((there >> (p * RPI + in)) & 1)) {
                        load_to_lds(kc + kp + (uint64_t)at_row[p] * 16, kt + p * R::KG);
                        load_to_lds(vc + vp + (uint64_t)at_row[p] * 16, vt + p * R::VG);
                    } else {
                        *reinterpret_cast<u32x4*>(kt + p * R::KG + 16 * lane) = mk4(0, 0, 0, 0);
                        *reinterpret_cast<u32x4*>(vt + p * R::VG + 16 * lane) = mk4(0, 0, 0, 0);
                    }
                }
            }
        };
        if (b < blocks) {
            if (!RUNS) entry = entry_of(a.pages, table, KEYS * b + (lane & 31), u.keys);
            if (RUNS) locate(b);
            fetch(b);
        }
        RowState<D, QB> st;
        u32x4 Q[QB][D / 32];
        const int64_t row0 = (int64_t)u.tile * BQ;
        load_rows<D, OP, QB>(a, u, hk, row0, i, g, Q, st);
        st.clear();
        int lo = 0, hi = 0x7fffffff;  // keys that every row sees
#pragma unroll
        for (int q = 0; q < QB; ++q) {
            lo = max(lo, st.first[q]);
            hi = min(hi, st.past[q]);
        }
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) {
            lo = max(lo, __shfl_xor(lo, d));
            hi = min(hi, __shfl_xor(hi, d));
        }
        lo = __builtin_amdgcn_readfirstlane(lo);
        hi = __builtin_amdgcn_readfirstlane(hi);
        for (; b < blocks; b += NW) {
            __builtin_amdgcn_s_waitcnt(0);  // (its own rows: no other wavefront waits for them)
            const int key0 = KEYS * b;
            const uint32_t t = there;
            const bool more = b + NW < blocks;
            if (t != 0xffffffffu || key0 < lo || key0 + KEYS > hi) {
                if (t) {
                    int ln = lane;
                    asm volatile("" : "+v"(ln));  // (see opaque_lane in the other kernel)
                    const int i = ln & 15, g = ln >> 4;
                    block_step<D, OP, QB, true>(
                        st, Q, [&](int f) { return k_fragment<D>(kt, 16 * (f & 1), f >> 1, i, g); },
                        [&](int cb) { return v_fragment<D>(vt, 0, cb, i, g); }, vt, key0, t, a.scale_log2, i, g);
                }
                __builtin_amdgcn_s_waitcnt(0);
                if (more) fetch(b + NW);
                continue;
            }
            u32x4 kf[NKF], vf[NCB];
#pragma unroll
            for (int f = 0; f < NKF; ++f) kf[f] = k_fragment<D>(kt, 16 * (f & 1), f >> 1, i, g);
#pragma unroll
            for (int cb = 0; cb < NCB; ++cb) vf[cb] = v_fragment<D>(vt, 0, cb, i, g);
            __builtin_amdgcn_s_waitcnt(0);
            __builtin_amdgcn_sched_barrier(0);
            if (more) fetch(b + NW);
            __builtin_amdgcn_sched_barrier(0);
            block_step<D, OP, QB, false>(st, Q, [&](int f) { return kf[f]; }, [&](int cb) { return vf[cb]; }, vt, key0, t,
                                         a.scale_log2, i, g);
        }
        // the wavefronts' rows: maxima, then sums and O relative to the largest
        float l[QB];
        __syncthreads();
        float2* const ml = reinterpret_cast<float2*>(smem);  // [wave][row]
#pragma unroll
        for (int q = 0; q < QB; ++q) {
            l[q] = sum_across_rows16(st.l[q]);
            if (g == 0) ml[wave * BQ + 16 * q + i] = make_float2(st.m[q], l[q]);
        }
        __syncthreads();
        float f[QB];
#pragma unroll
        for (int q = 0; q < QB; ++q) {
            float2 x[NW];
            float top = kNoScore;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                x[w] = ml[w * BQ + 16 * q + i];
                top = fmaxf(top, x[w].x);
            }
            l[q] = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) l[q] += x[w].y * __builtin_amdgcn_exp2f((x[w].x - top) * a.scale_log2);
            f[q] = __builtin_amdgcn_exp2f((st.m[q] - top) * a.scale_log2);
            st.m[q] = top;
        }
        // O: every wavefront leaves its own, and adds up all of them, in order, of channel blocks of its own
        constexpr int NB = D / 16 < NW ? 1 : D / 16 / NW;
        static_assert(2048 + NW * D * 64 <= few_lds<D, NW>() && NW * BQ * 8 <= 2048, "room for the results");
        float* const area = reinterpret_cast<float*>(smem + 2048);  // [wave][channel block][lane][4]
        const int cb0 = wave * NB;
#pragma unroll
        for (int q = 0; q < QB; ++q) {
            // (a block of 16 rows at a time: D / 16 pieces of 1 KiB a wavefront)
            if (q > 0) __syncthreads();
#pragma unroll
            for (int cb = 0; cb < D / 16; ++cb) {
#pragma unroll
                for (int r = 0; r < 4; ++r) st.O[q][cb][r] *= f[q];
                *reinterpret_cast<f32x4*>(area + ((wave * (D / 16) + cb) * 64 + lane) * 4) = st.O[q][cb];
            }
            __syncthreads();
            if (cb0 < D / 16) {
                f32x4 sum[NB];
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int w = 0; w < NW; ++w) {
                        const f32x4 x = *reinterpret_cast<const f32x4*>(area + ((w * (D / 16) + cb0 + n) * 64 + lane) * 4);
#pragma unroll
                        for (int r = 0; r < 4; ++r) sum[n][r] = w ? sum[n][r] + x[r] : x[r];
                    }
                store_blocks(a, u, hk, D, BQ, 16 * q + i, row0 + 16 * q + i, g, cb0, sum, st.m[q], l[q], prob_bits<OP>(true));
            }
        }
        __syncthreads();
    }
}

// ---- many rows: the wavefronts of a workgroup share the keys ----
// 16 QB rows a wavefront, NW wavefronts: 128 rows and two workgroups a compute unit (4 x 32), or 256 and one (8 x 32: half the bytes
// from L2 to LDS, and nothing under a tile's ends).  The matrix cores and the vector ALU hardly work at the same time here: a
// loop of 16x16x32 products with n vector instructions behind each takes about 17 + 3.3 n clocks, two wavefronts or one; so what
// counts is the sum, 32 products and 64 vector instructions (16 of them exponentials, 8 clocks each) a half, and the
// power that random operands take (zeros: 2.5 ms where these take 3.1).  4,680 rows x 32,760 keys at 40 heads of 128 (frame-wise, 2.99e12
// operations): 3.13 ms by 4 x 32, 2.90 by 8 x 32 (1,030 TFLOP/s), 3.70 where rows lie anywhere (8 x 16, below); fragments read 2, 4,
// 6 or 8 ahead, other priorities: level.  Software-pipelined in halves of a tile, 32 keys: while the
// matrix cores work on a half's scores the vector ALU takes the exponentials of the half before it, and while they multiply
// those with V it takes the maxima of the new scores.  So a half's scores are needed one half ahead of its V, and a turn of the
// loop, which multiplies V of tile j, takes K rows 32 keys on: K(j) in LDS is rows 64 j + 32 .. 64 j + 95.  K(j + 1) and V(j + 1) are
// on their way meanwhile.  A row's maximum is raised only where a score tops it by more than 2^8 (exponents stay far from their
// ends, and what divides the row takes it out again).
template <int D>
constexpr int big_buffers() { return 2 * (Rows<D>::k_bytes(kBK) + Rows<D>::v_bytes(kBK)); }
// Rows that lie anywhere: the places of sixteen tiles' rows, and which of them are there, twice.
constexpr int kPlaceTiles = 16, kPlaceBytes = kPlaceTiles * (kBK * 4 + 8);
template <int D, bool RUNS>
constexpr int big_lds() { return big_buffers<D>() + (RUNS ? 0 : 2 * kPlaceBytes); }

// RUNS: 16 tokens from a multiple of 16 on lie in one page, so that a wavefront's rows of a part start at one place.
template <int D, int OP, bool RUNS, int NW, int QB>
__global__ void __launch_bounds__(64 * NW, 2) attn_paged_big_kernel(const PagedAttnArgs a) {
    using R = Rows<D>;
    constexpr int BQ = 16 * QB * NW;
    constexpr int RW = kBK / NW, RPI = R::RPL, NL = RW / RPI;  // rows that a wavefront fetches of a part, rows a load, loads
    constexpr int NKS = D / 32, NCB = D / 16, NOG = NCB / 4, NKF = 2 * NKS;
    constexpr int LA = 4;        // fragments are read from LDS so many ahead of their products
    constexpr int NCH = 4 * QB;  // slices of two scores
    constexpr int PRE = NCH > 2 * NKF ? NCH / NKF : 2;       // exponentials run so many slices ahead of their rounding
    static_assert(LA <= NKF && LA <= NCB && PRE >= NCH / NKF, "look-ahead within a half");
    extern __shared__ __attribute__((aligned(16))) uint8_t dyn[];
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Requests<BQ> requests;
    requests.read(a, 0, lane);
    const Units all = count_units<BQ>(a, requests, lane);
    const int per_head = all.units, total = per_head * a.Hk;
    const float scale = a.scale_log2, thr = kRescaleThr / scale;
    constexpr float bits = prob_bits<OP>(false);
    static_assert(kRescaleThr + prob_bits<OP>(false) <= 15 || OP != OP_F16, "the largest probability is an fp16 number");
    // K buffers 0 and 1, then V's
    auto kbuf = [&](int b) { return dyn + b * R::k_bytes(kBK); };
    auto vbuf = [&](int b) { return dyn + 2 * R::k_bytes(kBK) + b * R::v_bytes(kBK); };
    // (In what runs for masked tiles only, all that hangs on the lane's number is worked out from one that the compiler cannot
    // see through: left to itself it works it out ahead of the loop, and then has no registers for the loop.)
    auto opaque_lane = [&]() {
        int x = lane;
        asm volatile("" : "+v"(x));
        return x;
    };
    for (int n = 0;; ++n) {
        const int id = nth_unit(total, n);
        if (id < 0) return;
        const int hk = id / per_head;
        Unit u;
        if (!find_unit<BQ, false>(a, requests, all.c, id - hk * per_head, lane, &u)) return;
        u32x4 Q[QB][NKS];
        f32x16 O[NOG][QB];
        // scores: quarter 2 (q % 2) + kb of word q / 2 = row block q, keys 16 kb .. of the half
        typedef f32x16 scores_t[(QB + 1) / 2];
        scores_t S0, S1;
        float m[QB], top[QB], off[QB];  // maximum, what a score has to top to raise it, what its exponent is short of
        float l[QB][2];                 // sums, of every other key of the lane's
        int lo = 0, hi = 0x7fffffff;  // keys that every row of the wavefront sees
        const int64_t row0 = (int64_t)u.tile * BQ + wave * 16 * QB;
        {
            RowState<D, QB> st;
            load_rows<D, OP, QB>(a, u, hk, row0, i, g, Q, st);
#pragma unroll
            for (int q = 0; q < QB; ++q) {
                lo = max(lo, st.first[q]);
                hi = min(hi, st.past[q]);
                m[q] = kNoScore;
                top[q] = kNoScore + thr;
                off[q] = -kNoScore * scale;
                l[q][0] = l[q][1] = 0.f;
#pragma unroll
                for (int og = 0; og < NOG; ++og)
#pragma unroll
                    for (int r = 0; r < 16; ++r) O[og][q][r] = 0.f;
            }
        }
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) {
            lo = max(lo, __shfl_xor(lo, d));
            hi = min(hi, __shfl_xor(hi, d));
        }
        lo = __builtin_amdgcn_readfirstlane(lo);
        hi = __builtin_amdgcn_readfirstlane(hi);
        int begin, end;
        key_tiles_of<BQ>(a, u, begin, end);
        const int32_t* const table = a.pages.table + (int64_t)u.r * a.pages.max_pages;
        const uint8_t* const kc = a.k_cache + (int64_t)hk * a.pages.head16 * 16;
        const uint8_t* const vc = a.v_cache + (int64_t)hk * a.pages.head16 * 16;

        // ---- where rows of K and V are ----
        // Of sixteen tiles at a time, from first_tile on; a turn needs its tile and the two behind it.  RUNS: lane x has run x % 4 (16
        // keys) of tile first_tile + x / 4: the place of its first row, and in `ok` whether its page is there; the pages of the sixteen
        // tiles behind the next turn but thirteen are asked for meanwhile.  Else the places of all rows are in LDS, written by all
        // wavefronts in turns, and `ok` has a bit for each tile all of which is there.  (In registers, two rows a lane, they pushed the
        // query rows of the 2 x 128 kernel into scratch memory, whose reloads wait for the keys on their way: 13.4 ms; in LDS, 5.9, of
        // which a wavefront of one row block has no spills at all: 3.7.)
        constexpr int kTurns = kPlaceTiles - 2;
        int first_tile = 0, entry = 0, half = 0;
        uint32_t off_a = 0;
        uint64_t ok = 0;
        auto places = [&]() { return reinterpret_cast<uint32_t*>(dyn + big_buffers<D>() + half * kPlaceBytes); };
        auto rows_there = [&]() { return reinterpret_cast<uint64_t*>(places() + kPlaceTiles * kBK); };
        auto ask = [&](int tile) { return entry_of(a.pages, table, kBK * tile + 16 * lane, u.keys); };
        auto place_rows = [&]() {
            const int lane = opaque_lane();
            int e[kPlaceTiles / NW];
#pragma unroll
            for (int x = 0; x < kPlaceTiles / NW; ++x) e[x] = entry_of(a.pages, table, kBK * (first_tile + wave + NW * x) + lane, u.keys);
#pragma unroll
            for (int x = 0; x < kPlaceTiles / NW; ++x) {
                const int tile = wave + NW * x;
                const KeyRow kr = row_of(a.pages, e[x], kBK * (first_tile + tile) + lane, u.keys);
                places()[kBK * tile + lane] = kr.off16;
                const uint64_t there = __ballot(kr.there);
                if (lane == 0) rows_there()[tile] = there;
            }
        };
        auto arrived = [&](int tile) {  // behind the barrier that follows step_to
            if (!RUNS && tile == first_tile) ok = __ballot(rows_there()[opaque_lane() & (kPlaceTiles - 1)] == ~0ull);
        };
        auto start_at = [&](int tile) {
            first_tile = tile;
            if constexpr (RUNS) {
                const KeyRow kr = row_of(a.pages, ask(tile), kBK * tile + 16 * lane, u.keys);
                ok = __ballot(kr.there);
                off_a = kr.off16;
                entry = ask(tile + kTurns);
            } else {
                place_rows();
                __syncthreads();
                arrived(tile);
            }
        };
        auto step_to = [&](int tile) {  // tile: the next turn's
            if (tile - first_tile < kTurns) return;
            first_tile = tile;
            if constexpr (RUNS) {
                const KeyRow kr = row_of(a.pages, entry, kBK * tile + 16 * lane, u.keys);
                ok = __ballot(kr.there);
                off_a = kr.off16;
                entry = ask(tile + kTurns);
            } else {
                half ^= 1;  // (others may be reading this half still)
                place_rows();
            }
        };
        // bit r: key r of the tile j + n is there (n = 0, 1, 2)
        auto there_of = [&](int j, int n) -> uint64_t {
            if constexpr (RUNS) {
                const uint32_t runs = (uint32_t)(ok >> (4 * (j + n - first_tile))) & 15u;
                uint64_t x = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) x |= (runs >> k) & 1u ? 0xffffull << (16 * k) : 0ull;
                const int left = u.keys - kBK * (j + n);
                return left >= kBK ? x : left <= 0 ? 0ull : x & ((1ull << left) - 1);
            } else {
                const uint64_t x = rows_there()[j + n - first_tile];
                return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
            }
        };
        auto pages_there = [&](int j) -> bool {  // of tiles j .. j + 2, whole ones
            if constexpr (RUNS) return ((uint32_t)(ok >> (4 * (j - first_tile))) & 0xfffu) == 0xfffu;
            else return ((uint32_t)(ok >> (j - first_tile)) & 7u) == 7u;
        };
        // This wavefront's rows of a part of tile j + 1's turn, from row `from` of the tile on (0, or for K 32: past its end the next
        // tile's follow).  whole: all of them are there.
        auto fetch_part = [&](int lane, const uint8_t* cache, uint8_t* buf, int j, int from, bool v, auto whole)
            __attribute__((always_inline)) {
            const int row_l = lane / R::PPR, slot_l = lane % R::PPR, first = RW * wave + from;
            const uint32_t piece = 16 * (v ? R::v_piece(row_l, slot_l) : R::k_piece(row_l, slot_l));
            uint8_t* const dst = buf + wave * NL * (v ? R::VG : R::KG);
            const uint64_t there = whole ? ~0ull : first < kBK ? there_of(j, 1) >> first : there_of(j, 2) >> (first - kBK);
            if constexpr (RUNS) {
                const uint8_t* src = cache + (uint64_t)(uint32_t)__builtin_amdgcn_readlane(
                                                 (int)off_a, 4 * (j + 1 - first_tile) + first / 16) * 16;
                const uint32_t row = 16 * a.pages.token16, in = (row_l + first % 16) * row + piece;
#pragma unroll
                for (int p = 0; p < NL; ++p) {
                    uint8_t* const to = dst + p * (v ? R::VG : R::KG);
                    if (whole || ((there >> (p * RPI + row_l)) & 1)) load_to_lds(src + p * RPI * row, in, to);
                    else *reinterpret_cast<u32x4*>(to + 16 * lane) = mk4(0, 0, 0, 0);
                }
            } else {
                const uint32_t* const from_row = places() + kBK * (j + 1 - first_tile) + first + row_l;
                uint32_t at[NL];
#pragma unroll
                for (int p = 0; p < NL; ++p) at[p] = from_row[p * RPI];
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int p = 0; p < NL; ++p) {
                    uint8_t* const to = dst + p * (v ? R::VG : R::KG);
                    if (whole || ((there >> (p * RPI + row_l)) & 1)) load_to_lds(cache + piece + (uint64_t)at[p] * 16, to);
                    else *reinterpret_cast<u32x4*>(to + 16 * lane) = mk4(0, 0, 0, 0);
                }
            }
        };
        // K and V of tile j + 1's turn: V's rows are the tile's, K's its second half and the first of the next one
        auto fetch = [&](int lane, int j, int b, auto whole) __attribute__((always_inline)) {
            fetch_part(lane, kc, kbuf(b), j, 32, false, whole);
            fetch_part(lane, vc, vbuf(b), j, 0, true, whole);
        };
        auto landed = [&](int tile) {
            __builtin_amdgcn_s_waitcnt(kWaitLoads);
            __syncthreads();
            arrived(tile);
        };

        auto is_masked = [&](int tile, uint64_t there) { return there != ~0ull || kBK * tile < lo || kBK * tile + kBK > hi; };
        // bit 4 kb + r: the lane's row q sees key key0 + 16 kb + 4 g + r; there: bits of the half's keys
        auto keep_of = [&](int q, int key0, uint32_t there) {
            const int ln = opaque_lane(), g = ln >> 4;
            int first, past;
            seen_by(a, (int64_t)u.keys - u.new_ + place_of(a, u, hk, row0 + 16 * q + (ln & 15)).token, u.keys, first, past);
            const uint32_t mine = there >> (4 * g);
            uint32_t k = 0;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int key = key0 + 16 * kb + 4 * g + r;
                    k |= (((mine >> (16 * kb + r)) & 1) && key >= first && key < past ? 1u : 0u) << (4 * kb + r);
                }
            return k;
        };
        bool far = false;  // a row's maximum is too large for (s - m) c in one fma (see block_step)
        auto raise = [&](scores_t& S) {
            far = false;
#pragma unroll
            for (int q = 0; q < QB; ++q) {
                float mx = S[q / 2][8 * (q % 2)];
#pragma unroll
                for (int e = 1; e < 8; ++e) mx = fmaxf(mx, S[q / 2][8 * (q % 2) + e]);
                mx = max_across_rows16(mx);
                const float to = mx > top[q] ? mx : m[q];
                const float alpha = __builtin_amdgcn_exp2f((m[q] - to) * scale);
                m[q] = to;
                // (a large one's sum is rounded, by as much as thr: more than fp16 has room for)
                top[q] = OP == OP_F16 && __builtin_fabsf(to * scale) > 4096.0f ? to : to + thr;
                off[q] = OP == OP_F16 ? fmaf(-to, scale, bits) : -to * scale;
                l[q][0] *= alpha;
                l[q][1] *= alpha;
                far = far || (to != kNoScore && __builtin_fabsf(off[q]) > 4096.0f);
#pragma unroll
                for (int og = 0; og < NOG; ++og)
#pragma unroll
                    for (int r = 0; r < 16; ++r) O[og][q][r] *= alpha;
            }
            far = __any(far);
        };
        // A half's scores of such rows: the difference first.  (off is that of the half: the next raise, or this again, sets it anew.)
        auto take_maxima = [&](scores_t& S) {
#pragma unroll
            for (int q = 0; q < QB; ++q) {
                const bool some = m[q] != kNoScore;
                off[q] = some ? bits : off[q];
#pragma unroll
                for (int e = 0; e < 8; ++e) S[q / 2][8 * (q % 2) + e] -= some ? m[q] : 0.f;
            }
        };
        // slice x = (q, w): word w of the operand of the half's keys for row block q
        auto exp_slice = [&](scores_t& S, int x) {
            const int q = x / 4, e = 2 * (x % 8);
            S[q / 2][e] = __builtin_amdgcn_exp2f(fmaf(S[q / 2][e], scale, off[q]));
            S[q / 2][e + 1] = __builtin_amdgcn_exp2f(fmaf(S[q / 2][e + 1], scale, off[q]));
        };
        auto pack_slice = [&](scores_t& S, uint32_t (&P)[QB][4], int x) {
            const int q = x / 4, e = 2 * (x % 8);
            P[q][x % 4] = pack2<OP>(S[q / 2][e], S[q / 2][e + 1]);
            l[q][0] += S[q / 2][e];
            l[q][1] += S[q / 2][e + 1];
        };
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        auto score = [&](u32x4 k, int f, int q, scores_t& S) {
            const int ks = f >> 1, kb = f & 1;
            const int at = 2 * (q % 2) + kb;
            S[q / 2] = ks == 0 ? mfma16_q_init<OP>(k, Q[q][ks], zero, S[q / 2], at) : mfma16_q<OP>(k, Q[q][ks], S[q / 2], at);
        };
        auto product = [&](u32x4 v, const uint32_t (&P)[QB][4], int cb, int q) {
            O[cb / 4][q] = mfma16_q<OP>(v, mk4(P[q][0], P[q][1], P[q][2], P[q][3]), O[cb / 4][q], cb % 4);
        };

        // One half (its scores in Sc) and the next one's scores (into Sn), no key of either masked for any row.  kn: the next one's
        // rows of K, vb: this one's of V
        // (the lane's own addresses in them).
        auto plain_half = [&](scores_t& Sc, scores_t& Sn, const uint8_t* kn, uint8_t* const (&vb)[4], auto half) __attribute__((always_inline)) {
            constexpr int H = decltype(half)::value;
            u32x4 kf[NKF], vf[NCB];
            auto k_frag = [&](int f) { return k_fragment_at<D>(kn, 32 * H + 16 * (f & 1), f >> 1); };
            auto v_frag = [&](int v) { return v_fragment_at<D>(vb[v & 3], 32 * H, v); };
#pragma unroll
            for (int f = 0; f < LA; ++f) kf[f] = k_frag(f);
            uint32_t P[QB][4];
#pragma unroll
            for (int x = 0; x < PRE; ++x) exp_slice(Sc, x);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int f = 0; f < NKF; ++f) {
                if (f + LA < NKF) kf[f + LA] = k_frag(f + LA);
                if (f >= NKF - LA) vf[f - (NKF - LA)] = v_frag(f - (NKF - LA));
#pragma unroll
                for (int q = 0; q < (QB + 1) / 2; ++q) score(kf[f], f, q, Sn);
#pragma unroll
                for (int x = f * NCH / NKF; x < (f + 1) * NCH / NKF; ++x)
                    if (x + PRE < NCH) exp_slice(Sc, x + PRE);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int q = (QB + 1) / 2; q < QB; ++q) score(kf[f], f, q, Sn);
#pragma unroll
                for (int x = f * NCH / NKF; x < (f + 1) * NCH / NKF; ++x) pack_slice(Sc, P, x);
                __builtin_amdgcn_sched_barrier(0);
            }
            float mx[QB];
#pragma unroll
            for (int q = 0; q < QB; ++q) mx[q] = -INFINITY;
            auto max_slice = [&](int x) {
                const int q = x % QB, e = 8 * (q % 2) + 2 * (x / QB);
                mx[q] = max3(mx[q], Sn[q / 2][e], Sn[q / 2][e + 1]);
            };
#pragma unroll
            for (int v = 0; v < NCB; ++v) {
                if (v + LA < NCB) vf[v + LA] = v_frag(v + LA);
#pragma unroll
                for (int q = 0; q < (QB + 1) / 2; ++q) product(vf[v], P, v, q);
                if (v >= 1) {
#pragma unroll
                    for (int x = (v - 1) * NCH / NCB; x < v * NCH / NCB; ++x) max_slice(x);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int q = (QB + 1) / 2; q < QB; ++q) product(vf[v], P, v, q);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int x = (NCB - 1) * NCH / NCB; x < NCH; ++x) max_slice(x);
            bool above = false;
#pragma unroll
            for (int q = 0; q < QB; ++q) above = above || mx[q] > top[q];
            if (__any(above)) raise(Sn);
        };

        // One half, whatever is masked of it, and the next one's scores (if there is one) into the same registers.
        auto any_half = [&](scores_t& S, bool masked, int key0, uint32_t there, uint8_t* vb, bool more, bool masked_next, uint32_t there_next,
                            const uint8_t* kn) __attribute__((always_inline)) {
            const int ln = opaque_lane(), i = ln & 15, g = ln >> 4;
            if (far) take_maxima(S);
#pragma unroll
            for (int q = 0; q < QB; ++q) off[q] = fminf(off[q], -kNoScore);  // (a row without a score: all exponents are to be -infinity)
            uint32_t P[QB][4];
#pragma unroll
            for (int x = 0; x < NCH; ++x) exp_slice(S, x);
#pragma unroll
            for (int x = 0; x < NCH; ++x) pack_slice(S, P, x);
            bool bad = false;
            if (masked) {
#pragma unroll
                for (int v = 0; v < NCB; ++v) {
                    const u32x4 x = v_fragment<D>(vb, 0, v, i, g);
#pragma unroll
                    for (int w = 0; w < 4; ++w) bad = bad || pair_not_finite<OP>(x[w]);
                }
            }
            if (__any(bad)) {
#pragma unroll
                for (int q = 0; q < QB; ++q)
                    pv_one_by_one<D, OP>(vb, P[q], keep_of(q, key0, there), [&](int cb, int r, auto&& add) {
                        O[cb / 4][q][4 * (cb % 4) + r] = add(O[cb / 4][q][4 * (cb % 4) + r]);
                    }, i, g);
            } else {
#pragma unroll
                for (int v = 0; v < NCB; ++v) {
                    const u32x4 x = v_fragment<D>(vb, 0, v, i, g);
#pragma unroll
                    for (int q = 0; q < QB; ++q) product(x, P, v, q);
                }
            }
            if (!more) return;
#pragma unroll
            for (int f = 0; f < NKF; ++f) {
                const u32x4 k = k_fragment<D>(kn, 16 * (f & 1), f >> 1, i, g);
#pragma unroll
                for (int q = 0; q < QB; ++q) score(k, f, q, S);
            }
            if (masked_next) {
#pragma unroll
                for (int q = 0; q < QB; ++q) {
                    const uint32_t k = keep_of(q, key0 + 32, there_next);
#pragma unroll
                    for (int e = 0; e < 8; ++e) S[q / 2][8 * (q % 2) + e] = (k >> e) & 1 ? S[q / 2][8 * (q % 2) + e] : -INFINITY;
                }
            }
            raise(S);
        };

        if (begin < end) {
            constexpr std::integral_constant<bool, true> whole{};
            constexpr std::integral_constant<bool, false> some{};
            constexpr int KH = R::k_bytes(32), VH = R::v_bytes(32);  // a half's bytes
            // as if tile begin - 1's turn were over: the first half's rows of K, in the other buffer's second half, and the first turn's
            int j = begin - 1;
            start_at(j);
            if (wave < NW / 2) fetch_part(lane, kc, kbuf(1) + KH, j, 0, false, some);
            fetch(lane, j, 0, some);
            j = begin;
            step_to(j);
            landed(j);
            // keys [key0, key0 + 32) of which the lane's rows see some, those of the half whose scores S are
            auto mask = [&](scores_t& S, int key0, uint32_t there) {
#pragma unroll
                for (int q = 0; q < QB; ++q) {
                    const uint32_t k = keep_of(q, key0, there);
#pragma unroll
                    for (int e = 0; e < 8; ++e) S[q / 2][8 * (q % 2) + e] = (k >> e) & 1 ? S[q / 2][8 * (q % 2) + e] : -INFINITY;
                }
            };
            const uint64_t there_0 = there_of(j, 0);
#pragma unroll
            for (int f = 0; f < NKF; ++f) {
                const u32x4 k = k_fragment<D>(kbuf(1) + KH, 16 * (f & 1), f >> 1, i, g);
#pragma unroll
                for (int q = 0; q < QB; ++q) score(k, f, q, S0);
            }
            if (is_masked(begin, there_0)) mask(S0, kBK * begin, (uint32_t)there_0);
            raise(S0);
            __syncthreads();  // (all have read the first half, whose place K(begin + 1) takes)
            int b = 0;  // buffers of tile j
            while (true) {
                const int ln = opaque_lane();  // (what the loop reads is worked out here, not spilled and read back)
                const int k_l = k_lane<D>(ln & 15, ln >> 4);
                int v_l[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) v_l[x] = v_lane<D>(x, ln & 15, ln >> 4);
                // Turns in which neither the tiles that are used nor what is fetched meanwhile holds a masked key.
                while (j + 2 < end && !far && kBK * j >= lo && kBK * j + 2 * kBK <= hi && pages_there(j)) {
                    fetch(RUNS ? ln : opaque_lane(), j, b ^ 1, whole);
                    const uint8_t* const kl = kbuf(b) + k_l;
                    uint8_t* vl[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) vl[x] = vbuf(b) + v_l[x];
                    plain_half(S0, S1, kl, vl, std::integral_constant<int, 0>{});
                    if (far) take_maxima(S1);  // (since the half before; the turn's end leaves the loop)
                    plain_half(S1, S0, kl, vl, std::integral_constant<int, 1>{});
                    ++j;
                    b ^= 1;
                    step_to(j);
                    landed(j);
                }
                const bool more = j + 1 < end;
                if (more) fetch(opaque_lane(), j, b ^ 1, some);
                const uint64_t t0 = there_of(j, 0), t1 = there_of(j, 1);
                const bool m0 = is_masked(j, t0), m1 = is_masked(j + 1, t1);
                any_half(S0, m0, kBK * j, (uint32_t)t0, vbuf(b), true, m0, (uint32_t)(t0 >> 32), kbuf(b));
                any_half(S0, m0, kBK * j + 32, (uint32_t)(t0 >> 32), vbuf(b) + VH, more, m1, (uint32_t)t1, kbuf(b) + KH);
                if (!more) break;
                ++j;
                b ^= 1;
                step_to(j);
                landed(j);
            }
        }
#pragma unroll
        for (int q = 0; q < QB; ++q) {
            f32x4 o[NCB];
#pragma unroll
            for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[cb][r] = O[cb / 4][q][4 * (cb % 4) + r];
            store_blocks(a, u, hk, D, BQ, (wave * QB + q) * 16 + i, row0 + 16 * q + i, g, 0, o, m[q], sum_across_rows16(l[q][0] + l[q][1]),
                         prob_bits<OP>(false));
        }
        __syncthreads();
    }
}

// ---- tiles in pieces put together ----
// D / 4 lanes a row, four channels each, in one pass: UN pieces at a time, all that is read of them asked for before any is used.  A
// piece's weight is of its maximum's difference, taken before the scale (their products differ by a rounding each, 2^-24 of themselves).
// 1,560 x 12 rows of 128 channels in three pieces 10.2 us, 40 rows in five 5.4 (a wavefront a row: 14.0, 7.5).
template <int D, int BQ, int UN>
__global__ void __launch_bounds__(256) attn_paged_join_kernel(const PagedAttnArgs a, int bits) {
    constexpr int LANES = D / 4, PER = 256 / LANES, PARTS = BQ / PER;  // of a row, rows of a workgroup, workgroups of a tile
    const int lane = threadIdx.x & 63;
    Requests<BQ> requests;
    requests.read(a, 0, lane);
    const Units all = count_units<BQ>(a, requests, lane);
    const int per_head = all.tiles;
    const int64_t total = (int64_t)per_head * a.Hk * PARTS;
    for (int64_t id = blockIdx.x; id < total; id += gridDim.x) {
        const int tile_id = (int)(id / PARTS), part = (int)(id % PARTS), hk = tile_id / per_head;
        Unit u;
        if (!find_unit<BQ, true>(a, requests, all.c, tile_id - hk * per_head, lane, &u)) return;
        // piece s of the tile is tiles-of-the-request slots behind piece s - 1; u.slot counts from the request's first
        const int64_t rows = (int64_t)u.new_ * a.G, row0 = (int64_t)u.tile * BQ;
        const int tiles = (int)((rows + BQ - 1) / BQ);
        if (u.pieces < 2 || u.slot + (u.pieces - 1) * tiles >= a.part_cap) continue;
        const int row = part * PER + threadIdx.x / LANES, ch = threadIdx.x % LANES * 4;
        const RowPlace p = place_of(a, u, hk, row0 + row);
        if (!p.live) continue;
        const int64_t first = ((int64_t)hk * a.part_cap + u.slot) * BQ + row, step = (int64_t)tiles * BQ;
        float top = kNoScore, sum = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < u.pieces; s += UN) {
            float2 ml[UN];
            f32x4 x[UN];
#pragma unroll
            for (int e = 0; e < UN; ++e) {
                const int64_t at = first + (s + e < u.pieces ? s + e : u.pieces - 1) * step;
                ml[e] = a.part_ml[at];
                x[e] = *reinterpret_cast<const f32x4*>(a.part_o + at * D + ch);
            }
            float m = top;
#pragma unroll
            for (int e = 0; e < UN; ++e) m = fmaxf(m, ml[e].x);
            const float before = __builtin_amdgcn_exp2f((top - m) * a.scale_log2);
            top = m;
            sum *= before;
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] *= before;
#pragma unroll
            for (int e = 0; e < UN; ++e) {
                if (s + e >= u.pieces) break;
                const float w = __builtin_amdgcn_exp2f((ml[e].x - m) * a.scale_log2);
                sum = fmaf(ml[e].y, w, sum);
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r] = fmaf(x[e][r], w, o[r]);
            }
        }
        const float inv = sum > 0.f || sum != sum ? 1.0f / sum : 0.f;
        store4(a.out, (int64_t)(u.q0 + p.token) * a.so_t + (int64_t)p.head * a.so_h + ch, a.out_type,
               f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv});
        if (a.lse && ch == 0)
            a.lse[(int64_t)p.head * a.N + u.q0 + p.token] = (top * a.scale_log2 + (__builtin_amdgcn_logf(sum) - (float)bits)) * 0.6931471805599453f;
    }
}
// Its launch, for so many tiles as are known of.
template <int D, int BQ, int UN>
hipError_t launch_join(const PagedAttnArgs& a, int units, int bits, hipStream_t s) {
    const int64_t n = (int64_t)units / a.pieces_each * (BQ * D / 1024);
    hipLaunchKernelGGL((attn_paged_join_kernel<D, BQ, UN>), dim3((unsigned)(n < 1 ? 1 : n < 65536 ? n : 65536)), dim3(256), 0, s, a, bits);
    return hipGetLastError();
}

template <int D, int OP, int QB, bool RUNS, int NW>
hipError_t launch_few_n(const PagedAttnArgs& a, int units, hipStream_t s) {
    static std::atomic<uint64_t> done{0};
    const auto kern = attn_paged_few_kernel<D, OP, QB, RUNS, NW>;
    constexpr int lds = few_lds<D, NW>();
    hipError_t e = allow_dynamic_lds(kern, lds, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((units + 7) / 8 * 8), dim3(64 * NW), lds, s, a);
    return hipGetLastError();
}
template <int D, int OP, int QB>
hipError_t launch_few(const PagedAttnArgs& a, int units, int nw, hipStream_t s) {
    hipError_t e;
    if (nw == 8) e = a.pages.runs ? launch_few_n<D, OP, QB, true, 8>(a, units, s) : launch_few_n<D, OP, QB, false, 8>(a, units, s);
    else e = a.pages.runs ? launch_few_n<D, OP, QB, true, 4>(a, units, s) : launch_few_n<D, OP, QB, false, 4>(a, units, s);
    return e != hipSuccess || !a.pieces ? e : launch_join<D, 16 * QB, 8>(a, units, prob_bits<OP>(true), s);
}
template <int D, int OP, bool RUNS, int NW, int QB>
hipError_t launch_big_n(const PagedAttnArgs& a, int units, hipStream_t s) {
    static std::atomic<uint64_t> done{0};
    const auto kern = attn_paged_big_kernel<D, OP, RUNS, NW, QB>;
    constexpr int lds = big_lds<D, RUNS>();
    hipError_t e = allow_dynamic_lds(kern, lds, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((units + 7) / 8 * 8), dim3(64 * NW), lds, s, a);
    e = hipGetLastError();
    return e != hipSuccess || !a.pieces ? e : launch_join<D, 16 * QB * NW, 4>(a, units, prob_bits<OP>(false), s);
}
template <int D, int OP>
hipError_t launch_big(const PagedAttnArgs& a, const PagedPlan& plan, hipStream_t s) {
    const int units = plan.big_units;
    if constexpr (D == 128) {
        if (!a.pages.runs) return launch_big_n<D, OP, false, 8, 1>(a, units, s);
    } else {
        if (!a.pages.runs)
            return plan.big_waves == 8 ? launch_big_n<D, OP, false, 8, 2>(a, units, s) : launch_big_n<D, OP, false, 4, 2>(a, units, s);
    }
    return plan.big_waves == 8 ? launch_big_n<D, OP, true, 8, 2>(a, units, s) : launch_big_n<D, OP, true, 4, 2>(a, units, s);
}

constexpr int kFewRows = 64;  // of a request, by the kernel for few
template <int D, int OP>
hipError_t launch_paged(const PagedAttnArgs& args, const PagedPlan& plan, uint8_t* ws, hipStream_t s) {
    PagedAttnArgs a = args;
    auto parts = [&](int pieces, int each, int cap, int rows) {
        a.pieces = pieces;
        a.pieces_each = each;
        a.part_cap = cap;
        a.part_o = reinterpret_cast<float*>(ws);
        a.part_ml = reinterpret_cast<float2*>(ws + (size_t)a.Hk * cap * rows * D * sizeof(float));
    };
    hipError_t e = hipSuccess;
    if (plan.few) {
        a.rows_lo = 1;
        a.rows_hi = plan.big ? kFewRows : 0x7fffffff;
        a.least = 2;
        parts(plan.few_pieces, plan.few_each, plan.few_cap, 16 * plan.few_qb);
        e = plan.few_qb == 1 ? launch_few<D, OP, 1>(a, plan.few_units, plan.few_waves, s) : launch_few<D, OP, 2>(a, plan.few_units, plan.few_waves, s);
    }
    if (e == hipSuccess && plan.big) {
        a.rows_lo = plan.few ? kFewRows + 1 : 1;
        a.rows_hi = 0x7fffffff;
        a.least = 4;
        ws += plan.few_bytes;
        parts(plan.big_pieces, plan.big_each, plan.big_cap, 16 * plan.big_qb * plan.big_waves);
        e = launch_big<D, OP>(a, plan, s);
    }
    return e;
}

}  // namespace

PagedPlan plan_paged(int N, int R, int H, int Hk, int D, int64_t max_keys, int max_q, int runs) {
    PagedPlan p{};
    const int64_t G = H / Hk, rows = (int64_t)N * G, some = N < R ? N : R;  // requests with a new token
    const int64_t most_q = max_q > 0 && max_q < N ? max_q : N;              // new tokens of a request
    p.few_qb = most_q * G > 16 ? 2 : 1;
    const bool uniform = most_q * some <= 2 * (int64_t)N;  // few requests have far fewer new tokens than that
    // (33 to 64 rows, by 32-row tiles and by those of many rows: 1 to 16 requests, 1,024 to 8,192 keys 31 and 40 us, 34 and 44, 41 and
    // 48; 80 rows 64 and 49)
    p.few = most_q * G <= kFewRows || !uniform;
    p.big = most_q * G > kFewRows;
    const int64_t key_tiles = max_keys > 0 ? (max_keys + kBK - 1) / kBK : 1;
    // Time in key tiles of one of two 4-wavefront workgroups of a compute unit: rounds of workgroups (`slots` at a time), each as long as
    // its keys (`step` a tile, `alone` where a compute unit has no second workgroup) and its two ends; tiles in pieces need the launch
    // that joins them, and room.  The constants are those under which, of 42 calls (1 to 4,680 new tokens, 257 to 100,000 keys, 1 to 256
    // requests, measured in every layout), the layout chosen is the fastest or up to 9 % from it; bytes bound the few-row kernel, so
    // that its steps are short against its ends.
    struct Costs {
        int BQ;
        int64_t slots;
        double step, alone, ends;
        int least;
        double join, room;  // once, and for 10^6 numbers
        bool even;          // of several requests, whose lengths may differ: fill the slots where pieces have 48 tiles left
    };
    struct Layout {
        double time;
        int units, pieces, each, cap;
        size_t bytes;
    };
    auto layout = [&](const Costs& c) {
        const int BQ = c.BQ;
        // tiles of a key head: at most (whatever q_start says, with what is left over of each request), and as far as is known
        const int64_t most = (rows + some * (BQ - 1)) / BQ;
        const int64_t each = (most_q * G + BQ - 1) / BQ, tiles = some * each < most ? some * each : most;
        auto time = [&](int n) {
            const int64_t units = tiles * Hk * n, rounds = units / c.slots, rest = units % c.slots;
            const double keys = (double)((key_tiles + n - 1) / n);
            return (double)rounds * (c.step * keys + c.ends) + (rest ? (rest > kCUs ? c.step : c.alone) * keys + c.ends : 0.0) +
                   (n > 1 ? c.join + c.room * 1e-6 * (double)(units * BQ * D) : 0.0);
        };
        int best = 1;
        // (one new token each, 16 to 8,190 keys: with 2 x 4,096 110 us, else 123)
        auto room = [&](int n) { return (tiles * n + most) * Hk * BQ <= (int64_t)1 << 19; };  // rows of pieces: 272 MB at head_dim 128
        while (c.even && some > 1 && tiles * Hk * best < c.slots && key_tiles >= 48 * (best + 1) && room(best + 1)) ++best;
        double least = time(best);
        for (int n = best + 1; n <= 64 && n * (int64_t)c.least <= key_tiles; ++n) {
            if (!room(n)) break;
            const double t = time(n);
            if (t >= 0.97 * least) continue;
            best = n;
            least = t;
        }
        Layout l{least, 0, 0, best, 0, 0};
        if (best > 1) {
            l.pieces = (int)(tiles * best);
            l.cap = (int)(tiles * best + most);
            l.bytes = ((size_t)Hk * l.cap * BQ * (D * sizeof(float) + sizeof(float2)) + 255) / 256 * 256;
        }
        const int64_t n = tiles * Hk * best;
        l.units = (int)(n < 65536 ? n : 65536);
        return l;
    };
    if (p.few) {
        const Layout four = layout({16 * p.few_qb, 2 * kCUs, 1.0, 0.25, 49.0, 2, 1.9, 0.006, true});
        const Layout eight = layout({16 * p.few_qb, kCUs, 0.09, 0.09, 57.0, 4, 1.9, 0.006, false});
        // (whole tiles, no more of them than compute units: 257 keys x 40/8 heads 10.7 us by 8 wavefronts, 11.0 by 4; 700 x 40 13.5, 14.1)
        const bool wide = (some == 1 && eight.time < four.time) || (four.each == 1 && eight.each == 1 && four.units <= kCUs);
        const Layout& l = wide ? eight : four;
        p.few_waves = wide ? 8 : 4;
        p.few_units = l.units;
        p.few_pieces = l.pieces;
        p.few_each = l.each;
        p.few_cap = l.cap;
        p.few_bytes = l.bytes;
    }
    if (p.big) {
        const bool one = D == 128 && !runs;  // a row block a wavefront
        const Layout four = layout(one ? Costs{128, kCUs, 0.62, 0.62, 12.0, 4, 4.0, 0.011, false} : Costs{128, 2 * kCUs, 1.0, 0.53, 7.0, 4, 4.0, 0.011, false});
        const Layout eight = layout({256, kCUs, 0.7, 0.7, 41.0, 4, 4.0, 0.011, false});
        const bool wide = !one && eight.time < four.time;
        const Layout& l = wide ? eight : four;
        p.big_waves = one || wide ? 8 : 4;
        p.big_qb = one ? 1 : 2;
        p.big_units = l.units;
        p.big_pieces = l.pieces;
        p.big_each = l.each;
        p.big_cap = l.cap;
        p.big_bytes = l.bytes;
    }
    return p;
}

hipError_t launch_attn_paged(const PagedAttnArgs& a, const PagedPlan& plan, int D, int op, uint8_t* workspace, hipStream_t s) {
    if (D == 128) return op == OP_F16 ? launch_paged<128, OP_F16>(a, plan, workspace, s) : launch_paged<128, OP_BF16>(a, plan, workspace, s);
    return op == OP_F16 ? launch_paged<64, OP_F16>(a, plan, workspace, s) : launch_paged<64, OP_BF16>(a, plan, workspace, s);
}

}  // namespace dit
