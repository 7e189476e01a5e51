// Rows of q and k, RMS-normalised and rotated by positions that are given for each token, to rows or (k, with v) to the pages of
// a cache.
//
//   y = rotate(x * gamma / sqrt(mean(x^2) + eps)),  pair i of axis a by the angle pos_a * base^(-2i / d_a).
//
// A lane holds eight channels, i.e. four pairs, of a head; the heads that a wavefront takes have those channels at the same
// place, so that their four angles are worked out once a wavefront.  An angle is a number of turns: the position times the
// pair's turns per position, in 64 bits, of which the whole turns are dropped before it becomes a 32-bit number.
//
// Memory bounds it where there is work, a launch where there is not.  Measured: 32,760 tokens x 80 heads of 128, normalised over the
// token 242 us = 5.5 TB/s; 4,680 x 120 heads into pages 72 us = 4.0 TB/s, where a lane's five pieces and their weights leave room for 12
// wavefronts a compute unit (two pieces a lane 81, three 97, four 100, eight 166; workgroups that keep the weights for several tokens and
// ask for the next one's rows ahead 98); one token x 80 heads 4.1 us, 769 x 12 of 64 in fp32 5.1.
#include "dit_paged.h"

#include "../../include/dit_attn.h"

namespace dit {

namespace {

enum RowNorm { RN_NONE = 0, RN_HEAD = 1, RN_TOKEN = 2 };
constexpr int kMostRowChunks = 8;

template <bool PAST>
__device__ __forceinline__ void store8(void* y, int64_t off, int type, const float v[8]) {
    if (type == DIT_F32) {
        float4* const p = reinterpret_cast<float4*>(static_cast<float*>(y) + off);
        p[0] = make_float4(v[0], v[1], v[2], v[3]);
        p[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        u32x4* const p = reinterpret_cast<u32x4*>(static_cast<uint16_t*>(y) + off);
        const u32x4 u = type == DIT_F16 ? pack8<OP_F16>(v) : pack8<OP_BF16>(v);
        if constexpr (PAST) __builtin_nontemporal_store(u, p);
        else *p = u;
    }
}

// Sum and largest magnitude over the L lanes of a head (8 or 16, neighbours).
template <int L>
__device__ __forceinline__ float head_sum(float x) {
#pragma unroll
    for (int d = L / 2; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}
template <int L>
__device__ __forceinline__ float head_max(float x) {
#pragma unroll
    for (int d = L / 2; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}

// A sum of squares that fp32 holds: neither past its range nor of squares that underflow.
__device__ __forceinline__ bool sum_holds(float sum, float eps) { return sum < 0x1p120f && eps >= 0x1p-100f; }

// Power of two that brings the larger of the row's largest magnitude and sqrt(eps) near 1 (none for 0, an infinity or a NaN).
__device__ __forceinline__ int norm_shift(float top, float eps) {
    if (!(top < INFINITY)) return 0;
    const int of_row = top > 0.f ? __builtin_amdgcn_frexp_expf(top) : -1000;
    const int of_eps = eps > 0.f ? __builtin_amdgcn_frexp_expf(eps) >> 1 : -1000;
    const int e = of_row > of_eps ? of_row : of_eps;
    return e == -1000 ? 0 : -e;
}

// Eight channels as they lie in memory.
template <bool F32>
struct Piece {
    u32x4 v[F32 ? 2 : 1];
};
template <bool F32, bool PAST>
__device__ __forceinline__ Piece<F32> load_piece(const void* x, int64_t off) {
    const u32x4* const p = reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(x) + off * (F32 ? 4 : 2));
    Piece<F32> k;
#pragma unroll
    for (int i = 0; i < (F32 ? 2 : 1); ++i) {
        if constexpr (PAST) k.v[i] = __builtin_nontemporal_load(p + i);
        else k.v[i] = p[i];
    }
    return k;
}
template <bool F32>
__device__ __forceinline__ void numbers(const Piece<F32>& k, float v[8]) {
    if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(k.v[i >> 2][i & 3]);
    } else {
        widen8(k.v[0], v);
    }
}

// W wavefronts a token, C heads' pieces a lane: wavefronts [0, wq) have the heads of q, the next wk those of k, the rest v's.
// RN_TOKEN: a workgroup has whole tokens, and exchanges the sums.  PAST: rows past the caches (non-temporal), for calls that exceed
// them; 288 MB, which do not, take 72 us through the caches and 75 past them.
template <int D, int NORM, int C, bool F32, bool PAST>
__global__ void __launch_bounds__(1024) rows_kernel(const RowsArgs a, int wq, int wk, int W, int t_end) {
    constexpr int L = D / 8;    // lanes of a head
    constexpr int HW = 64 / L;  // heads of a wavefront, a time
    __shared__ float s_part[16];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t id = blockIdx.x * (blockDim.x >> 6) + wave;
    const uint32_t tok = a.t0 + id / (uint32_t)W;
    const int w = (int)(id % (uint32_t)W);
    const bool there = tok < (uint32_t)t_end;  // (a wavefront without a token goes along to the barrier)
    const int t = there ? (int)tok : t_end - 1;
    const int kind = w < wq ? 0 : w < wq + wk ? 1 : 2;
    const RowTensor& x = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
    const int part = kind == 0 ? w : kind == 1 ? w - wq : w - wq - wk;
    const int slice = lane % L;
    const int head0 = part * (C * HW) + lane / L;
    auto head = [&](int c) { return head0 + c * HW < x.H ? head0 + c * HW : x.H - 1; };

    // All that a row needs is asked for before any of it is used: the counts (first: what is asked for later need not have come
    // when they have), the rows, the weights, the position and the pairs' turns.
    int start = 0, length = 0;  // of request `lane`
    if (a.cached) {
        start = a.pages.q_start[lane <= a.pages.n_requests ? lane : a.pages.n_requests];
        length = a.pages.kv_len[lane < a.pages.n_requests ? lane : a.pages.n_requests - 1];
    }
    const bool turned = kind != 2 && a.pos;
    const bool weighed = NORM != RN_NONE && kind != 2 && x.gamma;
    Piece<F32> raw[C];
#pragma unroll
    for (int c = 0; c < C; ++c) raw[c] = load_piece<F32, PAST>(x.x, (int64_t)t * x.sx_t + (int64_t)head(c) * x.sx_h + 8 * slice);
    [[maybe_unused]] Piece<true> gamma[C];
    if constexpr (NORM != RN_NONE) {
        if (weighed) {
#pragma unroll
            for (int c = 0; c < C; ++c) gamma[c] = load_piece<true, false>(x.gamma, (int64_t)head(c) * D + 8 * slice);
        }
    }
    // where the row goes
    int64_t place = -1;  // of the token in its request
    int entry = -1, r = -1;
    if (a.cached) {
        int past = 0, keys = 0;  // one past the request's last new token, its tokens
        if (a.pages.n_requests < 64) {
            const uint64_t b = __ballot(lane <= a.pages.n_requests && start <= t);
            r = b ? 63 - __builtin_clzll(b) : -1;
            if (r == a.pages.n_requests) r = -1;
            if (r >= 0) {
                past = __builtin_amdgcn_readlane(start, r + 1);
                keys = __builtin_amdgcn_readlane(length, r);
            }
        } else {
            r = request_of(a.pages, t, lane);
            if (r >= 0) {
                past = a.pages.q_start[r + 1];
                keys = a.pages.kv_len[r];
            }
        }
        past = past < a.N ? past : a.N;  // (as the attention has it: a place is counted from the request's last row that is there)
        place = r < 0 || kind == 0 ? -1 : (int64_t)keys - past + t;
        if (place < 0 || place >= (int64_t)a.pages.max_pages * a.pages.page.d || place > 0x7fffffff) place = -1;
        if (place >= 0) entry = a.pages.table[(int64_t)r * a.pages.max_pages + div_by((uint32_t)place, a.pages.page)];
    }
    const bool live = there && !(a.cached && r < 0);
    float2 cs[4];
    if (turned) {
        int at[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) at[i] = a.pos[3 * (int64_t)t + i];
        // (a pair of two axes holds the last pair of the one and the first of the next at most once in four)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int pair = 4 * slice + i;
            const int p = pair < a.hd[0] ? at[0] : pair < a.hd[0] + a.hd[1] ? at[1] : at[2];
            const double turns = (double)p * a.turn[pair];
            const float f = (float)(turns - rint(turns));
            float sn, c;
            sincospif(2.0f * f, &sn, &c);
            cs[i] = make_float2(c, sn);
        }
    }

    float v[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) numbers<F32>(raw[c], v[c]);
    if (NORM == RN_HEAD && kind != 2) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float sum = 0.f, eps = a.eps;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(v[c][i], v[c][i], sum);
            sum = head_sum<L>(sum);
            if (__any(!sum_holds(sum, eps))) {
                float top = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, __builtin_fabsf(v[c][i]));
                const int k = norm_shift(head_max<L>(top), eps);
                eps = ldexpf(eps, 2 * k);
                sum = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[c][i] = ldexpf(v[c][i], k);
                    sum = fmaf(v[c][i], v[c][i], sum);
                }
                sum = head_sum<L>(sum);
            }
            const float f = 1.0f / sqrtf(sum * (1.0f / D) + eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] *= f;
        }
    }
    if constexpr (NORM == RN_TOKEN) {
        // the token's wavefronts of this kind; v's go along
        const int base = wave - w + (kind == 0 ? 0 : kind == 1 ? wq : wq + wk);
        const int count = kind == 0 ? wq : kind == 1 ? wk : W - wq - wk;
        auto all = [&](float mine, auto&& join) {
            if (lane == 0) s_part[wave] = mine;
            __syncthreads();
            float r = s_part[base];
            for (int i = 1; i < count; ++i) r = join(r, s_part[base + i]);
            __syncthreads();
            return r;
        };
        auto squares = [&]() {
            float sum = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (head0 + c * HW < x.H)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum = fmaf(v[c][i], v[c][i], sum);
            return all(head_sum<64>(sum), [](float p, float q) { return p + q; });
        };
        float sum = squares(), eps = a.eps;
        if (__syncthreads_or(!sum_holds(sum, eps))) {
            float top = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (head0 + c * HW < x.H)
#pragma unroll
                    for (int i = 0; i < 8; ++i) top = fmaxf(top, __builtin_fabsf(v[c][i]));
            top = all(head_max<64>(top), [](float p, float q) { return fmaxf(p, q); });
            if (kind != 2) {
                const int k = norm_shift(top, eps);
                eps = ldexpf(eps, 2 * k);
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[c][i] = ldexpf(v[c][i], k);
            }
            sum = squares();
        }
        if (kind != 2) {
            const float f = 1.0f / sqrtf(sum / (float)(x.H * D) + eps);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] *= f;
        }
    }
    if (!live) return;
    if constexpr (NORM != RN_NONE) {
        if (weighed) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float g[8];
                numbers<true>(gamma[c], g);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] *= g[i];
            }
        }
    }
    if (turned) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 y = rotate_pair(v[c][2 * i], v[c][2 * i + 1], cs[i]);
                v[c][2 * i] = y.x;
                v[c][2 * i + 1] = y.y;
            }
    }
    if (a.cached && kind != 0) {
        if (place < 0 || entry < 0 || entry >= a.pages.n_pages) return;
        const uint32_t slot = (uint32_t)place - div_by((uint32_t)place, a.pages.page) * a.pages.page.d;
        const int64_t off16 = (int64_t)entry * a.pages.page16 + (int64_t)slot * a.pages.token16;
        u32x4* const rows = reinterpret_cast<u32x4*>(kind == 1 ? a.k_cache : a.v_cache) + off16;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int h = head0 + c * HW;
            if (h < x.H) rows[(int64_t)h * a.pages.head16 + slice] = a.cache_f16 ? pack8<OP_F16>(v[c]) : pack8<OP_BF16>(v[c]);
        }
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int h = head0 + c * HW;
            if (h < x.H) store8<PAST>(x.y, (int64_t)t * x.sy_t + (int64_t)h * x.sy_h + 8 * slice, a.y_type, v[c]);
        }
    }
}

// Wavefronts that the heads of q, k and v take with C pieces a lane.
struct RowWaves {
    int q, k, v;
    int all() const { return q + k + v; }
};
RowWaves row_waves(int H, int Hk, int Hv, int D, int C) {
    const int per = C * 512 / D;
    return {(H + per - 1) / per, (Hk + per - 1) / per, (Hv + per - 1) / per};
}

template <int D, int NORM, int C, bool F32, bool PAST>
hipError_t launch_rows_c(const RowsArgs& a, hipStream_t s) {
    const RowWaves w = row_waves(a.q.H, a.k.H, a.v.H, D, C);
    const int W = w.all();
    // whole tokens a workgroup where their wavefronts have to meet; a launch has fewer than 2^32 work items
    const int tokens = NORM == RN_TOKEN ? (W >= 4 ? 1 : 4 / W) : 0;
    const int64_t most = tokens ? 0xffffffffLL / (64 * W * tokens) * tokens : 0xffffffffLL / 256 * 4 / W;  // (W: rows_heads_fit)
    for (int64_t t = 0; t < a.N; t += most) {
        const int64_t n = a.N - t < most ? a.N - t : most;
        RowsArgs b = a;
        b.t0 = (int)t;
        const int64_t groups = tokens ? (n + tokens - 1) / tokens : (n * W + 3) / 4;
        hipLaunchKernelGGL((rows_kernel<D, NORM, C, F32, PAST>), dim3((unsigned)groups), dim3(tokens ? 64 * W * tokens : 256), 0, s,
                           b, w.q, w.k, W, (int)(t + n));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int D, int NORM, bool F32, bool PAST>
hipError_t launch_rows_p(const RowsArgs& a, hipStream_t s) {
    // Pieces a lane: as few as keep the memory busy (four wavefronts a compute unit) where there are few tokens; else those that
    // leave the fewest lanes without a head, many rather than few (the angles are worked out once a wavefront).  The wavefronts of
    // a token that have to meet are sixteen at most.
    constexpr int kPieces[] = {1, 2, 3, 4, 5, 8};
    int C = 0, best = 0;
    for (const int c : kPieces) {
        const int W = row_waves(a.q.H, a.k.H, a.v.H, D, c).all();
        if (NORM == RN_TOKEN && W > 16) continue;
        if (C && (c > 5 || (int64_t)a.N * W < 4 * kCUs)) break;
        if (!C || W * c <= best) {
            C = c;
            best = W * c;
        }
    }
    switch (C) {
        case 1: return launch_rows_c<D, NORM, 1, F32, PAST>(a, s);
        case 2: return launch_rows_c<D, NORM, 2, F32, PAST>(a, s);
        case 3: return launch_rows_c<D, NORM, 3, F32, PAST>(a, s);
        case 4: return launch_rows_c<D, NORM, 4, F32, PAST>(a, s);
        case 5: return launch_rows_c<D, NORM, 5, F32, PAST>(a, s);
        default: return launch_rows_c<D, NORM, 8, F32, PAST>(a, s);
    }
}

template <int D, int NORM>
hipError_t launch_rows_n(const RowsArgs& a, hipStream_t s) {
    if (a.x_f32) return launch_rows_p<D, NORM, true, false>(a, s);
    const bool past = exceeds_caches((int64_t)a.N * (a.q.H + a.k.H + a.v.H) * D * 2);
    return past ? launch_rows_p<D, NORM, false, true>(a, s) : launch_rows_p<D, NORM, false, false>(a, s);
}

template <int D>
hipError_t launch_rows_d(const RowsArgs& a, hipStream_t s) {
    return a.norm == RN_TOKEN ? launch_rows_n<D, RN_TOKEN>(a, s) : a.norm == RN_HEAD ? launch_rows_n<D, RN_HEAD>(a, s)
                                                                                     : launch_rows_n<D, RN_NONE>(a, s);
}

}  // namespace

bool rows_heads_fit(int H, int Hk, int Hv) { return (int64_t)H + Hk + Hv <= 1 << 27; }
bool rows_fit(int H, int Hk, int Hv, int D) { return row_waves(H, Hk, Hv, D, kMostRowChunks).all() <= 16; }

hipError_t launch_rows(const RowsArgs& a, int D, hipStream_t s) {
    return D == 128 ? launch_rows_d<128>(a, s) : launch_rows_d<64>(a, s);
}

}  // namespace dit
