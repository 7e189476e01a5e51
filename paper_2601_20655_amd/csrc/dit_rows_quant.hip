// Rows of numbers to 8-bit rows (N signed integers and one fp32 scale a row) and back: plainly, through a GELU, or behind
// the addition to the residual stream and an RMS normalisation.
//
// A row has to be seen whole before its first integer is known, and is read once: W wavefronts hold it in registers, C
// chunks of eight columns a lane, exchange its largest magnitude (and sum of squares) and write its integers.  The
// normalisation's factor 1 / sqrt(mean + eps) is common to the row, so it cancels in the integers
// q = rint(t * (127 * (1 / max|t|))), t = h * gamma, and appears in the scale alone: the integers do not wait for the sum.
//
// Squares below 2^-126 lose digits and below 2^-150 vanish.  An eps of 2^-100 or more outweighs what is lost; with a smaller one (0 is
// allowed) the row is first scaled by a power of two that brings its largest number, or sqrt(eps), near 1.  It rounds nothing and
// cancels in the integers and in the scale.
//
// What bounds it: memory.  32,760 x 5,120, new rows at every call: norm with 16-bit residual 194 us (6.0 TB/s of reads and
// writes), with a 32-bit one 332 (5.6), without 107 (4.7; 85 without weights, which come from the second-level cache twice as
// wide as the row), 16-bit rows to 8 bits 83 (6.1), back to 16 bits 81 (6.2) and 32 bits 128 (6.5); GELU, 32,760 x 20,480, 335
// to 359 (5.6 to 6.0; there the vector ALU is busy in 97 % of the clocks).  (A copy of 2 GiB: 4.95 TB/s.)  One row: 3.3 us.
// The norm of rows beyond 49,152 columns takes seven or eight chunks a lane, which spill 12 to 120 bytes a lane: 2,048 x 65,536
// with a 16-bit residual 203 us (4.6 TB/s), 2,048 x 40,960 102 (5.7).  Rows of 65,536 to 8 bits, no spill: 80 us, 32-bit ones 131
// (5.0 to 5.1).
// Tried without gain: workgroups that walk several rows with the weights in registers (norm 201 -> 219 to 249 us; 105 -> 98
// without a residual), weights asked for ahead of their use with rows past the caches (105 -> 121 without a residual).
#include <type_traits>

#include "dit_attn_device.h"
#include "dit_attn_internal.h"

namespace dit {

namespace {

constexpr int kMostChunks = 8;  // of a lane: 16 wavefronts of 64 lanes hold rows of 65,536 columns
static_assert(kMostChunks * 8 * 64 * 16 == kQuantMaxColumns, "the longest row fits one workgroup");

enum RowMode { ROW_PLAIN = 0, ROW_GELU = 1, ROW_NORM = 2 };
enum RowType { ROW_NONE = 0, ROW_BF16 = 1, ROW_F32 = 2 };  // of the residual

// x/2 (1 + tanh(u)) = x / (1 + exp(-2u)), u = sqrt(2/pi) (x + 0.044715 x^3)
__device__ __forceinline__ float gelu_tanh(float x) {
    constexpr float c1 = -2.0f * 0.7978845608028654f * kLog2e, c3 = c1 * 0.044715f;
    const float e = __builtin_amdgcn_exp2f(x * fmaf(c3, x * x, c1));
    return x * __builtin_amdgcn_rcpf(1.0f + e);
}

// Eight columns from `col` on, as they lie in memory.  PAST: past the caches, for rows that they cannot keep
// (exceeds_caches).  Not for 32-bit rows, whose eight columns are two loads or stores that each touch half of every 32 bytes:
// the caches join them (norm with a 32-bit residual 333 us, past the caches 365).
template <bool F32>
struct Chunk {
    u32x4 v[F32 ? 2 : 1];
};
template <bool F32, bool PAST>
__device__ __forceinline__ Chunk<F32> load_chunk(const void* row, int col) {
    const u32x4* const p = reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(row) + (size_t)col * (F32 ? 4 : 2));
    Chunk<F32> k;
    if constexpr (F32) {
        k.v[0] = p[0];
        k.v[1] = p[1];
    } else if constexpr (PAST) {
        k.v[0] = __builtin_nontemporal_load(p);
    } else {
        k.v[0] = p[0];
    }
    return k;
}
template <bool F32>
__device__ __forceinline__ void to_numbers(const Chunk<F32>& k, float v[8]) {
    if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(k.v[i >> 2][i & 3]);
    } else {
        widen8(k.v[0], v);
    }
}
template <bool F32, bool PAST>
__device__ __forceinline__ void store_chunk(void* row, int col, const float v[8]) {
    if constexpr (F32) {
        float4* const p = reinterpret_cast<float4*>(static_cast<float*>(row) + col);
        p[0] = make_float4(v[0], v[1], v[2], v[3]);
        p[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        u32x4* const p = reinterpret_cast<u32x4*>(static_cast<uint16_t*>(row) + col);
        if constexpr (PAST) __builtin_nontemporal_store(pack8<OP_BF16>(v), p);
        else *p = pack8<OP_BF16>(v);
    }
}
template <bool F32>
__device__ __forceinline__ float load_number(const void* row, int i) {
    if constexpr (F32) return static_cast<const float*>(row)[i];
    else return __uint_as_float((uint32_t)static_cast<const uint16_t*>(row)[i] << 16);
}
template <bool F32>
__device__ __forceinline__ void store_number(void* row, int i, float v) {
    if constexpr (F32) static_cast<float*>(row)[i] = v;
    else static_cast<uint16_t*>(row)[i] = (uint16_t)pack2<OP_BF16>(v, 0.f);
}

// v * inverse, rounded to the nearest even integer of magnitude 127 or less, in the low byte: 1.5 * 2^23 puts the integer's
// two's complement into the last bits of the significand.  (Product and sum are rounded one after the other, as the formula
// has them: fused, one number in ten million fell to the other side of a tie.)
__device__ __forceinline__ uint32_t to_byte(float v, float inverse) {
#pragma clang fp contract(off)
    const float p = v * inverse;
    return __float_as_uint(p + 12582912.0f);
}
__device__ __forceinline__ uint32_t to_bytes(const float v[4], float inverse) {
    const uint32_t lo = __builtin_amdgcn_perm(to_byte(v[1], inverse), to_byte(v[0], inverse), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(to_byte(v[3], inverse), to_byte(v[2], inverse), 0x04000c0cu);
    return lo | hi;
}

// W wavefronts a row, one row a workgroup or several.  CUT: N is no multiple of 8.  PAST: 16-bit rows past the
// caches.
template <int MODE, bool X_F32, int RES, int C, bool CUT, bool PAST>
__global__ void __launch_bounds__(1024) quant_rows_kernel(const QuantArgs a, int W) {
    constexpr bool R_F32 = RES == ROW_F32;
    __shared__ float s_top[16], s_sum[16];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rows = (blockDim.x >> 6) / W;  // of this workgroup
    const int sub = wave / W, part = wave - sub * W;
    const int64_t m = (int64_t)blockIdx.x * rows + sub;
    const bool live = m < a.M;  // (a wavefront without a row goes along to the barrier)
    const int64_t mm = live ? m : a.M - 1;
    const void* const x = static_cast<const uint8_t*>(a.x) + mm * a.ldx * (X_F32 ? 4 : 2);
    const void* const r = RES ? static_cast<const uint8_t*>(a.residual) + mm * a.ldr * (R_F32 ? 4 : 2) : nullptr;

    // Chunk c of lane l is chunk (c W + part) 64 + l of the row.  Whole chunks are loaded without a branch: behind the last
    // one it is loaded again, and counts as zeros.  (One chunk a lane: there may be no whole one.)  A last chunk that N cuts
    // is loaded number by number, by its one lane, ahead of the row: widening waits for it inside its branch, so that the wavefront
    // that has it asks for the row behind that.  (Behind the row, the whole chunks were waited for first: 7,800 x 1,537 with a
    // 16-bit residual 19.0 us, 17.2 this way.)
    const int whole = a.N >> 3, rest = CUT ? a.N & 7 : 0;
    const int first = part * 64 + lane, step = W * 64;
    float end_x[7] = {}, end_r[7] = {}, end_g[7] = {};
    if (CUT && (whole & 63) == lane && (whole >> 6) % W == part) {
#pragma unroll
        for (int i = 0; i < 7; ++i) end_x[i] = load_number<X_F32>(x, 8 * whole + (i < rest ? i : 0));
        if constexpr (RES != ROW_NONE) {
#pragma unroll
            for (int i = 0; i < 7; ++i) end_r[i] = load_number<R_F32>(r, 8 * whole + (i < rest ? i : 0));
        }
        if (MODE == ROW_NORM && a.gamma) {
#pragma unroll
            for (int i = 0; i < 7; ++i) end_g[i] = a.gamma[8 * whole + (i < rest ? i : 0)];
        }
    }
    // Weights are asked for with the row, where they and it take no more than 60 registers (and the rows are not past the caches:
    // norm of 32,760 x 5,120 with a 16-bit residual 193 us behind the row, 201 with it).  With them, and behind: 7,800 x 5,120
    // without a residual 26 and 31, 7,800 x 1,536 9.0 and 10.1, with a 16-bit one 15.0 and 16.3, with a 32-bit one 26.6 and 28.5;
    // but 3,600 x 5,120 with a 32-bit one, of more registers, 66 and 43.  (Behind the row they come chunk by chunk, each waited for,
    // and the first wait is for the stores of h too: a known lead, not taken.)
    constexpr bool AHEAD = MODE == ROW_NORM && !PAST && C > 1 &&
                           C * (8 + (X_F32 ? 8 : 4) + (RES == ROW_NONE ? 0 : R_F32 ? 8 : 4)) + (CUT ? 21 : 0) <= 60;
    [[maybe_unused]] Chunk<true> kg[C];
    float t[C][8];
    if constexpr (C == 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) t[0][i] = 0.f;
        if (first < whole) {
            const Chunk<X_F32> kx = load_chunk<X_F32, PAST>(x, 8 * first);
            float v[8];
            if constexpr (RES != ROW_NONE) to_numbers<R_F32>(load_chunk<R_F32, PAST>(r, 8 * first), v);
            to_numbers<X_F32>(kx, t[0]);
            if constexpr (RES != ROW_NONE) {
#pragma unroll
                for (int i = 0; i < 8; ++i) t[0][i] += v[i];
            }
        }
    } else {
        Chunk<X_F32> kx[C];
        Chunk<R_F32> kr[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = first + c * step;
            kx[c] = load_chunk<X_F32, PAST>(x, 8 * (at < whole ? at : whole - 1));
        }
        if constexpr (RES != ROW_NONE) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int at = first + c * step;
                kr[c] = load_chunk<R_F32, PAST>(r, 8 * (at < whole ? at : whole - 1));
            }
        }
        if constexpr (AHEAD) {
            if (a.gamma) {
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const int at = first + c * step;
                    kg[c] = load_chunk<true, false>(a.gamma, 8 * (at < whole ? at : whole - 1));
                }
            }
        }
        // (All are asked for before the first is used.  Left to the compiler, loads sank behind the test for the row's end and
        // were waited for one by one: norm of 7,800 x 1,536 17.3 us, 16.2 this way, 32,760 x 5,120 200 and 194.  Not the longest
        // rows, whose registers do not reach for it.)
        if constexpr (C <= 5) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                for (u32x4& u : kx[c].v) asm volatile("" : "+v"(u));
                if constexpr (RES != ROW_NONE) {
                    for (u32x4& u : kr[c].v) asm volatile("" : "+v"(u));
                }
            }
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = first + c * step;
            float v[8];
            to_numbers<X_F32>(kx[c], t[c]);
            if constexpr (RES != ROW_NONE) to_numbers<R_F32>(kr[c], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (RES != ROW_NONE) t[c][i] += v[i];
                t[c][i] = at < whole ? t[c][i] : 0.f;
            }
        }
    }
    if constexpr (CUT) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (first + c * step != whole) continue;
#pragma unroll
            for (int i = 0; i < 7; ++i) t[c][i] = i < rest ? RES != ROW_NONE ? end_x[i] + end_r[i] : end_x[i] : 0.f;
        }
    }

    if constexpr (RES != ROW_NONE) {
        if (a.h_out && live) {
            void* const h = static_cast<uint8_t*>(a.h_out) + m * a.ldh * (R_F32 ? 4 : 2);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int at = first + c * step;
                if (at < whole) {
                    store_chunk<R_F32, PAST>(h, 8 * at, t[c]);
                } else if (CUT && at == whole) {
#pragma unroll
                    for (int i = 0; i < 7; ++i)
                        if (i < rest) store_number<R_F32>(h, 8 * at + i, t[c][i]);
                }
            }
        }
    }
    float top = 0.f, sum = 0.f, eps = a.eps;
    if constexpr (MODE == ROW_NORM) {
        if (eps < kNormSmallEps) {  // (uniform)
            float big = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) big = fmaxf(big, __builtin_fabsf(t[c][i]));
#pragma unroll
            for (int d = 32; d > 0; d >>= 1) big = fmaxf(big, __shfl_xor(big, d));
            if (W > 1) {
                if (lane == 0) s_top[wave] = big;
                __syncthreads();
                for (int w = 0; w < W; ++w) big = fmaxf(big, s_top[sub * W + w]);
                __syncthreads();  // (s_top is written again below)
            }
            // up by 2^k, k >= 0: the larger of the row's largest number and sqrt(eps) to about 1.  (The exponent of 0, of an
            // infinity and of a NaN reads as 0.)
            const int of_row = big > 0.f ? __builtin_amdgcn_frexp_expf(big) : -1000;
            const int of_eps = eps > 0.f ? __builtin_amdgcn_frexp_expf(eps) >> 1 : -1000;
            const int e = of_row > of_eps ? of_row : of_eps, k = e < 0 ? -e : 0;
            eps = ldexpf(eps, 2 * k);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) t[c][i] = ldexpf(t[c][i], k);
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(t[c][i], t[c][i], sum);
        if (a.gamma) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int at = first + c * step;
                if (at < whole) {
                    float g[8];
                    if constexpr (AHEAD) to_numbers<true>(kg[c], g);
                    else load8(a.gamma, 8 * at, 1, g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) t[c][i] *= g[i];
                } else if (CUT && at == whole) {
#pragma unroll
                    for (int i = 0; i < 7; ++i) t[c][i] = i < rest ? t[c][i] * end_g[i] : t[c][i];
                }
            }
        }
    }
    if constexpr (MODE == ROW_GELU) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) t[c][i] = gelu_tanh(t[c][i]);
    }
    // (by IEEE maximum, which passes a NaN on)
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = __builtin_elementwise_maximum(top, __builtin_fabsf(t[c][i]));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        top = __builtin_elementwise_maximum(top, __shfl_xor(top, d));
        if constexpr (MODE == ROW_NORM) sum += __shfl_xor(sum, d);
    }
    if (W > 1) {
        if (lane == 0) {
            s_top[wave] = top;
            s_sum[wave] = sum;
        }
        __syncthreads();
        top = s_top[sub * W];
        sum = s_sum[sub * W];
        for (int w = 1; w < W; ++w) {
            top = __builtin_elementwise_maximum(top, s_top[sub * W + w]);
            sum += s_sum[sub * W + w];
        }
    }
    if (!live) return;

    bool good = top < INFINITY;
    float divisor = kQuantTop;  // the scale is top / divisor
    if constexpr (MODE == ROW_NORM) {
        good = good && sum < INFINITY;
        divisor *= sqrtf(sum / (float)a.N + eps);
    }
    const bool some = good && top >= kQuantZero;
    const float inverse = some ? kQuantTop * (1.0f / top) : 0.f;
    if (part == 0 && lane == 0) a.scale[m] = !good ? NAN : some ? top / divisor : 0.f;
    int8_t* const q = a.q + m * a.ldq;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = first + c * step;
        uint2 b = make_uint2(to_bytes(t[c], inverse), to_bytes(t[c] + 4, inverse));
        if (!some) b = make_uint2(0u, 0u);  // (a NaN times zero is no zero)
        if (at < whole) {
            *reinterpret_cast<uint2*>(q + 8 * at) = b;
        } else if (CUT && at == whole) {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < rest) q[8 * at + i] = (int8_t)((i < 4 ? b.x : b.y) >> (8 * (i & 3)));
        }
    }
}

// A lane writes 16 bytes at a time: V = 8 or 4 columns.  `parts` wavefronts a row, C pieces a lane.
template <bool OUT_F32, int C, bool CUT, bool PAST>
__global__ void __launch_bounds__(256) dequant_rows_kernel(const DequantArgs a, int parts) {
    constexpr int V = OUT_F32 ? 4 : 8;
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    typedef std::conditional_t<OUT_F32, uint32_t, u32x2> piece_t;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t id = (int64_t)blockIdx.x * 4 + wave;
    const int64_t m = id / parts;
    if (m >= a.M) return;
    const int first = (int)(id - m * parts) * (64 * C) + lane;
    const int8_t* const q = a.q + m * a.ldq;
    void* const y = static_cast<uint8_t*>(a.y) + m * a.ldy * (OUT_F32 ? 4 : 2);
    const float scale = a.scale[m];
    const int whole = a.N / V, rest = CUT ? a.N % V : 0;
    piece_t b[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = first + c * 64;
        b[c] = piece_t();
        if (at < whole) {
            const piece_t* const p = reinterpret_cast<const piece_t*>(q + V * (int64_t)at);
            // (past the caches too with 16-bit rows: GELU and reading back, 32,760 x 20,480, 690 -> 642 us; with 32-bit ones
            // 128 -> 130.  The 8-bit rows' own stores stay: this call finds them there, 148 us for rows to 8 bits and back at
            // 32,760 x 5,120, 162 with stores past the caches)
            if constexpr (PAST && !OUT_F32) b[c] = __builtin_nontemporal_load(p);
            else b[c] = *p;
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = first + c * 64;
        auto number = [&](uint32_t u, int i) { return (float)(int8_t)(u >> (8 * i)) * scale; };
        if (at < whole) {
            if constexpr (OUT_F32) {
                const f32x4 v = {number(b[c], 0), number(b[c], 1), number(b[c], 2), number(b[c], 3)};
                f32x4* const p = reinterpret_cast<f32x4*>(static_cast<float*>(y) + V * (int64_t)at);
                if constexpr (PAST) __builtin_nontemporal_store(v, p);
                else *p = v;
            } else {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = number(i < 4 ? b[c].x : b[c].y, i & 3);
                store_chunk<false, PAST>(y, V * at, v);
            }
        } else if (CUT && at == whole) {
            for (int i = 0; i < rest; ++i) store_number<OUT_F32>(y, V * at + i, (float)q[V * at + i] * scale);
        }
    }
}

// A launch has fewer than 2^32 work items: a longer one is not refused, its workgroups are counted modulo that, and rows are
// left out.  So calls of more rows are several launches, of as many groups of `rows` rows (`threads` work items each) as one takes.
template <class F>
hipError_t launch_slices(int M, int rows, int64_t threads, F&& launch) {
    const int64_t most = 0xffffffff / threads * rows;
    for (int64_t m = 0; m < M; m += most) {
        const int some = (int)(M - m < most ? M - m : most);
        launch(m, some, (unsigned)(((int64_t)some + rows - 1) / rows));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// How rows lie over wavefronts.  Where there are wavefronts enough to keep the memory busy, `most` chunks a lane; where there
// are not, one, the row over as many wavefronts as it takes (at most 16, a workgroup).  (A wavefront a SIMD is enough: norm of
// 769 x 5,120 9.3 us if four are asked for, 8.1 with one, 1,560 x 5,120 without a residual 11.2 and 8.5; 1,560 x 5,000 with a
// 32-bit one 21.6 and 24.6.)
constexpr int kBusy = 4 * kCUs;
struct RowLayout {
    int waves, per_lane, rows;  // wavefronts a row, chunks a lane, rows a workgroup
};
RowLayout layout_rows(int M, int N, int most) {
    const int need = ((N + 7) / 8 + 63) / 64;  // wavefronts of one chunk a lane
    if ((int64_t)M * ((need + most - 1) / most) < kBusy) most = 1;
    int w = (need + most - 1) / most;
    if (w > 16) w = 16;
    const int c = (need + w - 1) / w;
    w = (need + c - 1) / c;
    return {w, c, w >= 4 ? 1 : 4 / w};
}

template <int MODE, bool X_F32, int RES, int C>
hipError_t launch_quant(const QuantArgs& a, const RowLayout& l, hipStream_t s) {
    constexpr bool SOME_16 = !X_F32 || RES == ROW_BF16;
    const bool past = SOME_16 && exceeds_caches((int64_t)a.M * a.N * ((X_F32 ? 4 : 2) + (RES == ROW_F32 ? 4 : RES == ROW_BF16 ? 2 : 0)));
    const auto kern = a.N % 8 ? past ? quant_rows_kernel<MODE, X_F32, RES, C, true, SOME_16> : quant_rows_kernel<MODE, X_F32, RES, C, true, false>
                              : past ? quant_rows_kernel<MODE, X_F32, RES, C, false, SOME_16> : quant_rows_kernel<MODE, X_F32, RES, C, false, false>;
    return launch_slices(a.M, l.rows, 64 * l.waves * l.rows, [&](int64_t m, int rows, unsigned groups) {
        QuantArgs b = a;
        b.x = static_cast<const uint8_t*>(a.x) + m * a.ldx * (X_F32 ? 4 : 2);
        if (a.residual) b.residual = static_cast<const uint8_t*>(a.residual) + m * a.ldr * (RES == ROW_F32 ? 4 : 2);
        if (a.h_out) b.h_out = static_cast<uint8_t*>(a.h_out) + m * a.ldh * (RES == ROW_F32 ? 4 : 2);
        b.q = a.q + m * a.ldq;
        b.scale = a.scale + m;
        b.M = rows;
        hipLaunchKernelGGL(kern, dim3(groups), dim3(64 * l.waves * l.rows), 0, s, b, l.waves);
    });
}

template <int MODE, bool X_F32, int RES>
hipError_t launch_quant(const QuantArgs& a, hipStream_t s) {
    // (two chunks a lane where little is done with what is read: 16-bit rows to 8 bits 85 us with two, 90 with five, norm with
    // a 16-bit residual 201 and 212; five elsewhere: GELU 400 with two, 350 with five, norm with a 32-bit residual 341 and
    // 333, with none 111 and 105)
    const RowLayout l = layout_rows(a.M, a.N, MODE == ROW_PLAIN || RES == ROW_BF16 ? 2 : 5);
    switch (l.per_lane) {
        case 1: return launch_quant<MODE, X_F32, RES, 1>(a, l, s);
        case 2: return launch_quant<MODE, X_F32, RES, 2>(a, l, s);
        case 3: return launch_quant<MODE, X_F32, RES, 3>(a, l, s);
        case 4: return launch_quant<MODE, X_F32, RES, 4>(a, l, s);
        case 5: return launch_quant<MODE, X_F32, RES, 5>(a, l, s);
        case 6: return launch_quant<MODE, X_F32, RES, 6>(a, l, s);
        case 7: return launch_quant<MODE, X_F32, RES, 7>(a, l, s);
        case 8: return launch_quant<MODE, X_F32, RES, 8>(a, l, s);
    }
    return hipErrorInvalidValue;
}

template <bool OUT_F32, int C>
hipError_t launch_dequant(const DequantArgs& a, int need, hipStream_t s) {
    constexpr int V = OUT_F32 ? 4 : 8;
    const int parts = (need + C - 1) / C;
    const bool past = exceeds_caches((int64_t)a.M * a.N * (OUT_F32 ? 4 : 2));
    const auto kern = a.N % V ? past ? dequant_rows_kernel<OUT_F32, C, true, true> : dequant_rows_kernel<OUT_F32, C, true, false>
                              : past ? dequant_rows_kernel<OUT_F32, C, false, true> : dequant_rows_kernel<OUT_F32, C, false, false>;
    // (four wavefronts a workgroup; four rows, so that any number of parts makes whole workgroups)
    return launch_slices(a.M, 4, 256 * parts, [&](int64_t m, int rows, unsigned) {
        DequantArgs b = a;
        b.q = a.q + m * a.ldq;
        b.scale = a.scale + m;
        b.y = static_cast<uint8_t*>(a.y) + m * a.ldy * (OUT_F32 ? 4 : 2);
        b.M = rows;
        hipLaunchKernelGGL(kern, dim3((unsigned)(((int64_t)rows * parts + 3) / 4)), dim3(256), 0, s, b, parts);
    });
}

template <bool OUT_F32>
hipError_t launch_dequant(const DequantArgs& a, hipStream_t s) {
    constexpr int V = OUT_F32 ? 4 : 8;
    const int need = (int)((((int64_t)a.N + V - 1) / V + 63) / 64);  // wavefronts of one piece a lane
    // (two pieces a lane: 88 us in 16 bits and 134 in 32; five: 93 and 150)
    return (int64_t)a.M * need < kBusy ? launch_dequant<OUT_F32, 1>(a, need, s) : launch_dequant<OUT_F32, 2>(a, need, s);
}

}  // namespace

hipError_t launch_quant_rows(const QuantArgs& a, hipStream_t s) {
    if (!a.norm) {
        if (a.gelu) return a.x_f32 ? launch_quant<ROW_GELU, true, ROW_NONE>(a, s) : launch_quant<ROW_GELU, false, ROW_NONE>(a, s);
        return a.x_f32 ? launch_quant<ROW_PLAIN, true, ROW_NONE>(a, s) : launch_quant<ROW_PLAIN, false, ROW_NONE>(a, s);
    }
    if (!a.residual) return a.x_f32 ? launch_quant<ROW_NORM, true, ROW_NONE>(a, s) : launch_quant<ROW_NORM, false, ROW_NONE>(a, s);
    if (a.r_f32) return a.x_f32 ? launch_quant<ROW_NORM, true, ROW_F32>(a, s) : launch_quant<ROW_NORM, false, ROW_F32>(a, s);
    return a.x_f32 ? launch_quant<ROW_NORM, true, ROW_BF16>(a, s) : launch_quant<ROW_NORM, false, ROW_BF16>(a, s);
}

hipError_t launch_dequant_rows(const DequantArgs& a, hipStream_t s) {
    return a.out_f32 ? launch_dequant<true>(a, s) : launch_dequant<false>(a, s);
}

}  // namespace dit
