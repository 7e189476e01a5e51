// Projection of 8-bit rows: y[m, n] = (sum_k x[m, k] w[n, k]) * (x_scale[m] * w_scale[n]) + bias[n], the sum an exact 32-bit
// integer on the matrix cores.  Few token rows are done here, straight from memory; more by the tiles of dit_linear.hip and
// dit_linear_small.hip, which take 8-bit operands at twice the contraction indices a step.
#include "dit_attn_device.h"
#include "dit_attn_internal.h"

namespace dit {

namespace {

constexpr int kFewWaves = 8;

// 16 bytes of a row from byte `at` on, those from `end` on zeros.
__device__ __forceinline__ u32x4 load_cut_piece(const int8_t* row, int at, int end) {
    u32x4 v = mk4(0u, 0u, 0u, 0u);
    if (at < end) v = *reinterpret_cast<const u32x4*>(row + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int bits = 8 * (end - at - 4 * i);  // of this dword, those that count
        v[i] = bits <= 0 ? 0u : bits < 32 ? v[i] & ((1u << bits) - 1u) : v[i];
    }
    return v;
}

// A workgroup takes 16 features and all token rows (16 TB at most); its wavefronts share K in blocks of 128.  w rows ride the
// A operand of v_mfma_i32_16x16x64_i8, token rows the B operand, both straight from memory: a lane (i, g) holds 16
// bytes of row i and ends with token i, features 4 g .. 4 g + 3.
template <int TB, bool OUT_F32>
__global__ void __launch_bounds__(64 * kFewWaves) linear_few_kernel(const LinearQuantArgs a) {
    __shared__ i32x4 part[kFewWaves][TB][64];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lr = lane & 15, lg = lane >> 4;
    const int n0 = blockIdx.x * 16;
    // (rows past the end are the last one again: their sums are not stored)
    const int8_t* const wrow = a.w + (int64_t)(n0 + lr < a.N ? n0 + lr : a.N - 1) * a.ldw;
    const int8_t* xrow[TB];
#pragma unroll
    for (int tb = 0; tb < TB; ++tb) xrow[tb] = a.x + (int64_t)(16 * tb + lr < a.M ? 16 * tb + lr : a.M - 1) * a.ldx;
    i32x4 acc[TB];
#pragma unroll
    for (int tb = 0; tb < TB; ++tb) acc[tb] = i32x4{0, 0, 0, 0};

    const int blocks = a.K >> 7;
    constexpr int U = 4;
    int b = wave;
    for (; b + (U - 1) * kFewWaves < blocks; b += U * kFewWaves) {
        u32x4 w[U][2], x[U][2][TB];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = (b + u * kFewWaves) * 128 + 64 * h + 16 * lg;
                w[u][h] = *reinterpret_cast<const u32x4*>(wrow + at);
#pragma unroll
                for (int tb = 0; tb < TB; ++tb) x[u][h][tb] = *reinterpret_cast<const u32x4*>(xrow[tb] + at);
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int tb = 0; tb < TB; ++tb) acc[tb] = mfma16_i8(w[u][h], x[u][h][tb], acc[tb]);
    }
    for (; b < blocks; b += kFewWaves) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = b * 128 + 64 * h + 16 * lg;
            const u32x4 w = *reinterpret_cast<const u32x4*>(wrow + at);
#pragma unroll
            for (int tb = 0; tb < TB; ++tb)
                acc[tb] = mfma16_i8(w, *reinterpret_cast<const u32x4*>(xrow[tb] + at), acc[tb]);
        }
    }
    if (b == blocks && (a.K & 127)) {  // what is left behind the whole blocks is one wavefront's
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = b * 128 + 64 * h + 16 * lg;
            const u32x4 w = load_cut_piece(wrow, at, a.K);
#pragma unroll
            for (int tb = 0; tb < TB; ++tb) acc[tb] = mfma16_i8(w, load_cut_piece(xrow[tb], at, a.K), acc[tb]);
        }
    }
#pragma unroll
    for (int tb = 0; tb < TB; ++tb) part[wave][tb][lane] = acc[tb];
    __syncthreads();
    // thread t: token t / 16 of a block of 32, feature t % 16
    for (int i = tid; i < 256 * TB; i += 64 * kFewWaves) {
        const int m = i >> 4, f = i & 15, n = n0 + f;
        if (m >= a.M || n >= a.N) continue;
        int sum = 0;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) sum += part[w][m >> 4][16 * (f >> 2) + (m & 15)][f & 3];
        const float y = fmaf((float)sum, a.x_scale[m] * a.w_scale[n], a.bias ? __uint_as_float((uint32_t)a.bias[n] << 16) : 0.f);
        const int64_t o = (int64_t)m * a.ldy + n;
        if constexpr (OUT_F32) static_cast<float*>(a.y)[o] = y;
        else static_cast<uint16_t*>(a.y)[o] = (uint16_t)pack2<OP_BF16>(y, 0.f);
    }
}

template <int TB>
hipError_t launch_few(const LinearQuantArgs& a, hipStream_t s) {
    const auto kern = a.out_f32 ? linear_few_kernel<TB, true> : linear_few_kernel<TB, false>;
    hipLaunchKernelGGL(kern, dim3((unsigned)((a.N + 15) / 16)), dim3(64 * kFewWaves), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_quant(const LinearQuantArgs& q, hipStream_t s) {
    int cus = 0;
    hipError_t e = compute_units(&cus);
    if (e != hipSuccess) return e;
    if (q.M <= 16) return launch_few<1>(q, s);
    LinearArgs a{};
    a.x = reinterpret_cast<const uint16_t*>(q.x);
    a.w = reinterpret_cast<const uint16_t*>(q.w);
    a.x_scale = q.x_scale;
    a.w_scale = q.w_scale;
    a.bias = q.bias;
    a.y = q.y;
    a.M = q.M;
    a.N = q.N;
    a.K = q.K / 128 * 64;
    a.tail = q.K % 128;
    a.ldx = q.ldx / 2;
    a.ldw = q.ldw / 2;
    a.ldy = q.ldy;
    a.out_f32 = q.out_f32;
    const bool big_too = a.tail == 0 && a.N >= 8;
    const int form = choose_linear_form_i8(q.M, q.N, q.K, big_too, cus);
    if (form) return launch_linear_small_i8(a, form, s);
    // 256 x 256 tiles store whole 16-byte pieces: the last N % 8 features are a call of their own
    const int rest = a.N % 8;
    a.N -= rest;
    a.nTM = (a.M + kLinBM - 1) / kLinBM;
    a.nTN = (a.N + kLinBN - 1) / kLinBN;
    if ((int64_t)a.nTM * a.nTN > 0x7fffffff) return hipErrorInvalidValue;
    e = launch_linear_i8(a, s);
    if (e != hipSuccess || rest == 0) return e;
    a.w += (int64_t)a.N * a.ldw;
    a.w_scale += a.N;
    if (a.bias) a.bias += a.N;
    a.y = static_cast<uint8_t*>(a.y) + (int64_t)a.N * (a.out_f32 ? 4 : 2);
    a.N = rest;
    return launch_linear_small_i8(a, choose_linear_form_i8(a.M, a.N, q.K, false, cus), s);
}

}  // namespace dit
