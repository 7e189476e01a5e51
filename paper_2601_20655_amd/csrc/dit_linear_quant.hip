// Projection of 8-bit rows: y[m, n] = (sum_k x[m, k] w[n, k]) * (x_scale[m] * w_scale[n]) + bias[n], the sum an exact 32-bit
// integer on the matrix cores.
#include "dit_attn_device.h"
#include "dit_attn_internal.h"

namespace dit {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// 16 bytes of a row from column k on, those past the row's end zero.  `row` null: a row of zeros.
__device__ __forceinline__ i32x4 load_piece(const int8_t* row, int k, int K) {
    i32x4 v = {0, 0, 0, 0};
    if (row && k < K) {
        v = *reinterpret_cast<const i32x4*>(row + k);
        const int left = K - k;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int bits = 8 * (left - 4 * i);  // of this dword, those that count
            if (bits <= 0) v[i] = 0;
            else if (bits < 32) v[i] &= (1 << bits) - 1;
        }
    }
    return v;
}

// One wavefront a tile of 16 tokens x 16 features, operands straight from memory: w rows ride the A operand of
// v_mfma_i32_16x16x64_i8, token rows the B operand, a lane (i, g) holds bytes 16 g .. 16 g + 15 of row i and ends with token i,
// features 4 g .. 4 g + 3.
__global__ void __launch_bounds__(256) linear_quant_kernel(const LinearQuantArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lr = lane & 15, lg = lane >> 4;
    const int tiles_n = (a.N + 15) / 16;
    const int64_t tile = (int64_t)blockIdx.x * 4 + wave;
    if (tile >= (int64_t)tiles_n * ((a.M + 15) / 16)) return;
    const int m0 = (int)(tile / tiles_n) * 16, n0 = (int)(tile % tiles_n) * 16;
    const int8_t* const xrow = m0 + lr < a.M ? a.x + (int64_t)(m0 + lr) * a.ldx : nullptr;
    const int8_t* const wrow = n0 + lr < a.N ? a.w + (int64_t)(n0 + lr) * a.ldw : nullptr;
    i32x4 acc = {0, 0, 0, 0};
    for (int k = 0; k < a.K; k += 64)
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(load_piece(wrow, k + 16 * lg, a.K), load_piece(xrow, k + 16 * lg, a.K),
                                                    acc, 0, 0, 0);
    const int m = m0 + lr;
    if (m >= a.M) return;
    const float xs = a.x_scale[m];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int n = n0 + 4 * lg + e;
        if (n >= a.N) continue;
        const float b = a.bias ? __uint_as_float((uint32_t)a.bias[n] << 16) : 0.f;
        const float y = (float)acc[e] * (xs * a.w_scale[n]) + b;
        const int64_t i = (int64_t)m * a.ldy + n;
        if (a.out_f32) static_cast<float*>(a.y)[i] = y;
        else static_cast<uint16_t*>(a.y)[i] = (uint16_t)pack2<OP_BF16>(y, 0.f);
    }
}

}  // namespace

hipError_t launch_linear_quant(const LinearQuantArgs& a, hipStream_t s) {
    const int64_t tiles = (int64_t)((a.M + 15) / 16) * ((a.N + 15) / 16);
    hipLaunchKernelGGL(linear_quant_kernel, dim3((unsigned)((tiles + 3) / 4)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace dit
