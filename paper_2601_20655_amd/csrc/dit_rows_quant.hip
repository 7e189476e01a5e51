// Rows of numbers to 8-bit rows (N signed integers and one fp32 scale a row) and back: plainly, through a GELU, or behind
// the addition to the residual stream and an RMS normalisation.
#include "dit_attn_device.h"
#include "dit_attn_internal.h"

namespace dit {

namespace {

constexpr int kRowThreads = 256;

__device__ __forceinline__ float load_number(const void* base, int64_t i, int f32) {
    return f32 ? static_cast<const float*>(base)[i]
               : __uint_as_float((uint32_t)static_cast<const uint16_t*>(base)[i] << 16);
}

__device__ __forceinline__ void store_number(void* base, int64_t i, int f32, float v) {
    if (f32) static_cast<float*>(base)[i] = v;
    else static_cast<uint16_t*>(base)[i] = (uint16_t)pack2<OP_BF16>(v, 0.f);
}

__device__ __forceinline__ float gelu_tanh(float x) {
    const float u = 0.7978845608028654f * (x + 0.044715f * x * x * x);
    return 0.5f * x * (1.0f + tanhf(u));
}

// one workgroup a row, which is read twice: for its largest magnitude and sum of squares, and to quantise it
__global__ void __launch_bounds__(kRowThreads) quant_rows_kernel(const QuantArgs a) {
    __shared__ uint32_t s_top[kRowThreads];
    __shared__ float s_sum[kRowThreads];
    const int64_t m = blockIdx.x;
    const int tid = threadIdx.x;
    auto sum_of = [&](int n) {
        float h = load_number(a.x, m * a.ldx + n, a.x_f32);
        if (a.residual) h += load_number(a.residual, m * a.ldr + n, a.r_f32);
        return h;
    };
    auto value_of = [&](float h, int n) {
        if (a.gelu) return gelu_tanh(h);
        return a.gamma ? h * a.gamma[n] : h;
    };
    uint32_t top = 0;  // of the magnitudes' bit patterns, whose order puts infinities and NaNs above all numbers
    float sum = 0.f;
    for (int n = tid; n < a.N; n += kRowThreads) {
        const float h = sum_of(n);
        const uint32_t b = __float_as_uint(value_of(h, n)) & 0x7fffffffu;
        top = b > top ? b : top;
        sum = fmaf(h, h, sum);
    }
    s_top[tid] = top;
    s_sum[tid] = sum;
    for (int d = kRowThreads / 2; d > 0; d >>= 1) {
        __syncthreads();
        if (tid < d) {
            s_top[tid] = s_top[tid] > s_top[tid + d] ? s_top[tid] : s_top[tid + d];
            s_sum[tid] += s_sum[tid + d];
        }
    }
    __syncthreads();
    const float amax = __uint_as_float(s_top[0]);
    float factor = 1.0f / kQuantTop;
    bool good = s_top[0] < 0x7f800000u;
    if (a.norm) {
        good = good && s_sum[0] < INFINITY;
        factor = 1.0f / (sqrtf(s_sum[0] / (float)a.N + a.eps) * kQuantTop);
    }
    const bool some = good && amax >= kQuantZero;
    const float inverse = some ? kQuantTop / amax : 0.f;
    if (tid == 0) a.scale[m] = !good ? NAN : some ? amax * factor : 0.f;
    for (int n = tid; n < a.N; n += kRowThreads) {
        const float h = sum_of(n);
        if (a.h_out) store_number(a.h_out, m * a.ldh + n, a.r_f32, h);
        a.q[m * a.ldq + n] = some ? (int8_t)rintf(value_of(h, n) * inverse) : (int8_t)0;
    }
}

__global__ void __launch_bounds__(kRowThreads) dequant_rows_kernel(const DequantArgs a) {
    const int64_t m = blockIdx.x;
    const float scale = a.scale[m];
    for (int n = threadIdx.x; n < a.N; n += kRowThreads)
        store_number(a.y, m * a.ldy + n, a.out_f32, (float)a.q[m * a.ldq + n] * scale);
}

}  // namespace

hipError_t launch_quant_rows(const QuantArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(quant_rows_kernel, dim3((unsigned)a.M), dim3(kRowThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_dequant_rows(const DequantArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(dequant_rows_kernel, dim3((unsigned)a.M), dim3(kRowThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace dit
