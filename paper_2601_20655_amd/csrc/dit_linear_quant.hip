// Projection of 8-bit rows: y[m, n] = (sum_k x[m, k] w[n, k]) * x_scale[m] * w_scale[n] + bias[n], the sum an exact 32-bit
// integer on the matrix cores.  Few token rows are done here, straight from memory; more by the tiles of dit_linear.hip and
// dit_linear_small.hip, which take 8-bit operands at twice the contraction indices a step.
//
// What bounds the few rows' kernel: the stream of the weights.  1 x 15,360 x 5,120 12.6 us, 6.2 TB/s; 16 x 5,120 x 20,480
// 21.9 us, 4.8 TB/s (a copy: 4.95).
#include "dit_attn_device.h"
#include "dit_attn_internal.h"

namespace dit {

namespace {

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

typedef const __attribute__((address_space(1))) void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;

// Few token rows, or few tiles of a long sum: a workgroup takes 8 XI rows and F features, WI groups of 8 (the last one may be
// cut); its NW wavefronts share K in blocks of 128 bytes, one after the other, and add their sums at the end.  A wavefront
// streams its blocks through S stages of LDS of its own: the load-to-LDS DMA moves 8 rows of a block an instruction, whole
// lines, and no wavefront waits for another before the end.
template <int XI, int WI, int NW, int S>
struct FewTile {
    static constexpr int TB = (XI + 1) / 2, FB = (WI + 1) / 2;  // 16-token and 16-feature blocks
    static constexpr int LOADS = WI + XI;                       // DMA instructions of a block
    static constexpr int STAGE = 2048 * (FB + TB);
    static constexpr int RING = NW * S * STAGE, SUMS = NW * FB * TB * 1024;
    static constexpr int LDS = RING > SUMS ? RING : SUMS;
};

// the FB + TB fragments of one half block, waited for
template <int N>
__device__ __forceinline__ void read_fragments(u32x4 (&f)[N], uint32_t at) {
    static_assert(N >= 2 && N <= 6, "fragments of a half block");
    if constexpr (N == 2) {
        asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %2 offset:2048\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(f[0]), "=&v"(f[1]) : "v"(at) : "memory");
    } else if constexpr (N == 3) {
        asm volatile("ds_read_b128 %0, %3\n\tds_read_b128 %1, %3 offset:2048\n\tds_read_b128 %2, %3 offset:4096\n\t"
                     "s_waitcnt lgkmcnt(0)" : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]) : "v"(at) : "memory");
    } else if constexpr (N == 4) {
        asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:2048\n\tds_read_b128 %2, %4 offset:4096\n\t"
                     "ds_read_b128 %3, %4 offset:6144\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]) : "v"(at) : "memory");
    } else if constexpr (N == 5) {
        asm volatile("ds_read_b128 %0, %5\n\tds_read_b128 %1, %5 offset:2048\n\tds_read_b128 %2, %5 offset:4096\n\t"
                     "ds_read_b128 %3, %5 offset:6144\n\tds_read_b128 %4, %5 offset:8192\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]), "=&v"(f[4]) : "v"(at) : "memory");
    } else {
        asm volatile("ds_read_b128 %0, %6\n\tds_read_b128 %1, %6 offset:2048\n\tds_read_b128 %2, %6 offset:4096\n\t"
                     "ds_read_b128 %3, %6 offset:6144\n\tds_read_b128 %4, %6 offset:8192\n\t"
                     "ds_read_b128 %5, %6 offset:10240\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]), "=&v"(f[4]), "=&v"(f[5]) : "v"(at) : "memory");
    }
}

template <int XI, int WI, int NW, int S, bool OUT_F32>
__global__ void __launch_bounds__(64 * NW) linear_few_kernel(const LinearQuantArgs a, int F) {
    using T = FewTile<XI, WI, NW, S>;
    constexpr int TB = T::TB, FB = T::FB;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lr = lane & 15, lg = lane >> 4;
    const int n0 = blockIdx.x * F, n1 = n0 + F < a.N ? n0 + F : a.N;  // its features
    const int m0 = blockIdx.y * (8 * XI), m1 = m0 + 8 * XI < a.M ? m0 + 8 * XI : a.M;  // and token rows

    // DMA sources: 8 rows of 128 bytes an instruction.  LDS is filled in lane order, so the bank swizzle (piece p of row r in slot
    // p ^ ((r >> 1) & 7)) is in which piece a lane fetches.  Rows past the end are the last one again (their sums are not
    // stored); groups of 8 token rows that do not exist are not fetched.
    const int8_t* src[T::LOADS];
#pragma unroll
    for (int i = 0; i < T::LOADS; ++i) {
        const int r = 8 * (i < WI ? i : i - WI) + (lane >> 3);
        const int row = i < WI ? (n0 + r < n1 ? n0 + r : n1 - 1) : (m0 + r < m1 ? m0 + r : m1 - 1);
        src[i] = (i < WI ? a.w + (int64_t)row * a.ldw : a.x + (int64_t)row * a.ldx) + 16 * ((lane & 7) ^ ((r >> 1) & 7));
    }
    const int whole = a.K >> 7;
    const int mine = whole > wave ? (whole - wave + NW - 1) / NW : 0;  // blocks wave, wave + NW, ..
    uint8_t* const ring = smem + wave * (S * T::STAGE);
    auto request = [&](int j, int stage) __attribute__((always_inline)) {  // past the end: the last one again, for nobody
        const int at = 128 * (wave + NW * (j < mine ? j : mine - 1));
#pragma unroll
        for (int i = 0; i < T::LOADS; ++i)
            __builtin_amdgcn_global_load_lds((gptr_t)(src[i] + at), (lptr_t)(ring + stage * T::STAGE + 1024 * (i < WI ? i : 2 * FB + i - WI)), 16,
                                             0, 0);
    };
    // w rows ride the A operand of v_mfma_i32_16x16x64_i8, token rows the B operand: a lane (i, g) supplies 16 bytes of row i and
    // ends with token i, features 4 g .. 4 g + 3
    i32x4 acc[FB][TB];
#pragma unroll
    for (int fb = 0; fb < FB; ++fb)
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) acc[fb][tb] = i32x4{0, 0, 0, 0};
    const uint32_t lds0 = (uint32_t)(uintptr_t)ring + lr * 128 + 16 * (lg ^ ((lr >> 1) & 7));
    if (mine > 0) {
#pragma unroll
        for (int j = 0; j < S - 1; ++j) request(j, j);
        int stage = 0, free_stage = S - 1;
        for (int j = 0; j < mine; ++j) {
            // (the stage read in the step before: its fragments have been waited for)
            request(j + S - 1, free_stage);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 1) * T::LOADS) : "memory");
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 f[FB + TB];
                read_fragments(f, (lds0 + stage * T::STAGE) ^ (64 * h));
#pragma unroll
                for (int fb = 0; fb < FB; ++fb)
#pragma unroll
                    for (int tb = 0; tb < TB; ++tb) acc[fb][tb] = mfma16_i8(f[fb], f[FB + tb], acc[fb][tb]);
            }
            free_stage = stage;
            stage = stage + 1 == S ? 0 : stage + 1;
        }
    }
    if ((a.K & 127) && wave == whole % NW) {  // what is left behind the whole blocks is one wavefront's
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = whole * 128 + 64 * h + 16 * lg;
            u32x4 x[TB];
#pragma unroll
            for (int tb = 0; tb < TB; ++tb)
                x[tb] = load_cut_piece(a.x + (int64_t)(m0 + 16 * tb + lr < m1 ? m0 + 16 * tb + lr : m1 - 1) * a.ldx, at, a.K);
#pragma unroll
            for (int fb = 0; fb < FB; ++fb) {
                const int n = n0 + 16 * fb + lr;
                const u32x4 w = load_cut_piece(a.w + (int64_t)(n < n1 ? n : n1 - 1) * a.ldw, at, a.K);
#pragma unroll
                for (int tb = 0; tb < TB; ++tb) acc[fb][tb] = mfma16_i8(w, x[tb], acc[fb][tb]);
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (the loads for nobody)
    __syncthreads();
    i32x4* const part = reinterpret_cast<i32x4*>(smem);  // [wave][fb][tb][lane]
#pragma unroll
    for (int fb = 0; fb < FB; ++fb)
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) part[((wave * FB + fb) * TB + tb) * 64 + lane] = acc[fb][tb];
    __syncthreads();
    for (int i = tid; i < 16 * FB * (m1 - m0); i += 64 * NW) {
        const int r = i / (16 * FB), f = i % (16 * FB), m = m0 + r, n = n0 + f;
        if (n >= n1) continue;
        const int at = (f >> 4) * TB + (r >> 4), l = 16 * ((f & 15) >> 2) + (r & 15);
        int sum = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) sum += part[(w * FB * TB + at) * 64 + l][f & 3];
        const float y = fmaf((float)sum * a.x_scale[m], a.w_scale[n], a.bias ? __uint_as_float((uint32_t)a.bias[n] << 16) : 0.f);
        const int64_t o = (int64_t)m * a.ldy + n;
        if constexpr (OUT_F32) static_cast<float*>(a.y)[o] = y;
        else static_cast<uint16_t*>(a.y)[o] = (uint16_t)pack2<OP_BF16>(y, 0.f);
    }
}

template <int XI, int WI, int NW, int S, bool OUT_F32>
hipError_t launch_few(const LinearQuantArgs& a, int F, hipStream_t s) {
    constexpr int smem = FewTile<XI, WI, NW, S>::LDS;
    const auto kern = linear_few_kernel<XI, WI, NW, S, OUT_F32>;
    static std::atomic<uint64_t> attr_set{0};
    const hipError_t e = allow_dynamic_lds(kern, smem, attr_set);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)((a.N + F - 1) / F), (unsigned)((a.M + 8 * XI - 1) / (8 * XI))), dim3(64 * NW), smem, s,
                       a, F);
    return hipGetLastError();
}

template <int XI, int NW, int S>
hipError_t launch_few(const LinearQuantArgs& a, int F, hipStream_t s) {
    switch ((F + 7) / 8) {
        case 1: return a.out_f32 ? launch_few<XI, 1, NW, S, true>(a, F, s) : launch_few<XI, 1, NW, S, false>(a, F, s);
        case 2: return a.out_f32 ? launch_few<XI, 2, NW, S, true>(a, F, s) : launch_few<XI, 2, NW, S, false>(a, F, s);
        case 3: return a.out_f32 ? launch_few<XI, 3, NW, S, true>(a, F, s) : launch_few<XI, 3, NW, S, false>(a, F, s);
        case 4: return a.out_f32 ? launch_few<XI, 4, NW, S, true>(a, F, s) : launch_few<XI, 4, NW, S, false>(a, F, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace

// Few rows: as many workgroups as there are compute units, or twice as many, so that all of them pull the weights in at the same
// rate, and at most 32 features each.  Past 16 rows, and with more features, the tiles read the token rows fewer times.
// Measured, us, this kernel and the best tile: 1 x 20,480 x 5,120 (three workgroups a unit) 22 and 26; 1 x 15,360 x 5,120 16 and 18;
// 16 x 5,120 x 20,480 25 and 41; 32 x 5,120 x 5,120 7.8 and 10.5; 64 x 5,120 x 20,480 39 and 44; but 32 x 15,360 x 5,120 22 and 20,
// 64 x 15,360 x 5,120 29 and 24.
// More rows go there too, in blocks of 32 rows x 32 features, where those are no more than the compute units: a long sum is then
// shared by four wavefronts and streams deeper than in a tile.  300 x 300 x 300 4.1 and 4.7, 298 x 768 x 5,376 7.6 and 11.2,
// 1,049 x 26 x 9,426 10 and 17, 191 x 640 x 18,048 16 and 27; of 90 drawn sizes none loses more than 4 %.  Past that number the
// tiles win: 859 x 320 x 2,688 (270 blocks) 9.1 and 7.2, 1,863 x 129 x 3,368 (295) 12.7 and 10.3.
int choose_linear_quant(int M, int N, int K, int cus, int* features) {
    const int64_t per = ((int64_t)N + 32 * cus - 1) / (32 * cus);  // workgroups a compute unit
    *features = 0;
    if (M <= 16 ? per <= 3 : M <= 64 && per == 1) {
        const int f = (int)((N + per * cus - 1) / (per * cus));
        *features = f < 8 ? 8 : f;
        return 0;
    }
    if (M > 64 && (int64_t)((M + 31) / 32) * ((N + 31) / 32) <= cus) {
        *features = N < 32 ? (N + 7) / 8 * 8 : 32;
        return 0;
    }
    return choose_linear_form_i8(M, N, K, cus);
}

hipError_t launch_linear_quant(const LinearQuantArgs& q, hipStream_t s) {
    int cus = 0;
    hipError_t e = compute_units(&cus);
    if (e != hipSuccess) return e;
    int features;
    const int form = choose_linear_quant(q.M, q.N, q.K, cus, &features);
    if (features) {
        // (3 stages are level with 4 and better than 2 at 16 rows: 25 and 26 us; with more rows 2 leave room for two workgroups)
        if (q.M <= 8) return launch_few<1, 4, 3>(q, features, s);
        if (q.M <= 16) return launch_few<2, 4, 3>(q, features, s);
        if (q.M <= 32 || q.M > 64) return launch_few<4, 4, 2>(q, features, s);
        return launch_few<8, 4, 2>(q, features, s);
    }
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
    if (form && form != 64) return launch_linear_small_i8(a, form, s);
    // 256 x 256 tiles store whole 16-byte pieces: the last N % 8 features are a call of their own
    const int rest = a.N % 8;
    a.N -= rest;
    e = launch_linear_i8(a, form == 64 ? 192 : 256, s);
    if (e != hipSuccess || rest == 0) return e;
    a.w += (int64_t)a.N * a.ldw;
    a.w_scale += a.N;
    if (a.bias) a.bias += a.N;
    a.y = static_cast<uint8_t*>(a.y) + (int64_t)a.N * (a.out_f32 ? 4 : 2);
    a.N = rest;
    return launch_linear_small_i8(a, choose_linear_form_i8(a.M, a.N, q.K, cus), s);
}

}  // namespace dit
