// Projection of 8-bit rows: y[m, n] = (sum_k x[m, k] w[n, k]) * x_scale[m] * w_scale[n] + bias[n], the sum an exact 32-bit
// integer on the matrix cores.  Few token rows are done here, through LDS rings of each wavefront's own; more by the tiles of
// dit_linear.hip and dit_linear_small.hip, which take 8-bit operands at twice the contraction indices a step.
//
// What bounds the few rows' kernel: the stream of the weights.  From memory (as where a model's layers follow each other)
// 1 x 15,360 x 5,120 15 to 16.3 us, 4.8 to 5.2 TB/s, 16 x 5,120 x 20,480 25 us, 4.2 TB/s (a copy: 4.95); weights that the 256 MB
// cache still holds 12.6 to 13.2 us and 17.7 to 22.
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
// Eight wavefronts where a workgroup streams so few bytes that its own trips to memory are what it waits for: 1 x 40 x 16,912
// 4.9 us and with four 6.6, 113 x 96 x 12,928 5.8 and 6.4; with more features four are level or better (119 x 547 x 16,978
// in 16-row blocks 12.1 and 13.0).  (3 stages are level with 4 and better than 2 at 16 rows: 16 x 5,120 x 20,480 25 and 26; with
// more rows 2 leave room for two workgroups.)
template <int XI, int WI>
struct FewTile {
    static constexpr int NW = XI <= 2 && WI == 1 ? 8 : 4;
    static constexpr int S = XI == 1 || (XI == 2 && WI > 1) ? 3 : 2;
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

// How the blocks of F features and 8 XI rows lie over the workgroups.  One row block: a feature block each.  Several: each XCD
// (workgroups go round them one by one) takes `share` neighbours, along the shorter operand first, so that its L2 fetches the
// longer one once: 799 x 96 x 18,816 in blocks of 16 x 20 11.4 us and 16.0 without, 363 x 275 x 11,204 11.9 and 13.9, 41 x 1,974 x
// 3,622 5.8 and 7.4.
struct FewGrid {
    int F, blocks, share;
    int xcds, shift;  // 7 and 3, or 0 and 0 for one row block
    int along;        // blocks along the shorter operand
    uint32_t magic;   // 2^20 / along, rounded up: i * magic >> 20 is i / along for numbers below 2^10; 0 for one row block
    int rows_longer;
};

template <int XI, int WI, bool OUT_F32>
__global__ void __launch_bounds__((64 * FewTile<XI, WI>::NW)) linear_few_kernel(const LinearQuantArgs a, const FewGrid g) {
    using T = FewTile<XI, WI>;
    constexpr int TB = T::TB, FB = T::FB, NW = T::NW, S = T::S;
    const int F = g.F;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lr = lane & 15, lg = lane >> 4;
    // (Without a branch: the arguments behind one would be loaded behind it, 0.2 us.)
    int bn = blockIdx.x, bm = 0;
    bool surplus = false;
    if constexpr (XI > 1) {
        const int own = (blockIdx.x & g.xcds) * g.share + (blockIdx.x >> g.shift);
        surplus = own >= g.blocks;  // (the last block again, for nobody)
        const int i = surplus ? g.blocks - 1 : own;
        const int far = (int)(i * g.magic >> 20), near = i - far * g.along;
        bm = g.rows_longer ? far : near;
        bn = g.rows_longer ? near : far;
    }
    const int n0 = bn * F, n1 = n0 + F < a.N ? n0 + F : a.N;  // its features
    const int m0 = bm * (8 * XI), m1 = m0 + 8 * XI < a.M ? m0 + 8 * XI : a.M;  // and token rows

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
    for (int i = tid; i < (surplus ? 0 : 16 * FB * (m1 - m0)); i += 64 * NW) {
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

template <int XI, int WI, bool OUT_F32>
hipError_t launch_few(const LinearQuantArgs& a, int F, hipStream_t s) {
    using T = FewTile<XI, WI>;
    const auto kern = linear_few_kernel<XI, WI, OUT_F32>;
    static std::atomic<uint64_t> attr_set{0};
    const hipError_t e = allow_dynamic_lds(kern, T::LDS, attr_set);
    if (e != hipSuccess) return e;
    const int row_blocks = (a.M + 8 * XI - 1) / (8 * XI), feature_blocks = (a.N + F - 1) / F;
    FewGrid g{F, feature_blocks, 0, 0, 0, 1, 0, 1};
    if (row_blocks > 1) {
        g.blocks = row_blocks * feature_blocks;
        if (g.blocks >= 1 << 10) return hipErrorInvalidValue;
        g.share = (g.blocks + 7) / 8;
        g.xcds = 7;
        g.shift = 3;
        g.rows_longer = a.M > a.N;
        g.along = g.rows_longer ? feature_blocks : row_blocks;
        g.magic = ((1u << 20) + g.along - 1) / g.along;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)(g.share ? 8 * g.share : g.blocks)), dim3(64 * T::NW), T::LDS, s, a, g);
    return hipGetLastError();
}

template <int XI>
hipError_t launch_few(const LinearQuantArgs& a, int F, hipStream_t s) {
    switch ((F + 7) / 8) {
        case 1: return a.out_f32 ? launch_few<XI, 1, true>(a, F, s) : launch_few<XI, 1, false>(a, F, s);
        case 2: return a.out_f32 ? launch_few<XI, 2, true>(a, F, s) : launch_few<XI, 2, false>(a, F, s);
        case 3: return a.out_f32 ? launch_few<XI, 3, true>(a, F, s) : launch_few<XI, 3, false>(a, F, s);
        case 4: return a.out_f32 ? launch_few<XI, 4, true>(a, F, s) : launch_few<XI, 4, false>(a, F, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace

// The few rows' kernel: a workgroup a compute unit, of at most 32 features, so that all of them pull in the weights at the
// same rate; its row block the smallest that leaves so few.  Up to 16 rows two or three workgroups a unit pay too.  Else the
// tiles, which read the rows fewer times.  Measured, us, operands that change from call to call and come from memory, this
// kernel and the best tile: 1 x 20,480 x 5,120 (three workgroups a
// unit) 22 and 26; 1 x 15,360 x 5,120 16 and 18; 16 x 5,120 x 20,480 25 and 41; 32 x 5,120 x 5,120 7.8 and 10.5; 64 x 5,120 x
// 20,480 39 and 44; but 32 x 15,360 x 5,120 22 and 20, 64 x 15,360 x 5,120 29 and 24.  Blocks of 16 rows and up to 16 features:
// 113 x 96 x 12,928 5.8 and 18, 428 x 128 x 3,712 4.6 and 7.0, 33 x 41 x 14,220 5.6 and 22; with more features those of 32 rows
// are level or better (41 x 1,974 x 3,622 5.5 and 5.3, tile 9.1).  Of 32: 298 x 768 x 5,376 7.6 and 11, 37 x 2,775 x 18,763 18
// and 31.  Of 64, where K is long enough: 113 x 4,000 x 17,280 22 and 30, 1,281 x 237 x 3,155 9.2 and 9.7, but 782 x 544 x 1,792
// 6.9 and 6.2, 48 x 5,376 x 2,176 7.3 and 6.5.  Over 250 drawn sizes that it is chosen for (M 1 .. 2,900, N 16 .. 8,192, K 512 ..
// 20,000) it takes 0.46 of the tiles' time in the geometric mean, 0.15 at best and 1.00 at worst.
int choose_linear_quant(int M, int N, int K, int cus, int* rows, int* features) {
    *rows = *features = 0;
    for (int r = M <= 8 ? 8 : 16; r <= 64; r *= 2) {
        const int row_blocks = (int)(((int64_t)M + r - 1) / r);
        if (row_blocks > cus || (r == 64 && K < 3000)) continue;
        const int each = cus / row_blocks, f = (int)(((int64_t)N + each - 1) / each);
        if (f > (r == 16 && row_blocks > 1 ? 16 : 32)) continue;
        *rows = r;
        *features = f < 8 ? 8 : f;
        return 0;
    }
    const int64_t per = ((int64_t)N + 32 * cus - 1) / (32 * cus);  // workgroups a compute unit
    if (M <= 16 && per <= 3) {
        *rows = M <= 8 ? 8 : 16;
        *features = (int)((N + per * cus - 1) / (per * cus));
        return 0;
    }
    return choose_linear_form_i8(M, N, K, cus);
}

static hipError_t launch_slice(const LinearQuantArgs& q, int cus, hipStream_t s) {
    int rows, features;
    const int form = choose_linear_quant(q.M, q.N, q.K, cus, &rows, &features);
    switch (rows) {
        case 8: return launch_few<1>(q, features, s);
        case 16: return launch_few<2>(q, features, s);
        case 32: return launch_few<4>(q, features, s);
        case 64: return launch_few<8>(q, features, s);
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
    const hipError_t e = launch_linear_i8(a, form == 64 ? 192 : 256, s);
    if (e != hipSuccess || rest == 0) return e;
    a.w += (int64_t)a.N * a.ldw;
    a.w_scale += a.N;
    if (a.bias) a.bias += a.N;
    a.y = static_cast<uint8_t*>(a.y) + (int64_t)a.N * (a.out_f32 ? 4 : 2);
    a.N = rest;
    return launch_linear_small_i8(a, choose_linear_form_i8(a.M, a.N, q.K, cus), s);
}

// In slices of 2^30 rows and features: the kernels count both in 32 bits, to the ends of their tiles, and the narrowest outputs
// (under 8 features, 160 rows a tile) have no more tiles than a launch takes.
hipError_t launch_linear_quant(const LinearQuantArgs& q, hipStream_t s) {
    constexpr int kSlice = 1 << 30;
    int cus = 0;
    hipError_t e = compute_units(&cus);
    for (int64_t m = 0; m < q.M && e == hipSuccess; m += kSlice) {
        for (int64_t n = 0; n < q.N && e == hipSuccess; n += kSlice) {
            LinearQuantArgs a = q;
            a.x += m * q.ldx;
            a.x_scale += m;
            a.w += n * q.ldw;
            a.w_scale += n;
            if (a.bias) a.bias += n;
            a.y = static_cast<uint8_t*>(a.y) + (m * q.ldy + n) * (q.out_f32 ? 4 : 2);
            a.M = (int)(q.M - m < kSlice ? q.M - m : kSlice);
            a.N = (int)(q.N - n < kSlice ? q.N - n : kSlice);
            e = launch_slice(a, cus, s);
        }
    }
    return e;
}

}  // namespace dit
