// Layer norm of rows of C channels, forward and backward.
//     h = x (+ residual, rounded to bf16),  mu = sum h / C,  rstd = (sum (h - mu)^2 / C + eps)^-1/2,  y = (h - mu) rstd w + b
//     n = (h - mu) rstd,  g = dy w,  dx = rstd (g - sum g / C - n sum(g n) / C) (+ dsummed),  dw = sum_rows dy n,  db = sum_rows dy
// The sums are over the row as it lies in registers, the mean first and the squares of what is left then, in 32 bits: a row far
// off zero loses nothing.  The forward can leave h in 8 bits (va_ops.h) in the same pass, for the backward to read.
// Bound by memory: 4 to 12 bytes per channel against some 20 operations.
//
// G threads hold a row, NV runs of 8 channels each: run j of thread i are the channels 8 (i + j G)...  Threads of a workgroup
// beyond that take further rows.  A workgroup walks rows with the stride of the grid, so that weight and bias stay in registers,
// and in the backward pass the sums for dw and db do: every thread adds up its own channels over its rows, a workgroup adds its
// threads through LDS and leaves one row of partial sums, and a second kernel adds those.  No atomics: the same bits every time.
#include "va_internal.h"
#include "va_ops.h"

namespace va {

template <int G>
struct RowGroup {
    static constexpr int THREADS = G > 256 ? G : 256;
    static constexpr int ROWS = THREADS / G;        // rows a workgroup has in work at a time
    static constexpr int WAVES = G > 64 ? G / 64 : 1;
    static constexpr int LANES = G > 64 ? 64 : G;
};

// Sums of N values over the threads of a row.  `at` alternates between the two halves of `lds`, so that one barrier a sum is enough.
template <int G, int N>
__device__ __forceinline__ void row_sum(float (&x)[N], float (*lds)[4][RowGroup<G>::THREADS / 64], int& at) {
    using R = RowGroup<G>;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = lanes_sum<R::LANES>(x[i]);
    if constexpr (R::WAVES > 1) {
        const int wave = threadIdx.x / 64, first = wave / R::WAVES * R::WAVES;
        if (threadIdx.x % 64 == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) lds[at][i][wave] = x[i];
        }
        wg_barrier();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = lds[at][i][first];
#pragma unroll
            for (int w = 1; w < R::WAVES; ++w) s += lds[at][i][first + w];
            x[i] = s;
        }
        at ^= 1;
    }
}

// Eight values of weight or bias from column `col` on, n of them there, else `other`.
template <bool WIDE>
__device__ __forceinline__ void load_weights(const void* w, int type, int col, int n, float other, float* x) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = other;
    if (!w) return;
    if (type == VA_BF16) {
        to_float8(load8<WIDE>((const uint16_t*)w + col, n), x);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < n ? ((const float*)w)[col + e] : 0.f;
    }
}

// Where row `row` of a tensor with a stride between tokens starts.
__device__ __forceinline__ int64_t row_offset(const NormArgs& a, int64_t row, int64_t stride) {
    if (stride == (int64_t)a.rows_per_token * a.channels) return row * a.channels;
    if (a.rows_per_token == 1) return row * stride;
    if (a.rows <= INT32_MAX) {  // (a division in 64 bits is 100 instructions, on rows of as few as 8 channels a lane)
        const uint32_t r = (uint32_t)row, t = r / (uint32_t)a.rows_per_token;
        return t * stride + (int64_t)(r - t * (uint32_t)a.rows_per_token) * a.channels;
    }
    return row / a.rows_per_token * stride + row % a.rows_per_token * a.channels;
}

template <int G, int NV, bool WIDE>
__global__ void __launch_bounds__(RowGroup<G>::THREADS) norm_fwd_kernel(NormArgs a) {
    using R = RowGroup<G>;
    __shared__ float lds[2][4][R::THREADS / 64];
    int at = 0;
    const int C = a.channels, lane = threadIdx.x % G;
    const int blocks = (C + kAct8Block - 1) / kAct8Block;
    float w[NV][8], b[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int col = 8 * (lane + j * G);
        load_weights<WIDE>(a.weight, a.weight_type, col, C - col, 1.f, w[j]);
        load_weights<WIDE>(a.bias, a.weight_type, col, C - col, 0.f, b[j]);
    }
    const int64_t step = (int64_t)gridDim.x * R::ROWS;
    u32x4 xs[NV], rs[NV];
    auto fetch = [&](int64_t row) {
        const uint16_t* const x = (const uint16_t*)a.x + row_offset(a, row, a.x_stride);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = 8 * (lane + j * G), n = row < a.rows ? C - col : 0;
            xs[j] = load8<WIDE>(x + col, n);
            if (a.residual) rs[j] = load8<WIDE>((const uint16_t*)a.residual + row * C + col, n);
        }
    };
    int64_t row = (int64_t)blockIdx.x * R::ROWS + threadIdx.x / G;
    fetch(row);
    for (int64_t base = (int64_t)blockIdx.x * R::ROWS; base < a.rows; base += step, row += step) {
        const bool there = row < a.rows;
        float h[NV][8];
        u32x4 kept[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            kept[j] = xs[j];
            to_float8(xs[j], h[j]);
            if (a.residual) {
                float r[8];
                to_float8(rs[j], r);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[j][e] += r[e];
                kept[j] = to_bf16x8(h[j]);  // the stream goes on in bf16, and the norm is of what goes on
                to_float8(kept[j], h[j]);
            }
        }
        fetch(row + step);  // (in flight while this row is worked on)
        float sum[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = 8 * (lane + j * G), n = there ? C - col : 0;
            if (a.residual) store8<WIDE>((uint16_t*)a.summed + row * C + col, kept[j], n);
            if (a.format >= 0) {
                constexpr int L = R::LANES < 16 ? R::LANES : 16;
                const float s = act8_scale(lanes_max<L>(magnitude8(kept[j])), a.format);
                store_codes<WIDE>((uint8_t*)a.codes + row * C + col, act8_encode(h[j], s, a.format), n);
                if (lane % L == 0 && n > 0) a.scales[row * blocks + col / kAct8Block] = s;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[0] += h[j][e];
        }
        row_sum<G>(sum, lds, at);
        const float mean = sum[0] / (float)C;
        float sq[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int n = C - 8 * (lane + j * G);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[j][e] -= mean;
                const float d = (WIDE ? n > 0 : e < n) ? h[j][e] : 0.f;
                sq[0] += d * d;
            }
        }
        row_sum<G>(sq, lds, at);
        const float rstd = 1.f / sqrtf(sq[0] / (float)C + a.eps);
        if (there && lane == 0) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = 8 * (lane + j * G), n = there ? C - col : 0;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = h[j][e] * rstd * w[j][e] + b[j][e];
            store8<WIDE>((uint16_t*)a.y + row * C + col, to_bf16x8(y), n);
        }
    }
}

// FORMAT: -1 the row in bf16, else its 8-bit codes.
template <int G, int NV, bool WIDE, int FORMAT>
__global__ void __launch_bounds__(RowGroup<G>::THREADS) norm_bwd_kernel(NormArgs a) {
    using R = RowGroup<G>;
    __shared__ float lds[2][4][R::THREADS / 64];
    __shared__ float part[2][R::ROWS > 1 ? 8 * NV * G : 1];
    int at = 0;
    const int C = a.channels, lane = threadIdx.x % G;
    const int blocks = (C + kAct8Block - 1) / kAct8Block;
    float w[NV][8];
    float dw[NV][8] = {}, db[NV][8] = {};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int col = 8 * (lane + j * G);
        load_weights<WIDE>(a.weight, a.weight_type, col, C - col, 1.f, w[j]);
    }
    const int64_t step = (int64_t)gridDim.x * R::ROWS;
    struct Row {
        u32x4 x[NV], dy[NV];
        u32x2 codes[NV];
        float scale[NV], mean, rstd;
    } next;
    auto fetch = [&](int64_t row) {
        const bool there = row < a.rows;
        next.mean = there ? a.mean[row] : 0.f;
        next.rstd = there ? a.rstd[row] : 0.f;
        const uint16_t* const dy = (const uint16_t*)a.dy + row_offset(a, row, a.dy_stride);
        const uint16_t* const x = FORMAT < 0 ? (const uint16_t*)a.x + row_offset(a, row, a.x_stride) : nullptr;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = 8 * (lane + j * G), n = there ? C - col : 0;
            if constexpr (FORMAT < 0) {
                next.x[j] = load8<WIDE>(x + col, n);
            } else {
                next.scale[j] = n > 0 ? a.scales[row * blocks + col / kAct8Block] : 0.f;
                next.codes[j] = load_codes<WIDE>((const uint8_t*)a.codes + row * C + col, n);
            }
            next.dy[j] = load8<WIDE>(dy + col, n);
        }
    };
    int64_t row = (int64_t)blockIdx.x * R::ROWS + threadIdx.x / G;
    fetch(row);
    for (int64_t base = (int64_t)blockIdx.x * R::ROWS; base < a.rows; base += step, row += step) {
        const bool there = row < a.rows;
        const float mean = next.mean, rstd = next.rstd;
        float n[NV][8], g[NV][8];
        u32x4 ds[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if constexpr (FORMAT < 0) to_float8(next.x[j], n[j]);
            else act8_decode(next.codes[j], next.scale[j], FORMAT, n[j]);
            to_float8(next.dy[j], g[j]);
        }
        fetch(row + step);  // (in flight while this row is worked on)
        if (a.dsummed) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int col = 8 * (lane + j * G);
                ds[j] = load8<WIDE>((const uint16_t*)a.dsummed + row * C + col, there ? C - col : 0);
            }
        }
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int left = C - 8 * (lane + j * G);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float dy = g[j][e];
                n[j][e] = (WIDE ? left > 0 : e < left) ? (n[j][e] - mean) * rstd : 0.f;
                g[j][e] = dy * w[j][e];
                dw[j][e] += dy * n[j][e];
                db[j][e] += dy;
                sum[0] += g[j][e];
                sum[1] += g[j][e] * n[j][e];
            }
        }
        row_sum<G>(sum, lds, at);
        const float c0 = sum[0] / (float)C, c1 = sum[1] / (float)C;
        uint16_t* const out = (uint16_t*)a.dx + row_offset(a, row, a.dx_stride);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = 8 * (lane + j * G), left = there ? C - col : 0;
            float dx[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) dx[e] = rstd * (g[j][e] - c0 - n[j][e] * c1);
            if (a.dsummed) {
                float r[8];
                to_float8(ds[j], r);
#pragma unroll
                for (int e = 0; e < 8; ++e) dx[e] += r[e];
            }
            store8<WIDE>(out + col, to_bf16x8(dx), left);
        }
    }
    if (!a.weight) return;
    // One row of partial sums per workgroup, its row groups added one after the other.
    float* const out = a.partial + (size_t)blockIdx.x * 2 * C;
    if constexpr (R::ROWS == 1) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int c = 8 * (lane + j * G) + e;
                if (c < C) { out[c] = dw[j][e]; out[C + c] = db[j][e]; }
            }
    } else {
        for (int s = 0; s < R::ROWS; ++s) {
            if ((int)threadIdx.x / G == s) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int i = (j * 8 + e) * G + lane;
                        part[0][i] = s ? part[0][i] + dw[j][e] : dw[j][e];
                        part[1][i] = s ? part[1][i] + db[j][e] : db[j][e];
                    }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < C; c += R::THREADS) {
            const int i = ((c / 8 / G) * 8 + c % 8) * G + c / 8 % G;
            out[c] = part[0][i];
            out[C + c] = part[1][i];
        }
    }
}

// dw and db from the workgroups' partial sums [wgs, 2 C]: 32 columns a workgroup, 32 threads a column.
__global__ void __launch_bounds__(1024) norm_sum_kernel(const float* __restrict__ partial, int wgs, int C, float* __restrict__ dweight,
                                                        float* __restrict__ dbias) {
    __shared__ float lds[32][33];
    const int x = threadIdx.x % 32, y = threadIdx.x / 32, c = blockIdx.x * 32 + x;
    float s = 0.f;
    if (c < 2 * C) {
#pragma unroll 8
        for (int i = y; i < wgs; i += 32) s += partial[(size_t)i * 2 * C + c];
    }
    lds[y][x] = s;
    __syncthreads();
    if (y == 0 && c < 2 * C) {
#pragma unroll
        for (int i = 1; i < 32; ++i) s += lds[i][x];
        if (c < C) dweight[c] = s;
        else dbias[c - C] = s;
    }
}

static bool norm_wide(const NormArgs& a) {
    const uint64_t bits = (uint64_t)(uintptr_t)a.x | (uintptr_t)a.residual | (uintptr_t)a.y | (uintptr_t)a.summed | (uintptr_t)a.dy |
                          (uintptr_t)a.dsummed | (uintptr_t)a.dx | (uintptr_t)a.weight | (uintptr_t)a.bias | 2 * (uintptr_t)a.codes |
                          2 * (uint64_t)(a.x_stride | a.dy_stride | a.dx_stride | a.channels);
    return bits % 16 == 0;
}

// Threads a row and runs a thread: rows of up to 2048 channels stay in one wave, whose sums need no barrier.
#define VA_NORM_SHAPES(GO) \
    if (C <= 64) GO(8, 1) else if (C <= 128) GO(16, 1) else if (C <= 256) GO(32, 1) else if (C <= 512) GO(64, 1) \
    else if (C <= 1024) GO(64, 2) else if (C <= 1536) GO(64, 3) else if (C <= 2048) GO(64, 4) else if (C <= 4096) GO(256, 2) \
    else if (C <= 8192) GO(256, 4) else GO(1024, 2)

static int norm_rows_per_wg(int C) {
#define VA_NORM_GO(G, NV) return RowGroup<G>::ROWS;
    VA_NORM_SHAPES(VA_NORM_GO)
#undef VA_NORM_GO
}

// Workgroups of the backward pass: up to what fits the chip at once, with four rows a thread group as soon as every CU has one.
int norm_bwd_wgs(int64_t rows, int C) {
    const int64_t r = norm_rows_per_wg(C), one = (rows + r - 1) / r, four = (rows + 4 * r - 1) / (4 * r);
    const int64_t wgs = four > 256 ? four : one < 256 ? one : 256;
    return (int)(wgs < 1024 ? wgs : 1024);
}

hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t stream) {
    const int C = a.channels;
    const bool wide = norm_wide(a);
    const int64_t r = norm_rows_per_wg(C), want = (a.rows + r - 1) / r;
    const dim3 grid((unsigned)(want < 2048 ? want : 2048));
#define VA_NORM_GO(G, NV)                                                                                                     \
    {                                                                                                                         \
        if (wide) hipLaunchKernelGGL((norm_fwd_kernel<G, NV, true>), grid, dim3(RowGroup<G>::THREADS), 0, stream, a);          \
        else hipLaunchKernelGGL((norm_fwd_kernel<G, NV, false>), grid, dim3(RowGroup<G>::THREADS), 0, stream, a);              \
    }
    VA_NORM_SHAPES(VA_NORM_GO)
#undef VA_NORM_GO
    return hipGetLastError();
}

hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t stream) {
    const int C = a.channels;
    const bool wide = norm_wide(a);
    const int wgs = norm_bwd_wgs(a.rows, C);
    if (wgs) {
        const dim3 grid((unsigned)wgs);
#define VA_NORM_BWD(G, NV, WIDE, FORMAT) \
    hipLaunchKernelGGL((norm_bwd_kernel<G, NV, WIDE, FORMAT>), grid, dim3(RowGroup<G>::THREADS), 0, stream, a)
#define VA_NORM_FORMAT(G, NV, WIDE)                                                  \
    if (a.format < 0) VA_NORM_BWD(G, NV, WIDE, -1);                                  \
    else if (a.format == VA_ACT8_INT8) VA_NORM_BWD(G, NV, WIDE, VA_ACT8_INT8);       \
    else VA_NORM_BWD(G, NV, WIDE, VA_ACT8_E4M3);
#define VA_NORM_GO(G, NV) { if (wide) { VA_NORM_FORMAT(G, NV, true) } else { VA_NORM_FORMAT(G, NV, false) } }
        VA_NORM_SHAPES(VA_NORM_GO)
#undef VA_NORM_GO
#undef VA_NORM_FORMAT
#undef VA_NORM_BWD
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.weight)
        hipLaunchKernelGGL(norm_sum_kernel, dim3((unsigned)((2 * C + 31) / 32)), dim3(1024), 0, stream, a.partial, wgs, C, a.dweight,
                           a.dbias);
    return hipGetLastError();
}

}  // namespace va
