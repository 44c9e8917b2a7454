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
        __syncthreads();
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

// Eight weights from column `col` on, n of them there.
template <bool WIDE>
__device__ __forceinline__ void load_weights(const void* w, int type, int col, int n, float* x) {
    if (type == VA_BF16) {
        to_float8(load8<WIDE>((const uint16_t*)w + col, n), x);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < n ? ((const float*)w)[col + e] : 0.f;
    }
}

template <int G, int NV, bool WIDE>
__global__ void __launch_bounds__(RowGroup<G>::THREADS) norm_fwd_kernel(NormArgs a) {
    using R = RowGroup<G>;
    __shared__ float lds[2][4][R::THREADS / 64];
    int at = 0;
    const int C = a.channels, lane = threadIdx.x % G;
    const int blocks = (C + kAct8Block - 1) / kAct8Block;
    for (int64_t base = (int64_t)blockIdx.x * R::ROWS; base < a.rows; base += (int64_t)gridDim.x * R::ROWS) {
        const int64_t row = base + threadIdx.x / G;
        const bool there = row < a.rows;
        const int64_t token = row / a.rows_per_token;
        const uint16_t* const x = (const uint16_t*)a.x + token * a.x_stride + (row % a.rows_per_token) * C;
        float h[NV][8];
        float sum[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = 8 * (lane + j * G), n = there ? C - col : 0;
            u32x4 w = load8<WIDE>(x + col, n);
            to_float8(w, h[j]);
            if (a.residual) {
                float r[8];
                to_float8(load8<WIDE>((const uint16_t*)a.residual + row * C + col, n), r);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[j][e] += r[e];
                w = to_bf16x8(h[j]);  // the stream goes on in bf16, and the norm is of what goes on
                store8<WIDE>((uint16_t*)a.summed + row * C + col, w, n);
                to_float8(w, h[j]);
            }
            if (a.format >= 0) {
                constexpr int L = R::LANES < 16 ? R::LANES : 16;
                const float s = act8_scale(lanes_max<L>(magnitude8(w)), a.format);
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
                if (e < n) sq[0] += h[j][e] * h[j][e];
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
            float w[8], b[8], y[8];
            if (a.weight) load_weights<WIDE>(a.weight, a.weight_type, col, n, w);
            if (a.bias) load_weights<WIDE>(a.bias, a.weight_type, col, n, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y[e] = h[j][e] * rstd;
                if (a.weight) y[e] *= w[e];
                if (a.bias) y[e] += b[e];
            }
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
    float dw[NV][8] = {}, db[NV][8] = {};
    for (int64_t base = (int64_t)blockIdx.x * R::ROWS; base < a.rows; base += (int64_t)gridDim.x * R::ROWS) {
        const int64_t row = base + threadIdx.x / G;
        const bool there = row < a.rows;
        const int64_t token = row / a.rows_per_token, inner = (row % a.rows_per_token) * C;
        const float mean = there ? a.mean[row] : 0.f, rstd = there ? a.rstd[row] : 0.f;
        float n[NV][8], g[NV][8];
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = 8 * (lane + j * G), left = there ? C - col : 0;
            if (FORMAT < 0) {
                to_float8(load8<WIDE>((const uint16_t*)a.x + token * a.x_stride + inner + col, left), n[j]);
            } else {
                const float s = left > 0 ? a.scales[row * blocks + col / kAct8Block] : 0.f;
                act8_decode(load_codes<WIDE>((const uint8_t*)a.codes + row * C + col, left), s, FORMAT, n[j]);
            }
            float dy[8];
            to_float8(load8<WIDE>((const uint16_t*)a.dy + token * a.dy_stride + inner + col, left), dy);
            float w[8];
            if (a.weight) load_weights<WIDE>(a.weight, a.weight_type, col, left, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                n[j][e] = e < left ? (n[j][e] - mean) * rstd : 0.f;
                g[j][e] = a.weight ? dy[e] * w[e] : dy[e];
                dw[j][e] += dy[e] * n[j][e];
                db[j][e] += dy[e];
                sum[0] += g[j][e];
                sum[1] += g[j][e] * n[j][e];
            }
        }
        row_sum<G>(sum, lds, at);
        const float c0 = sum[0] / (float)C, c1 = sum[1] / (float)C;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = 8 * (lane + j * G), left = there ? C - col : 0;
            float dx[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) dx[e] = rstd * (g[j][e] - c0 - n[j][e] * c1);
            if (a.dsummed) {
                float r[8];
                to_float8(load8<WIDE>((const uint16_t*)a.dsummed + row * C + col, left), r);
#pragma unroll
                for (int e = 0; e < 8; ++e) dx[e] += r[e];
            }
            store8<WIDE>((uint16_t*)a.dx + token * a.dx_stride + inner + col, to_bf16x8(dx), left);
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
        return;
    }
    for (int s = 0; s < R::ROWS; ++s) {
        if ((int)threadIdx.x / G == s) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at8 = ((j * 8 + e) * G + lane) % (R::ROWS > 1 ? 8 * NV * G : 1);
                    part[0][at8] = s ? part[0][at8] + dw[j][e] : dw[j][e];
                    part[1][at8] = s ? part[1][at8] + db[j][e] : db[j][e];
                }
        }
        __syncthreads();
    }
    for (int c = threadIdx.x; c < C; c += R::THREADS) {
        const int at8 = ((c / 8 / G) * 8 + c % 8) * G + c / 8 % G;
        out[c] = part[0][at8];
        out[C + c] = part[1][at8];
    }
}

// dw and db from the workgroups' partial sums [wgs, 2, C]: 32 columns a workgroup, 8 threads a column.
__global__ void __launch_bounds__(256) norm_sum_kernel(const float* __restrict__ partial, int wgs, int C, float* __restrict__ dweight,
                                                       float* __restrict__ dbias) {
    __shared__ float lds[8][32];
    const int c = blockIdx.x * 32 + threadIdx.x % 32, part = threadIdx.x / 32, which = blockIdx.y;
    float s = 0.f;
    if (c < C)
        for (int i = part; i < wgs; i += 8) s += partial[((size_t)i * 2 + which) * C + c];
    lds[part][threadIdx.x % 32] = s;
    __syncthreads();
    if (part == 0 && c < C) {
#pragma unroll
        for (int i = 1; i < 8; ++i) s += lds[i][threadIdx.x];
        (which ? dbias : dweight)[c] = s;
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

// Workgroups of the backward pass: what fits the chip at once, as long as there are rows.
int norm_bwd_wgs(int64_t rows, int C) {
    const int64_t r = norm_rows_per_wg(C);
    const int64_t wgs = (rows + r - 1) / r;
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
        hipLaunchKernelGGL(norm_sum_kernel, dim3((unsigned)((C + 31) / 32), 2), dim3(256), 0, stream, a.partial, wgs, C, a.dweight,
                           a.dbias);
    return hipGetLastError();
}

}  // namespace va
