// Layer norm of rows of C channels, forward and backward.
//     h = x (+ residual, rounded to bf16),  mu = sum h / C,  rstd = (sum (h - mu)^2 / C + eps)^-1/2,  y = (h - mu) rstd w + b
//     n = (h - mu) rstd,  g = dy w,  dx = rstd (g - sum g / C - n sum(g n) / C) (+ dsummed),  dw = sum_rows dy n,  db = sum_rows dy
// The sums are over the row as it lies in registers, the mean first and the squares of what is left then, in 32 bits: a row far
// off zero loses nothing.  The forward can leave h in 8 bits (va_ops.h) in the same pass, for the backward to read.
// Bound by memory: 4 to 9 bytes per channel against some 10 operations forward and 15 backward.  What the counters read and write is
// what the formulas need.  Forward / backward: 178572 x 1024 with residual 251 / 261 us (5.8 / 5.6 TB/s), 65537 x 1280 with and from
// int8 72 / 82 us (5.8 / 5.2: half of the vector unit's issue slots), 32768 x 32 heads of 128 92 / 144 us (5.8 / 5.6).
//
// G threads hold a row, NV runs of 8 channels each: run j of thread i are the channels 8 (i + j G)...  Threads of a workgroup
// beyond that take further rows.  A workgroup walks rows with the stride of the grid, so that weight and bias are brought into LDS
// once, and the sums for dw and db stay in registers: every thread adds up its own channels over its rows, a workgroup adds its
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
    // Which of the workgroup's rows this thread works on.  Where a whole wave shares it, a scalar: then a row's addresses are, too.
    __device__ __forceinline__ static int row_in_wg() { return G >= 64 ? uniform_wave_id() / WAVES : (int)threadIdx.x / G; }
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

// s / C and v^-1/2 without the library's care for the ends of the range, which is 45 instructions a row beside the 130 of a thread with 8
// channels of it (32768 x 32 heads of 80, forward / backward, 75.5 / 111.5 -> 73.2 / 103.2 us).  The quotient is corrected by its
// remainder (exact where the true one is), the root by one Newton step, to within 2^-23 of it; numbers that this is not for take the
// long way.
__device__ __forceinline__ float over(float s, float c, float inv_c) {
    const float q = s * inv_c;
    return fabsf(q) < INFINITY ? fmaf(fmaf(-q, c, s), inv_c, q) : q;
}
__device__ __forceinline__ float inverse_root(float v) {
    if (!(v >= 0x1p-100f && v <= 0x1p100f)) return 1.f / sqrtf(v);
    const float y = __builtin_amdgcn_rsqf(v), half = 0.5f * y;
    return fmaf(half, fmaf(-v * y, y, 1.f), y);
}

// Weight or bias in fp32 in LDS, as threads of a row read them: 16 bytes a thread, neighbours side by side.  (In registers they
// cost 8 a run and with that a wave per SIMD or two, which is bytes in flight.)
template <int G, int NV>
struct Weights {
    float4 x[NV * 2 * G];
    // `w`, or `other` everywhere without one, and zeros behind the row's end; a barrier has to follow.
    template <int MODE>
    __device__ __forceinline__ void fill(const void* w, int type, int C, float other) {
        for (int i = threadIdx.x; i < NV * G; i += RowGroup<G>::THREADS) {
            const int n = C - 8 * i;
            float v[8];
            if (w && type == VA_BF16) {
                to_float8(load8<MODE>((const uint16_t*)w + 8 * i, n), v);
            } else if (w && n >= 8) {
                typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
                const f32x4_any lo = *(const f32x4_any*)((const float*)w + 8 * i), hi = *(const f32x4_any*)((const float*)w + 8 * i + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) { v[e] = lo[e]; v[4 + e] = hi[e]; }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = e >= n ? 0.f : w ? ((const float*)w)[8 * i + e] : other;
            }
            const int at = i / G * 2 * G + i % G;
            x[at] = float4{v[0], v[1], v[2], v[3]};
            x[at + G] = float4{v[4], v[5], v[6], v[7]};
        }
    }
    __device__ __forceinline__ void get(int j, int lane, float* v) const {
        const float4 a = x[2 * j * G + lane], b = x[(2 * j + 1) * G + lane];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
};

// A thread's row and where it starts: in tensors whose rows lie one after the other, and in N with a stride between tokens.  All of it
// moves on by additions; with products and a division a row the forward of q's heads inside the projection (32768 x 32 of 128) took 97.5
// us instead of 92.9, the backward of 65537 x 1280 93.0 instead of 89.8.
template <int N>
struct RowPlace {
    int64_t row, flat, at[N];
    uint32_t inner;  // which of its token's rows
};
template <int N>
struct RowWalk {
    int64_t step, by_flat, by[N], wrap[N];
    uint32_t by_inner, rows_per_token;  // (unsigned: up to 2^31 - 1 rows a token and a step's rows do not fit 31 bits together)
    // step and first are below 2^31: rows of one round of the grid
    __device__ __forceinline__ RowPlace<N> begin(const NormArgs& a, int64_t first, int64_t step_, const int64_t (&stride)[N]) {
        const uint32_t rpt = (uint32_t)a.rows_per_token, f = (uint32_t)first, s = (uint32_t)step_;
        const uint32_t token = rpt == 1 ? f : f / rpt, tokens = rpt == 1 ? s : s / rpt;
        const int C = a.channels;
        rows_per_token = rpt;
        step = step_;
        by_flat = step * C;
        by_inner = s - tokens * rpt;
        RowPlace<N> p;
        p.row = first;
        p.flat = first * C;
        p.inner = f - token * rpt;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            p.at[i] = token * stride[i] + (int64_t)p.inner * C;
            by[i] = tokens * stride[i] + (int64_t)by_inner * C;
            wrap[i] = stride[i] - (int64_t)rows_per_token * C;
        }
        return p;
    }
    __device__ __forceinline__ void advance(RowPlace<N>& p) const {
        p.row += step;
        p.flat += by_flat;
        p.inner += by_inner;
        const bool wrapped = p.inner >= rows_per_token;
        p.inner -= wrapped ? rows_per_token : 0;
#pragma unroll
        for (int i = 0; i < N; ++i) p.at[i] += by[i] + (wrapped ? wrap[i] : 0);
    }
};

template <int G, int NV, int MODE>
__global__ void __launch_bounds__(RowGroup<G>::THREADS) norm_fwd_kernel(NormArgs a) {
    using R = RowGroup<G>;
    __shared__ float lds[2][4][R::THREADS / 64];
    __shared__ Weights<G, NV> weight, bias;
    int at = 0;
    const int C = a.channels, lane = threadIdx.x % G;
    const float inv_c = 1.f / (float)C;
    const int blocks = (C + kAct8Block - 1) / kAct8Block;
    const int64_t step = (int64_t)gridDim.x * R::ROWS;
    u32x4 xs[NV], rs[NV];
    RowWalk<1> walk;
    RowPlace<1> next = walk.begin(a, (int64_t)blockIdx.x * R::ROWS + R::row_in_wg(), step, {a.x_stride});
    auto fetch = [&]() {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = 8 * (lane + j * G), n = next.row < a.rows ? C - col : 0;
            xs[j] = load8<MODE>((const uint16_t*)a.x + next.at[0] + col, n);
            if (a.residual) rs[j] = load8<MODE>((const uint16_t*)a.residual + next.flat + col, n);
        }
    };
    fetch();
    weight.template fill<MODE>(a.weight, a.weight_type, C, 1.f);
    bias.template fill<MODE>(a.bias, a.weight_type, C, 0.f);
    __syncthreads();
    for (int64_t base = (int64_t)blockIdx.x * R::ROWS; base < a.rows; base += step) {
        const int64_t row = next.row, flat = next.flat;
        const bool there = row < a.rows;
        float h[NV][8];
        float sum[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = 8 * (lane + j * G), n = there ? C - col : 0;
            u32x4 kept = xs[j];
            to_float8(kept, h[j]);
            if (a.residual) {
                float r[8];
                to_float8(rs[j], r);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[j][e] += r[e];
                kept = to_bf16x8(h[j]);  // the stream goes on in bf16, and the norm is of what goes on
                to_float8(kept, h[j]);
                store8<MODE>((uint16_t*)a.summed + flat + col, kept, n);
            }
            if (a.format >= 0) {
                constexpr int L = R::LANES < 16 ? R::LANES : 16;
                const float s = act8_scale(lanes_max<L>(magnitude8(kept)), a.format);
                // (through the caches: 8 bytes a thread are half a line a wave at the row's end; 5.07 -> 5.36 TB/s at 1280 channels)
                store_codes<MODE == STREAM ? WIDE : MODE>((uint8_t*)a.codes + flat + col, act8_encode(h[j], s, a.format), n);
                if (lane % L == 0 && n > 0) a.scales[row * blocks + col / kAct8Block] = s;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[0] += h[j][e];
        }
        walk.advance(next);
        fetch();  // (in flight while this row is worked on)
        row_sum<G>(sum, lds, at);
        const float mean = over(sum[0], (float)C, inv_c);
        float sq[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int n = C - 8 * (lane + j * G);
            float run = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[j][e] -= mean;
                const float d = MODE != RAGGED || e < n ? h[j][e] : 0.f;
                run += d * d;
            }
            sq[0] += n > 0 ? run : 0.f;
        }
        row_sum<G>(sq, lds, at);
        const float rstd = inverse_root(over(sq[0], (float)C, inv_c) + a.eps);
        if (there && lane == 0) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = 8 * (lane + j * G), n = there ? C - col : 0;
            float y[8], w[8], b[8];
            weight.get(j, lane, w);
            bias.get(j, lane, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = h[j][e] * rstd * w[e] + b[e];
            store8<MODE>((uint16_t*)a.y + flat + col, to_bf16x8(y), n);
        }
    }
}

// FORMAT: -1 the row in bf16, else its 8-bit codes.
template <int G, int NV, int MODE, int FORMAT>
__global__ void __launch_bounds__(RowGroup<G>::THREADS) norm_bwd_kernel(NormArgs a) {
    using R = RowGroup<G>;
    __shared__ float lds[2][4][R::THREADS / 64];
    __shared__ union {
        Weights<G, NV> weight;
        float part[2][R::ROWS > 1 ? 8 * NV * G : 1];  // (behind the last row)
    } u;
    int at = 0;
    const int C = a.channels, lane = threadIdx.x % G;
    const float inv_c = 1.f / (float)C;
    const int blocks = (C + kAct8Block - 1) / kAct8Block;
    float dw[NV][8] = {}, db[NV][8] = {};
    const int64_t step = (int64_t)gridDim.x * R::ROWS;
    struct Row {
        u32x4 x[NV], dy[NV];
        u32x2 codes[NV];
        float scale[NV], mean, rstd;
    } next;
    RowWalk<3> walk;  // x, dy, dx
    RowPlace<3> place = walk.begin(a, (int64_t)blockIdx.x * R::ROWS + R::row_in_wg(), step, {a.x_stride, a.dy_stride, a.dx_stride});
    auto fetch = [&]() {
        const int64_t row = place.row;
        const bool there = row < a.rows;
        next.mean = there ? a.mean[row] : 0.f;
        next.rstd = there ? a.rstd[row] : 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = 8 * (lane + j * G), n = there ? C - col : 0;
            if constexpr (FORMAT < 0) {
                next.x[j] = load8<MODE>((const uint16_t*)a.x + place.at[0] + col, n);
            } else {
                next.scale[j] = n > 0 ? a.scales[row * blocks + col / kAct8Block] : 0.f;
                next.codes[j] = load_codes<MODE>((const uint8_t*)a.codes + place.flat + col, n);
            }
            next.dy[j] = load8<MODE>((const uint16_t*)a.dy + place.at[1] + col, n);
        }
    };
    fetch();
    u.weight.template fill<MODE>(a.weight, a.weight_type, C, 1.f);
    __syncthreads();
    for (int64_t base = (int64_t)blockIdx.x * R::ROWS; base < a.rows; base += step) {
        const int64_t flat = place.flat, out_at = place.at[2];
        const bool there = place.row < a.rows;
        Row now = next;
        // n = (h - mean) rstd, dy and g = dy w of run j; `plain`: h - mean in place of n.  Formed twice, for the sums and for dx: kept,
        // they would be 24 registers a run instead of 8 or 6, which is a wave per SIMD or two.  In 8 bits h - mean is one product and sum
        // from the code, rounded once; never code (scale rstd) - mean rstd, whose parts are beyond fp32 for rows that are far off zero and
        // hardly vary, and whose difference loses what the row's distance from zero takes of fp32.  Behind the row's end dy, and so g, is
        // zero, and n is no infinity (mean rstd may be one).
        auto run = [&](int j, bool plain, float* n, float* dy, float* g) {
            const int left = C - 8 * (lane + j * G);
            if constexpr (FORMAT < 0) {
                to_float8(now.x[j], n);
#pragma unroll
                for (int e = 0; e < 8; ++e) n[e] -= now.mean;
            } else {
                act8_decode(now.codes[j], now.scale[j], FORMAT, n, now.mean);
            }
            if (!plain) {
                const float rstd = MODE == RAGGED || left > 0 ? now.rstd : 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) n[e] *= rstd;
                if (MODE == RAGGED && left < 8) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) n[e] = e < left ? n[e] : 0.f;
                }
            }
            to_float8(now.dy[j], dy);
            u.weight.get(j, lane, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] *= dy[e];
        };
        u32x4 ds[NV];
        walk.advance(place);
        fetch();  // (in flight while this row is worked on)
        if (a.dsummed) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int col = 8 * (lane + j * G);
                ds[j] = load8<MODE>((const uint16_t*)a.dsummed + flat + col, there ? C - col : 0);
            }
        }
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float n[8], dy[8], g[8];
            run(j, false, n, dy, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dw[j][e] += dy[e] * n[e];
                db[j][e] += dy[e];
                sum[0] += g[e];
                sum[1] += g[e] * n[e];
            }
        }
        row_sum<G>(sum, lds, at);
        // dx = rstd (g - n sum(g n) / C) - rstd sum g / C.  (rstd^2, which the other order forms from h - mean, is beyond fp32 for rows of
        // next to no variance.)
        const float c1 = -now.rstd * (sum[1] * inv_c), c0 = -now.rstd * (sum[0] * inv_c);
        uint16_t* const out = (uint16_t*)a.dx + out_at;
#pragma unroll
        for (int j = 0; j < NV; ++j) {  // (the compiler must not see that it has formed them before)
            if constexpr (FORMAT < 0) asm volatile("" : "+v"(now.x[j]));
            else asm volatile("" : "+v"(now.codes[j]));
            asm volatile("" : "+v"(now.dy[j]) : : "memory");
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = 8 * (lane + j * G), left = there ? C - col : 0;
            float dx[8], n[8], dy[8], g[8];
            run(j, true, n, dy, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) dx[e] = (g[e] + n[e] * c1) * now.rstd + c0;
            if (a.dsummed) {
                float r[8];
                to_float8(ds[j], r);
#pragma unroll
                for (int e = 0; e < 8; ++e) dx[e] += r[e];
            }
            store8<MODE>(out + col, to_bf16x8(dx), left);
        }
    }
    if (!a.weight) return;
    // One row of partial sums per workgroup: the row groups of a wave by exchanges between lanes, then the waves one after the other.
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
        __syncthreads();  // (the weights are in the way)
        if constexpr (G < 64) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    dw[j][e] = groups_sum<G>(dw[j][e]);
                    db[j][e] = groups_sum<G>(db[j][e]);
                }
        }
        for (int s = 0; s < R::THREADS / 64; ++s) {
            if ((int)threadIdx.x / 64 == s && (int)threadIdx.x % 64 < G) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int i = (j * 8 + e) * G + lane;
                        u.part[0][i] = s ? u.part[0][i] + dw[j][e] : dw[j][e];
                        u.part[1][i] = s ? u.part[1][i] + db[j][e] : db[j][e];
                    }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < C; c += R::THREADS) {
            const int i = ((c / 8 / G) * 8 + c % 8) * G + c / 8 % G;
            out[c] = u.part[0][i];
            out[C + c] = u.part[1][i];
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

// Threads a row, runs a thread, workgroups a CU forward and backward.  Rows of up to 2048 channels stay in one wave, whose sums need
// no barrier.  Two workgroups a CU that read ahead are what the memory wants where rows are long, and more of them are slower: forward /
// backward TB/s with 1, 2, 3, 4, 8 a CU,
//   178572 x 1024   3.92 5.84 5.68 5.47 5.49 / 4.02 6.01 5.67 5.05 5.48        65537 x 1280   3.99 5.63 5.45 5.45 5.33 / 3.76 5.43 4.38 5.02 4.50
//   65536 x 2048    5.39 5.98 5.69 5.76 5.84 / 4.80 5.71 5.06 5.49 5.12        32768 x 4096   3.52 5.80 5.94 5.54 5.49 / 3.32 5.27 5.31 4.42 4.46
//   32768 x 32 heads of 128   2.32 3.88 5.13 5.58 4.73 / 2.61 4.47 5.43 5.45 5.38        16000 x 8000   4.46 5.60 4.76 5.33 4.93 / 5.27 4.96 4.54 4.26 3.40
//   8000 x 16000    5.60 5.37 5.17 4.90 4.15 / 4.95 4.21 3.71 3.32 2.27
// (the backward's registers allow two at 1280 channels: with three the third waits; of 512 threads for more than 8192 they allow one, and
// 3 to 7 of them go to scratch).  Rows just above a limit leave lanes or runs empty at the same number of workgroups, so fewer bytes are in
// flight: 520 channels 3.6 / 3.9 TB/s, 640 4.4 / 4.7, 1032 5.4 / 5.3, 2056 3.5 / 3.4, 2560 4.3 / 4.2, 4104 4.4 / 3.3, 5120 5.6 / 4.1, 8200
// 4.8 / 4.2.  A forward that leaves codes has more to do between
// a row's arrival and its end, and takes one more: 65537 x 1280 5.36 -> 5.63, 65536 x 2048 5.80 -> 6.30 (two runs a thread: 6.24 -> 5.81).
#define VA_NORM_SHAPES(GO) \
    if (C <= 64) GO(8, 1, 4, 4) else if (C <= 128) GO(16, 1, 4, 4) else if (C <= 256) GO(32, 1, 4, 4) else if (C <= 512) GO(64, 1, 4, 4) \
    else if (C <= 1024) GO(64, 2, 2, 2) else if (C <= 1536) GO(64, 3, 2, 2) else if (C <= 2048) GO(64, 4, 2, 2) \
    else if (C <= 4096) GO(256, 2, 2, 2) else if (C <= 8192) GO(256, 4, 2, 1) else GO(512, 4, 1, 1)
constexpr int CUS = 256;

// Workgroups: as many as that, but no more than one a CU while they have fewer than `least` rows each (the backward's leave a row of
// sums each, for another kernel to add up: 2000 x 4096 27.8 -> 25.2 us with 8 rows instead of 2).
static int64_t norm_wgs(int64_t rows, int rows_per_wg, int wgs_per_cu, int least) {
    const int64_t one = (rows + rows_per_wg - 1) / rows_per_wg, many = (rows + least - 1) / least;
    const int64_t wgs = many > CUS ? many : one < CUS ? one : CUS;
    return wgs < wgs_per_cu * CUS ? wgs : wgs_per_cu * CUS;
}

int norm_bwd_wgs(int64_t rows, int C) {
#define VA_NORM_GO(G, NV, FWD, BWD) return (int)norm_wgs(rows, RowGroup<G>::ROWS, BWD, RowGroup<G>::ROWS > 4 ? 2 * RowGroup<G>::ROWS : 8);
    VA_NORM_SHAPES(VA_NORM_GO)
#undef VA_NORM_GO
}

// What is moved past the caches: more than the last one's 256 MB, which nobody finds there again; if what a wave moves at a time, one row
// or several short ones, is whole lines (32768 x 32 heads of 96 channels, forward / backward, 4.8 / 4.9 -> 5.05 / 5.15 TB/s).
static int norm_mode(const NormArgs& a, int bytes_per_channel) {
    const int C = a.channels, rows = C <= 64 ? 8 : C <= 128 ? 4 : C <= 256 ? 2 : 1;
    if (C % 8) return RAGGED;
    return rows * C % 64 == 0 && a.rows * C * bytes_per_channel > (int64_t)256 << 20 ? STREAM : WIDE;
}

hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t stream) {
    const int C = a.channels, mode = norm_mode(a, a.residual ? 8 : 4);
#define VA_NORM_FWD(G, NV, MODE) hipLaunchKernelGGL((norm_fwd_kernel<G, NV, MODE>), grid, dim3(RowGroup<G>::THREADS), 0, stream, a)
#define VA_NORM_GO(G, NV, FWD, BWD)                                             \
    {                                                                           \
        const dim3 grid((unsigned)norm_wgs(a.rows, RowGroup<G>::ROWS, FWD + (NV > 2 && a.format >= 0), RowGroup<G>::ROWS)); \
        if (mode == STREAM) VA_NORM_FWD(G, NV, STREAM);                         \
        else if (mode == WIDE) VA_NORM_FWD(G, NV, WIDE);                        \
        else VA_NORM_FWD(G, NV, RAGGED);                                        \
    }
    VA_NORM_SHAPES(VA_NORM_GO)
#undef VA_NORM_GO
#undef VA_NORM_FWD
    return hipGetLastError();
}

hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t stream) {
    const int C = a.channels, mode = norm_mode(a, a.dsummed ? 8 : a.format < 0 ? 6 : 5);
    const int wgs = norm_bwd_wgs(a.rows, C);
    if (wgs) {
        const dim3 grid((unsigned)wgs);
#define VA_NORM_BWD(G, NV, MODE, FORMAT) \
    hipLaunchKernelGGL((norm_bwd_kernel<G, NV, MODE, FORMAT>), grid, dim3(RowGroup<G>::THREADS), 0, stream, a)
#define VA_NORM_FORMAT(G, NV, MODE)                                                  \
    if (a.format < 0) VA_NORM_BWD(G, NV, MODE, -1);                                  \
    else if (a.format == VA_ACT8_INT8) VA_NORM_BWD(G, NV, MODE, VA_ACT8_INT8);       \
    else VA_NORM_BWD(G, NV, MODE, VA_ACT8_E4M3);
#define VA_NORM_GO(G, NV, FWD, BWD)                          \
    {                                                        \
        if (mode == STREAM) { VA_NORM_FORMAT(G, NV, STREAM) } \
        else if (mode == WIDE) { VA_NORM_FORMAT(G, NV, WIDE) } \
        else { VA_NORM_FORMAT(G, NV, RAGGED) }               \
    }
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
