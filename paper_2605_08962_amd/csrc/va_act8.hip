// Checkpoints of activations in 8 bits (the format: va_ops.h): several tensors packed or unpacked by one launch.
// Bound by memory: 3 bytes and some 5 operations per channel.
#include "va_internal.h"
#include "va_ops.h"

namespace va {

// G lanes (8 where every row is at most 64 channels, else 16) take one block of a row, 8 channels each; a group of lanes takes U
// blocks, whose loads are under way together.  MODE: see load8.  Measured, pack / unpack TB/s of q, k, v, o, U = 1, 2, 4, 8, past the caches
// (through them: 3 to 10 % less from U = 2 on):
//   178572 x 16 heads of 64, int8    5.58 6.64 6.43 6.36 / 5.75 6.50 5.85 5.98       32768 x 32/8 of 128   5.53 6.47 6.43 6.37 / 5.72 6.41 5.86 5.81
//   of 80, e4m3 (10 of 16 lanes)     4.31 5.82 6.31 6.23 / 4.10 5.57 5.91 4.53       of 96 (12 of 16)      4.94 6.20 6.39 6.51 / 4.73 6.01 6.19 5.20
// so two blocks where every lane of a group has channels, else four.
constexpr int ACT8_THREADS = 256;
template <int G, int U, int MODE, bool PACK>
__global__ void __launch_bounds__(ACT8_THREADS) act8_kernel(Act8Args a) {
    constexpr int GROUPS = ACT8_THREADS / G;
    const uint32_t wg = a.first_wg + blockIdx.x;
    int ti = 0;
    while (ti + 1 < a.num && wg >= a.t[ti + 1].first_wg) ++ti;
    const Act8Tensor& x = a.t[ti];
    const int lane = threadIdx.x % G;
    const int blocks = (x.channels + kAct8Block - 1) / kAct8Block;
    const int64_t groups = x.rows * blocks, first = (int64_t)(wg - x.first_wg) * (GROUPS * U) + threadIdx.x / G;
    int64_t row[U];
    int block[U], n[U];  // n: channels from this lane's on (lanes without any keep the others company)
    uint16_t* v[U];
    u32x4 w[U];
    u32x2 c[U];
    float s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t g = first + u * GROUPS;  // block of the tensor
        // (into row[] once: assigned in branches it may be copied as a whole, after a wait for the loads so far, which took unpacking heads of
        // 80 channels from 472 to 568 us)
        int64_t r = g;
        int b = 0;
        if (blocks > 1 && groups <= INT32_MAX) {
            r = (uint32_t)g / (uint32_t)blocks;
            b = (int)((uint32_t)g - (uint32_t)r * (uint32_t)blocks);
        } else if (blocks > 1) {
            r = g / blocks;
            b = (int)(g - r * blocks);
        }
        row[u] = r;
        block[u] = b;
        const int col = block[u] * kAct8Block + 8 * lane;
        n[u] = g < groups ? x.channels - col : 0;
        v[u] = (uint16_t*)x.values + strided_row(row[u], x.rows, x.rows_per_token, x.channels, x.stride) + col;
        if (PACK) {
            w[u] = load8<MODE>(v[u], n[u]);
        } else {
            c[u] = load_codes<MODE>((const uint8_t*)x.codes + row[u] * x.channels + col, n[u]);
            s[u] = n[u] > 0 ? x.scales[row[u] * blocks + block[u]] : 0.f;
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[8];
        if (PACK) {
            to_float8(w[u], f);
            const float scale = act8_scale(lanes_max<G>(magnitude8(w[u])), a.format);
            store_codes<MODE>((uint8_t*)x.codes + row[u] * x.channels + block[u] * kAct8Block + 8 * lane, act8_encode(f, scale, a.format), n[u]);
            if (lane == 0 && n[u] > 0) x.scales[row[u] * blocks + block[u]] = scale;
        } else {
            act8_decode(c[u], s[u], a.format, f);
            store8<MODE>(v[u], to_bf16x8(f), n[u]);
        }
    }
}

template <bool PACK>
static hipError_t launch_act8(Act8Args a, hipStream_t stream) {
    bool wide = true, full = true;
    int most = 0;
    int64_t bytes = 0;
    for (int i = 0; i < a.num; ++i) {
        const Act8Tensor& x = a.t[i];
        wide = wide && x.channels % 8 == 0;
        most = x.channels > most ? x.channels : most;
        bytes += 3 * x.rows * x.channels;
    }
    const int G = most <= 64 ? 8 : 16;
    for (int i = 0; i < a.num; ++i) full = full && a.t[i].channels % (8 * G) == 0;
    const int U = full ? 2 : 4, per_wg = ACT8_THREADS / G * U;
    int64_t wgs = 0;
    for (int i = 0; i < a.num; ++i) {
        a.t[i].first_wg = (uint32_t)wgs;
        const int64_t groups = a.t[i].rows * ((a.t[i].channels + kAct8Block - 1) / kAct8Block);
        wgs += (groups + per_wg - 1) / per_wg;
    }
    if (wgs > INT32_MAX) return hipErrorInvalidConfiguration;
    const bool stream_past = bytes > (int64_t)256 << 20;  // beyond the last-level cache nothing is found there again
    return launch_in_parts(wgs, [&](uint32_t first, unsigned n) {
        const dim3 grid(n), block(ACT8_THREADS);
        a.first_wg = first;
#define VA_ACT8(G, U, MODE) hipLaunchKernelGGL((act8_kernel<G, U, MODE, PACK>), grid, block, 0, stream, a)
#define VA_ACT8_MODE(G, U)                           \
    if (!wide) VA_ACT8(G, U, RAGGED);                \
    else if (stream_past) VA_ACT8(G, U, STREAM);     \
    else VA_ACT8(G, U, WIDE);
        if (G == 8) {
            if (full) { VA_ACT8_MODE(8, 2) } else { VA_ACT8_MODE(8, 4) }
        } else {
            if (full) { VA_ACT8_MODE(16, 2) } else { VA_ACT8_MODE(16, 4) }
        }
#undef VA_ACT8_MODE
#undef VA_ACT8
    });
}

hipError_t launch_act8_pack(const Act8Args& a, hipStream_t stream) { return launch_act8<true>(a, stream); }
hipError_t launch_act8_unpack(const Act8Args& a, hipStream_t stream) { return launch_act8<false>(a, stream); }

}  // namespace va
