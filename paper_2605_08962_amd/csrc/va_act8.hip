// Checkpoints of activations in 8 bits (the format: va_ops.h): several tensors packed or unpacked by one launch.
// Bound by memory: 3 bytes and a few operations per channel.
#include "va_internal.h"
#include "va_ops.h"

namespace va {

// G lanes (8 where every row is at most 64 channels, else 16) take one block of a row, 8 channels each; one thread handles one
// such run.  MODE: see load8.
template <int G, int MODE, bool PACK>
__global__ void __launch_bounds__(256) act8_kernel(Act8Args a) {
    int ti = 0;
    while (ti + 1 < a.num && blockIdx.x >= a.t[ti + 1].first_wg) ++ti;
    const Act8Tensor& x = a.t[ti];
    const int64_t group = (int64_t)(blockIdx.x - x.first_wg) * (256 / G) + threadIdx.x / G;  // block of the tensor
    const int lane = threadIdx.x % G;
    const int blocks = (x.channels + kAct8Block - 1) / kAct8Block;
    const int64_t row = group / blocks;
    const int block = (int)(group % blocks);
    const int col = block * kAct8Block + 8 * lane;
    const int n = row < x.rows ? x.channels - col : 0;  // channels from here on (the lanes beyond keep the others company)
    const int64_t token = row / x.rows_per_token;
    uint16_t* const v = (uint16_t*)x.values + token * x.stride + (row % x.rows_per_token) * x.channels + col;
    uint8_t* const codes = (uint8_t*)x.codes + row * x.channels + col;
    float* const scale = x.scales + row * blocks + block;
    if (PACK) {
        const u32x4 w = load8<MODE>(v, n);
        float f[8];
        to_float8(w, f);
        const float s = act8_scale(lanes_max<G>(magnitude8(w)), a.format);
        store_codes<MODE>(codes, act8_encode(f, s, a.format), n);
        if (lane == 0 && n > 0) *scale = s;
    } else if (n > 0) {
        float f[8];
        act8_decode(load_codes<MODE>(codes, n), *scale, a.format, f);
        store8<MODE>(v, to_bf16x8(f), n);
    }
}

template <bool PACK>
static hipError_t launch_act8(Act8Args a, hipStream_t stream) {
    bool wide = true;
    int most = 0;
    for (int i = 0; i < a.num; ++i) {
        const Act8Tensor& x = a.t[i];
        wide = wide && x.channels % 8 == 0;
        most = x.channels > most ? x.channels : most;
    }
    const int G = most <= 64 ? 8 : 16;
    int64_t wgs = 0;
    for (int i = 0; i < a.num; ++i) {
        a.t[i].first_wg = (uint32_t)wgs;
        const int64_t groups = a.t[i].rows * ((a.t[i].channels + kAct8Block - 1) / kAct8Block);
        wgs += (groups * G + 255) / 256;
    }
    if (wgs == 0) return hipSuccess;
    if (wgs > INT32_MAX) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)wgs), block(256);
    if (G == 8 && wide) hipLaunchKernelGGL((act8_kernel<8, WIDE, PACK>), grid, block, 0, stream, a);
    else if (G == 8) hipLaunchKernelGGL((act8_kernel<8, RAGGED, PACK>), grid, block, 0, stream, a);
    else if (wide) hipLaunchKernelGGL((act8_kernel<16, WIDE, PACK>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((act8_kernel<16, RAGGED, PACK>), grid, block, 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_act8_pack(const Act8Args& a, hipStream_t stream) { return launch_act8<true>(a, stream); }
hipError_t launch_act8_unpack(const Act8Args& a, hipStream_t stream) { return launch_act8<false>(a, stream); }

}  // namespace va
