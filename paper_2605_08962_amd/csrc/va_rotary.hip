// Rotary positions with several axes (time, height, width) on packed tokens, and the positions of packed images and video.
//
// Pair j of a head's first 2P channels (the channels j and j + P, or 2j and 2j + 1) is turned by the angle
//     phi = positions[pair_axis[j]][t] * inv_freq[j]:    y1 = x1 cos phi - x2 sin phi,   y2 = x2 cos phi + x1 sin phi;
// the backward pass turns by -phi (the inverse of a rotation is its transpose).  Channels from 2P on, and all of v, are copied.
// Bound by memory: 4 bytes per channel moved against 3 operations; the angles are formed once per token and pair and shared by
// its heads through LDS.
#include "va_internal.h"
#include "va_ops.h"

namespace va {

constexpr int ROT_THREADS = 256;

// cos and sin of a position's angle.  The angle of a far position does not fit 32 bits (2^20 at frequency 1 leaves steps of 1/16):
// it is reduced to turns in 64 bits, of which the fraction is taken, and the rest is 32-bit work.
__device__ __forceinline__ void rotary_angle(int position, float inv_freq, float& c, float& s) {
    const double turns = (double)position * (double)inv_freq * 0.15915494309189535;  // 1 / (2 pi)
    sincospif(2.f * (float)(turns - __builtin_rint(turns)), &s, &c);
}

template <int VEC> struct RotaryVec;
// (at any alignment: see load8)
template <> struct RotaryVec<8> { typedef u32x4 type; typedef u32x4_any any; };
template <> struct RotaryVec<4> { typedef u32x2 type; typedef u32x2 any __attribute__((aligned(2))); };
template <> struct RotaryVec<1> { typedef uint16_t type; typedef uint16_t any; };

template <int VEC>
__device__ __forceinline__ void unpack_vec(const typename RotaryVec<VEC>::type& w, float* x) {
    if constexpr (VEC == 1) x[0] = bf16_lo(w);
    else {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
    }
}
template <int VEC>
__device__ __forceinline__ typename RotaryVec<VEC>::type pack_vec(const float* x) {
    typename RotaryVec<VEC>::type w;
    if constexpr (VEC == 1) w = __builtin_bit_cast(uint16_t, (__bf16)x[0]);
    else {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
            const bf16x2 v = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, v);
        }
    }
    return w;
}

// One workgroup turns a.tokens_per_wg tokens.  A thread's item is two runs of VEC channels: of the two halves of VEC pairs, or
// (copied channels and v) side by side.  Both are read before either is written, so a tensor may be turned in place.
template <int VEC, bool INTERLEAVED>
__global__ void __launch_bounds__(ROT_THREADS) rotary_kernel(RotaryArgs a) {
    extern __shared__ float angles[];  // cos [tokens_per_wg][P], then sin
    typedef typename RotaryVec<VEC>::type Vec;
    typedef typename RotaryVec<VEC>::any VecAny;
    const int P = a.num_pairs, D = a.head_dim;
    const int64_t t0 = (int64_t)blockIdx.x * a.tokens_per_wg;
    const int nt = (int)min((int64_t)a.tokens_per_wg, a.total_tokens - t0);
    float* const cs = angles;
    float* const sn = angles + a.tokens_per_wg * P;
    for (int i = threadIdx.x; i < nt * P; i += ROT_THREADS) {
        const int t = i / P, j = i % P;
        const int axis = min(max(a.pair_axis[j], 0), a.num_axes - 1);
        float c, s;
        rotary_angle(a.positions[(size_t)axis * a.total_tokens + t0 + t], a.inv_freq[j], c, s);
        cs[i] = c;
        sn[i] = a.inverse ? -s : s;
    }
    __syncthreads();

    const int turned = P / VEC, copied = ((D - 2 * P) / VEC + 1) / 2;  // items of a head of q or k
    const int per_head = turned + copied, per_v = (D / VEC + 1) / 2;
    const int nq = a.num_q_heads * per_head, nk = a.num_kv_heads * per_head, nv = a.v ? a.num_kv_heads * per_v : 0;
    const int per_token = nq + nk + nv;
    for (int i = threadIdx.x; i < nt * per_token; i += ROT_THREADS) {
        const int t = i / per_token;
        int r = i % per_token;
        const uint16_t* src;
        uint16_t* dst;
        int c0, c1;
        bool two = true, turn = false;
        if (r < nq + nk) {
            const bool is_k = r >= nq;
            r -= is_k ? nq : 0;
            const int head = r / per_head, slot = r % per_head;
            src = (is_k ? a.k + (t0 + t) * a.k_stride : a.q + (t0 + t) * a.q_stride) + (size_t)head * D;
            dst = (is_k ? a.k_out + (t0 + t) * a.k_out_stride : a.q_out + (t0 + t) * a.q_out_stride) + (size_t)head * D;
            turn = slot < turned;
            c0 = turn ? (INTERLEAVED ? 2 * VEC * slot : VEC * slot) : 2 * P + 2 * VEC * (slot - turned);
            c1 = turn && !INTERLEAVED ? c0 + P : c0 + VEC;
            two = c1 < D;
            r = slot;
        } else {
            r -= nq + nk;
            const int head = r / per_v;
            c0 = 2 * VEC * (r % per_v);
            c1 = c0 + VEC;
            two = c1 < D;
            src = a.v + (t0 + t) * a.v_stride + (size_t)head * D;
            dst = a.v_out + (t0 + t) * a.v_out_stride + (size_t)head * D;
        }
        Vec w0 = *(const VecAny*)(src + c0), w1 = {};
        if (two) w1 = *(const VecAny*)(src + c1);
        if (turn) {
            float x0[VEC], x1[VEC];
            unpack_vec<VEC>(w0, x0);
            unpack_vec<VEC>(w1, x1);
            const float* const c = cs + t * P + VEC * r;
            const float* const s = sn + t * P + VEC * r;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                // interleaved: the 2 VEC channels side by side hold the pairs (2e, 2e + 1)
                float& u = INTERLEAVED ? (2 * e < VEC ? x0[2 * e % VEC] : x1[2 * e % VEC]) : x0[e];
                float& v = INTERLEAVED ? (2 * e + 1 < VEC ? x0[(2 * e + 1) % VEC] : x1[(2 * e + 1) % VEC]) : x1[e];
                const float u1 = u * c[e] - v * s[e];
                v = v * c[e] + u * s[e];
                u = u1;
            }
            w0 = pack_vec<VEC>(x0);
            w1 = pack_vec<VEC>(x1);
        }
        *(VecAny*)(dst + c0) = w0;
        if (two) *(VecAny*)(dst + c1) = w1;
    }
}

// Position of every packed token.  Segment s holds the rows [cu[s], cu[s + 1]); grids[s] = (time, height, width) of an image or
// video, whose patches lie time by time in blocks of merge x merge, rows of blocks one after the other; a height or width below 1
// means text, which advances on all three axes.  first[s] is added to all.  Tokens outside every segment get 0.
// One thread a token finds its segment by bisection; no contents of cu or grids lead outside the tensors.
__global__ void __launch_bounds__(256)
positions_kernel(int total_tokens, int num_segments, int merge, const int32_t* __restrict__ cu, const int32_t* __restrict__ grids,
                 const int32_t* __restrict__ first, int32_t* __restrict__ positions) {
    const int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (t >= total_tokens) return;
    int lo = 0, hi = num_segments;  // the last segment that starts at or before t
    while (lo < hi) {
        const int mid = (int)(((unsigned)lo + (unsigned)hi) >> 1);
        if (cu[mid + 1] <= t) lo = mid + 1; else hi = mid;
    }
    uint32_t p0 = 0, p1 = 0, p2 = 0;
    if (lo < num_segments && t >= cu[lo]) {
        const uint32_t i = (uint32_t)((int64_t)t - cu[lo]);
        const int h = grids[3 * (size_t)lo + 1], w = grids[3 * (size_t)lo + 2];
        if (h < 1 || w < 1) {
            p0 = p1 = p2 = i;
        } else {
            const uint32_t m = (uint32_t)merge, area = (uint32_t)min((int64_t)h * w, (int64_t)INT32_MAX);
            const uint32_t across = max((uint32_t)w / m, 1u), r = i % area, block = r / (m * m), e = r % (m * m);
            p0 = i / area;
            p1 = block / across * m + e / m;
            p2 = block % across * m + e % m;
        }
        const uint32_t f = first ? (uint32_t)first[lo] : 0;
        p0 += f; p1 += f; p2 += f;
    }
    positions[t] = (int32_t)p0;
    positions[(size_t)total_tokens + t] = (int32_t)p1;
    positions[2 * (size_t)total_tokens + t] = (int32_t)p2;
}

hipError_t launch_rotary_positions(int total_tokens, int num_segments, int merge, const int32_t* cu, const int32_t* grids,
                                   const int32_t* first, int32_t* positions, hipStream_t stream) {
    hipLaunchKernelGGL(positions_kernel, dim3((unsigned)(((int64_t)total_tokens + 255) / 256)), dim3(256), 0, stream, total_tokens,
                       num_segments, merge, cu, grids, first, positions);
    return hipGetLastError();
}

hipError_t launch_rotary(RotaryArgs a, hipStream_t stream) {
    const int shape = a.head_dim | a.num_pairs, vec = shape % 8 == 0 ? 8 : shape % 4 == 0 ? 4 : 1;  // the widest run that divides both
    a.tokens_per_wg = a.total_tokens >= 4096 ? (a.num_pairs <= 32 ? 8 : 4) : 1;
    const dim3 grid((unsigned)((a.total_tokens + (int64_t)a.tokens_per_wg - 1) / a.tokens_per_wg)), block(ROT_THREADS);
    const size_t lds = 2 * sizeof(float) * a.tokens_per_wg * a.num_pairs;
#define VA_ROTARY(VEC, INTER) hipLaunchKernelGGL((rotary_kernel<VEC, INTER>), grid, block, lds, stream, a)
#define VA_ROTARY_STYLE(VEC) if (a.interleaved) VA_ROTARY(VEC, true); else VA_ROTARY(VEC, false)
    if (vec == 8) { VA_ROTARY_STYLE(8); }
    else if (vec == 4) { VA_ROTARY_STYLE(4); }
    else { VA_ROTARY_STYLE(1); }
#undef VA_ROTARY_STYLE
#undef VA_ROTARY
    return hipGetLastError();
}

}  // namespace va
