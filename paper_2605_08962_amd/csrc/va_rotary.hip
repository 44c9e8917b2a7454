// Rotary positions with several axes (time, height, width) on packed tokens, and the positions of packed images and video.
//
// Pair j of a head's first 2P channels (the channels j and j + P, or 2j and 2j + 1) is turned by the angle
//     phi = positions[pair_axis[j]][t] * inv_freq[j]:    y1 = x1 cos phi - x2 sin phi,   y2 = x2 cos phi + x1 sin phi;
// the backward pass turns by -phi (the inverse of a rotation is its transpose).  Channels from 2P on, and all of v, are copied.
// Bound by memory: 4 bytes per channel moved against 3 operations; the angles are formed once per token and pair and shared by
// its heads through LDS.  178572 tokens, 16/16 heads of 64, out of the fused projection 375 us (5.9 TB/s), 32768 tokens, 32/8 heads of 128
// 134 us (6.0 TB/s).
#include "va_internal.h"
#include "va_ops.h"

namespace va {

constexpr int ROT_THREADS = 256;

// cos and sin of a position's angle.  The angle of a far position does not fit 32 bits (2^20 at frequency 1 leaves steps of 1/16):
// it is reduced to turns in 64 bits, of which the fraction is taken, and the rest is 32-bit work.  The two products and the constant are
// each off by half a step, 3 * 2^-53 of the angle together: under 2^-20 with the 32-bit part up to 2^31, 2^-51 of the angle beyond.
__device__ __forceinline__ void rotary_angle(int position, float inv_freq, float& c, float& s) {
    const double turns = (double)position * (double)inv_freq * 0.15915494309189535;  // 1 / (2 pi)
    sincospif(2.f * (float)(turns - __builtin_rint(turns)), &s, &c);
}

template <int VEC> struct RotaryVec;
template <> struct RotaryVec<4> { typedef u32x2 type; typedef u32x2 any __attribute__((aligned(2))); };  // (at any alignment: see load8)
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

// n / d for n < 2^31 by a product.
__device__ __forceinline__ uint32_t divide(uint32_t n, RotaryArgs::Divisor d) { return (uint32_t)(((uint64_t)n * d.factor) >> d.shift); }

// Heads or numbers of pairs that whole 16-byte runs do not divide.  One workgroup turns a.tile_tokens tokens.  A thread's item is two runs
// of VEC channels: of the two halves of VEC pairs, or (copied channels and v) side by side.  Both are read before either is written,
// so a tensor may be turned in place.  Two items are under way together, the first of them while the angles are formed.  100000 x 16/16
// heads out of the fused projection: 20 pairs of 80 channels 345 us, 36 of 72 309 (4.5 TB/s both), 33 of 66, one channel at a time, 624 (2.0).
template <int VEC, bool INTERLEAVED>
__global__ void __launch_bounds__(ROT_THREADS) rotary_kernel(RotaryArgs a) {
    constexpr int U = 2;
    extern __shared__ float angles[];  // cos [tile_tokens][P], then sin
    typedef typename RotaryVec<VEC>::type Vec;
    typedef typename RotaryVec<VEC>::any VecAny;
    const int P = a.num_pairs, D = a.head_dim;
    const int64_t t0 = (int64_t)(a.first_wg + blockIdx.x) * a.tile_tokens;
    const int nt = (int)min((int64_t)a.tile_tokens, a.total_tokens - t0);
    const int turned = P / VEC;                     // items of a head that turn; then those that are copied
    const int nq = a.num_q_heads * a.per_head, nqk = nq + a.num_kv_heads * a.per_head;
    const int items = nt * a.per_token;

    struct Item {
        uint16_t *d0, *d1;  // null: nothing there
        Vec w0, w1;
        int angle;          // of the first pair in LDS; below 0: copied
    } it[U];
    auto fetch = [&](int i, Item& x) {
        x.d0 = x.d1 = nullptr;
        if (i >= items) return;
        const int t = (int)divide(i, a.by_token);
        int r = i - t * a.per_token;
        const uint16_t* src;
        uint16_t* dst;
        int c0, c1;
        x.angle = -1;
        if (r < nqk) {
            const bool is_k = r >= nq;
            r -= is_k ? nq : 0;
            const int head = (int)divide(r, a.by_head), slot = r - head * a.per_head;
            src = (is_k ? a.k + (t0 + t) * a.k_stride : a.q + (t0 + t) * a.q_stride) + head * D;
            dst = (is_k ? a.k_out + (t0 + t) * a.k_out_stride : a.q_out + (t0 + t) * a.q_out_stride) + head * D;
            const bool turn = slot < turned;
            c0 = turn ? (INTERLEAVED ? 2 * VEC * slot : VEC * slot) : 2 * P + 2 * VEC * (slot - turned);
            c1 = turn && !INTERLEAVED ? c0 + P : c0 + VEC;
            if (turn) x.angle = t * P + VEC * slot;
        } else {
            r -= nqk;
            const int head = (int)divide(r, a.by_v);
            c0 = 2 * VEC * (r - head * a.per_v);
            c1 = c0 + VEC;
            src = a.v + (t0 + t) * a.v_stride + head * D;
            dst = a.v_out + (t0 + t) * a.v_out_stride + head * D;
        }
        x.d0 = dst + c0;
        x.w0 = *(const VecAny*)(src + c0);
        if (c1 < D) {
            x.d1 = dst + c1;
            x.w1 = *(const VecAny*)(src + c1);
        }
    };
#pragma unroll
    for (int u = 0; u < U; ++u) fetch(threadIdx.x + u * ROT_THREADS, it[u]);

    float* const cs = angles;
    float* const sn = angles + a.tile_tokens * P;
    for (int i = threadIdx.x; i < nt * P; i += ROT_THREADS) {
        const int t = (int)divide(i, a.by_pairs), j = i - t * P;
        const int axis = min(max(a.pair_axis[j], 0), a.num_axes - 1);
        float c, s;
        rotary_angle(a.positions[(size_t)axis * a.total_tokens + t0 + t], a.inv_freq[j], c, s);
        cs[i] = c;
        sn[i] = a.inverse ? -s : s;
    }
    wg_barrier();

    for (int i = threadIdx.x; i < items; i += U * ROT_THREADS) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Item& x = it[u];
            if (x.d0 && x.angle >= 0) {
                float x0[VEC], x1[VEC];
                unpack_vec<VEC>(x.w0, x0);
                unpack_vec<VEC>(x.w1, x1);
                const float* const c = cs + x.angle;
                const float* const s = sn + x.angle;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    // interleaved: the 2 VEC channels side by side hold the pairs (2e, 2e + 1)
                    float& p = INTERLEAVED ? (2 * e < VEC ? x0[2 * e % VEC] : x1[2 * e % VEC]) : x0[e];
                    float& q = INTERLEAVED ? (2 * e + 1 < VEC ? x0[(2 * e + 1) % VEC] : x1[(2 * e + 1) % VEC]) : x1[e];
                    const float p1 = p * c[e] - q * s[e];
                    q = q * c[e] + p * s[e];
                    p = p1;
                }
                x.w0 = pack_vec<VEC>(x0);
                x.w1 = pack_vec<VEC>(x1);
            }
            if (x.d0) *(VecAny*)x.d0 = x.w0;
            if (x.d1) *(VecAny*)x.d1 = x.w1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) fetch(i + (U + u) * ROT_THREADS, it[u]);
    }
}

template <bool STREAMED>
__device__ __forceinline__ u32x4 load_run(const uint16_t* p) {
    return STREAMED ? __builtin_nontemporal_load((const u32x4_any*)p) : *(const u32x4_any*)p;
}
// What lane l ^ N holds, N = 4 or 8.
template <int N>
__device__ __forceinline__ u32x4 from_lane_xor(const u32x4& w, bool upper) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (N == 8) r[i] = dpp<0x128>(w[i]);                              // rotated by 8 within 16 lanes
        else { const uint32_t up = dpp<0x104>(w[i]), down = dpp<0x114>(w[i]); r[i] = upper ? down : up; }  // shifted by 4, either way
    }
    return r;
}

// Heads of whole 16-byte runs.  The runs of a token's heads of q, k and v are numbered in a row, and a workgroup takes a tile of them,
// whole heads, three a thread: neighbouring threads read and write neighbouring 16 bytes, so that whole lines leave a wave at once
// (written by two instructions, half a line each, past the caches, they cost up to twice the time).  All of a tile is read before any of
// it is written.  Where a run's pairs' other channels are:
//   HERE      in the run itself (interleaved)        LANE4, LANE8   4 or 8 lanes on (whole heads of 64 and 128 channels)
//   MEMORY    elsewhere: read once more, out of the line that another thread of the tile has just fetched
// STREAMED: past the caches.  Measured, TB/s forward, one / two / three / four runs a thread, through the caches / past them (where one
// thread took both halves of a pair instead: 5.46, 5.33, 5.04 and, interleaved, 4.96 at best)
//   178572 x 16/16 heads of 64   5.80 5.90 5.68 5.53 / 5.46 6.05 6.03 6.01       32768 x 32/8 of 128   5.54 5.60 5.55 5.53 / 5.56 5.89 6.02 6.12
//   100000 x 16/16 of 80         4.55 5.40 5.41 4.99 / 4.58 5.03 5.82 5.10       ... interleaved       5.71 5.56 5.54 5.39 / 5.48 6.00 6.09 5.96
enum RotaryPartner { HERE, LANE4, LANE8, MEMORY };
constexpr int ROT_RUNS = 3;
template <int PARTNER, bool STREAMED>
__global__ void __launch_bounds__(ROT_THREADS) rotary_flat_kernel(RotaryArgs a) {
    constexpr int U = ROT_RUNS;
    constexpr bool INTERLEAVED = PARTNER == HERE;
    extern __shared__ float angles[];  // cos [tile_tokens][P], then sin
    const int P = a.num_pairs;
    const int64_t f0 = (int64_t)(a.first_wg + blockIdx.x) * a.tile, total = (int64_t)a.total_tokens * a.per_token;
    const int64_t t0 = f0 / a.per_token;
    const int r0 = (int)(f0 - t0 * a.per_token), n = (int)min((int64_t)a.tile, total - f0);
    const int nq = a.num_q_heads * a.per_head, nqk = nq + a.num_kv_heads * a.per_head;
    u32x4 w[U], m[U];
    uint16_t* dst[U];
    int angle[U];  // of the run's first pair in LDS; below 0: copied
    bool second[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = threadIdx.x + u * ROT_THREADS;
        dst[u] = nullptr;
        angle[u] = -1;
        second[u] = false;
        if (i >= n) continue;
        const int x = r0 + i, t = (int)divide(x, a.by_token), r = x - t * a.per_token;
        const int64_t token = t0 + t;
        const uint16_t* src;
        if (r < nqk) {
            const bool is_k = r >= nq;
            src = (is_k ? a.k + token * a.k_stride : a.q + token * a.q_stride) + 8 * (r - (is_k ? nq : 0));
            dst[u] = (is_k ? a.k_out + token * a.k_out_stride : a.q_out + token * a.q_out_stride) + 8 * (r - (is_k ? nq : 0));
            const int c = 8 * (r - (int)divide(r, a.by_head) * a.per_head);  // first channel in the head
            if (c < 2 * P) {
                if (INTERLEAVED) {
                    angle[u] = t * P + c / 2;
                } else {
                    second[u] = c >= P;
                    angle[u] = t * P + c - (second[u] ? P : 0);
                    if (PARTNER == MEMORY) m[u] = load_run<STREAMED>(src + (second[u] ? -P : P));
                }
            }
        } else {
            src = a.v + token * a.v_stride + 8 * (r - nqk);
            dst[u] = a.v_out + token * a.v_out_stride + 8 * (r - nqk);
        }
        w[u] = load_run<STREAMED>(src);
    }

    const int tokens = (int)divide(r0 + n - 1, a.by_token) + 1;
    float* const cs = angles;
    float* const sn = angles + a.tile_tokens * P;
    for (int i = threadIdx.x; i < tokens * P; i += ROT_THREADS) {
        const int t = (int)divide(i, a.by_pairs), j = i - t * P;
        const int axis = min(max(a.pair_axis[j], 0), a.num_axes - 1);
        float c, s;
        rotary_angle(a.positions[(size_t)axis * a.total_tokens + t0 + t], a.inv_freq[j], c, s);
        cs[i] = c;
        sn[i] = a.inverse ? -s : s;
    }
    wait_vmcnt<0>();  // (a partner may be written by another thread, where the tensor is turned in place)
    wg_barrier();

#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (PARTNER == LANE4 || PARTNER == LANE8) m[u] = from_lane_xor<PARTNER == LANE8 ? 8 : 4>(w[u], second[u]);  // (all lanes)
        if (!dst[u]) continue;
        if (angle[u] >= 0) {
            float x[8], y[8];
            to_float8(w[u], x);
            const float* const c = cs + angle[u];
            const float* const s = sn + angle[u];
            if (INTERLEAVED) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[2 * e] = x[2 * e] * c[e] - x[2 * e + 1] * s[e];
                    y[2 * e + 1] = x[2 * e + 1] * c[e] + x[2 * e] * s[e];
                }
            } else {
                float p[8];
                to_float8(m[u], p);
                const float sign = second[u] ? 1.f : -1.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = x[e] * c[e] + p[e] * (sign * s[e]);
            }
            w[u] = to_bf16x8(y);
        }
        if (STREAMED) __builtin_nontemporal_store(w[u], (u32x4_any*)dst[u]);
        else *(u32x4_any*)dst[u] = w[u];
    }
}

// Position of every packed token.  Segment s holds the rows [cu[s], cu[s + 1]); grids[s] = (time, height, width) of an image or
// video, whose patches lie time by time in blocks of merge x merge, rows of blocks one after the other; a height or width below 1
// means text, which advances on all three axes.  first[s] is added to all.  Tokens outside every segment get 0.
// One thread a token finds its segment by bisection; no contents of cu or grids lead outside the tensors.  609226 tokens in 400 segments
// 6.5 us, 246 in 4 1.9 us.  The difference is instruction issue: nine steps of bisection and five divisions by numbers known only
// here are 203 vector instructions a wave, of which a SIMD runs nine waves (over 3 us); the rest is a dozen loads one after the other.
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

static RotaryArgs::Divisor divisor(uint32_t d) {
    uint32_t l = 0;  // the smallest with 2^l >= d; then ceil(2^(31 + l) / d) < 2^32 is exact for n < 2^31
    while (((uint64_t)1 << l) < d) ++l;
    return {(uint32_t)((((uint64_t)1 << (31 + l)) + d - 1) / d), 31 + l};
}

hipError_t launch_rotary(RotaryArgs a, hipStream_t stream) {
    const dim3 block(ROT_THREADS);
    const int kinds = a.v ? 2 : 1;
    a.by_pairs = divisor(a.num_pairs);
    if (a.head_dim % 8 == 0 && a.num_pairs % (a.interleaved ? 4 : 8) == 0) {
        a.per_head = a.head_dim / 8;
        a.per_token = (a.num_q_heads + kinds * a.num_kv_heads) * a.per_head;
        a.tile = ROT_THREADS * ROT_RUNS / a.per_head * a.per_head;
        a.tile_tokens = a.tile / a.per_token + 2;
        a.by_token = divisor(a.per_token);
        a.by_head = divisor(a.per_head);
        const int64_t runs = (int64_t)a.total_tokens * a.per_token, wgs = (runs + a.tile - 1) / a.tile;
        if (wgs > INT32_MAX) return hipErrorInvalidConfiguration;
        const size_t lds = 2 * sizeof(float) * a.tile_tokens * a.num_pairs;
        const bool streamed = runs * 32 > (int64_t)256 << 20;  // beyond the last-level cache nothing is found there again
        const bool whole = a.head_dim == 2 * a.num_pairs;
        const int partner = a.interleaved ? HERE : whole && a.num_pairs == 32 ? LANE4 : whole && a.num_pairs == 64 ? LANE8 : MEMORY;
        return launch_in_parts(wgs, [&](uint32_t first, unsigned n) {
            const dim3 grid(n);
            a.first_wg = first;
#define VA_ROTARY(PARTNER)                                                                                               \
    if (streamed) hipLaunchKernelGGL((rotary_flat_kernel<PARTNER, true>), grid, block, lds, stream, a);                  \
    else hipLaunchKernelGGL((rotary_flat_kernel<PARTNER, false>), grid, block, lds, stream, a);                          \
    break;
            switch (partner) {
                case HERE: VA_ROTARY(HERE)
                case LANE4: VA_ROTARY(LANE4)
                case LANE8: VA_ROTARY(LANE8)
                default: VA_ROTARY(MEMORY)
            }
#undef VA_ROTARY
        });
    }
    const int vec = (a.head_dim | a.num_pairs) % 4 == 0 ? 4 : 1;  // the widest run that divides both
    a.tile_tokens = a.total_tokens >= 4096 ? 4 : 1;
    a.per_head = a.num_pairs / vec + ((a.head_dim - 2 * a.num_pairs) / vec + 1) / 2;
    a.per_v = (a.head_dim / vec + 1) / 2;
    a.per_token = (a.num_q_heads + a.num_kv_heads) * a.per_head + (a.v ? a.num_kv_heads * a.per_v : 0);
    a.by_token = divisor(a.per_token);
    a.by_head = divisor(a.per_head);
    a.by_v = divisor(a.per_v);
    const size_t lds = 2 * sizeof(float) * a.tile_tokens * a.num_pairs;
    return launch_in_parts((a.total_tokens + (int64_t)a.tile_tokens - 1) / a.tile_tokens, [&](uint32_t first, unsigned n) {
        const dim3 grid(n);
        a.first_wg = first;
        if (vec == 4 && a.interleaved) hipLaunchKernelGGL((rotary_kernel<4, true>), grid, block, lds, stream, a);
        else if (vec == 4) hipLaunchKernelGGL((rotary_kernel<4, false>), grid, block, lds, stream, a);
        else if (a.interleaved) hipLaunchKernelGGL((rotary_kernel<1, true>), grid, block, lds, stream, a);
        else hipLaunchKernelGGL((rotary_kernel<1, false>), grid, block, lds, stream, a);
    });
}

}  // namespace va
