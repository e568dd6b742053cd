// Rotary positions of queries and keys: of every head the first R channels are R / 2 pairs (a, b), and a token at position t has them
// turned by the angle t f_i of the pair,
//   a' = scale (a cos - b sin),  b' = scale (b cos + a sin),
// the other channels passing as they are.  Bound: HBM, every row read once and written once.  65536 tokens of 40 heads, 1.34 GB, 244 us = 5.5 TB/s (a
// copy of 1 GiB runs at 5.1); 9217 out of a fused projection, half of the channels turning, 40 us = 4.7 TB/s, 30 where the rows are in the last
// cache still; 16 tokens 3.0 us, which is a launch, a position, an angle and a row one after the other.
//
// The angle is taken in 64 bits: in 32 a position of 10^6 would be off by 0.06 radians.  Its whole turns are dropped there (t f_i / 2 pi less the
// nearest whole number, exact), and sine and cosine of the rest, once per token and pair and not once per head, are 32-bit ones, three
// products of 32 bits and one rounding follow.
#include <algorithm>

#include "rotary.h"

namespace lserve {

namespace {

constexpr int kRotaryThreads = 256, kRotaryWaves = kRotaryThreads / kWave;

// Row of head h of token t: queries first, then keys.
struct HeadRow {
    const uint16_t* from;
    uint16_t* to;
};
__device__ __forceinline__ HeadRow head_row(const RotaryArgs& a, int t, int h) {
    const bool q = h < a.heads_q;
    const int i = q ? h : h - a.heads_q, heads = q ? a.heads_q : a.heads_k;
    return {(const uint16_t*)(q ? a.q : a.k) + (size_t)t * (q ? a.q_stride : a.k_stride) + i * kHeadDim,
            (uint16_t*)(q ? a.q_out : a.k_out) + ((size_t)t * heads + i) * kHeadDim};
}

}  // namespace

// Rows in pieces of eight channels, two to a lane and eight lanes to a head, so that a wavefront works on eight heads at a time and its sixteen-byte
// loads of a head are whole rows.  With halves (channel i with i + R / 2) a lane has one piece of either half and turns eight
// pairs, interleaved (2 i with 2 i + 1) it has four pairs in each of two pieces; eight angles a lane in both, the same for all heads.  Wavefront w of
// `share` to a token takes every share-th eight heads.  Requires R % 16 == 0 (halves) or R % 8 == 0.
template <class T, bool INTERLEAVED>
__global__ __launch_bounds__(kRotaryThreads) void rotary_rows_kernel(RotaryArgs a, int share) {
    const int unit = blockIdx.x * kRotaryWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int t = unit / share, part = unit % share;
    if (t >= a.total) return;
    const int position = a.positions[t];
    if (position < 0) return;  // a row that is only there to fill up the batch
    const int l = lane % 8, pieces = a.rotary_dim / 8;
    // the lane's pieces: of either half, then of what does not turn; or two, eight apart
    int p0, p1;
    bool turns0, turns1;
    if (INTERLEAVED) {
        p0 = l;
        p1 = l + 8;
        turns0 = p0 < pieces;
        turns1 = p1 < pieces;
    } else {
        turns0 = turns1 = l < pieces / 2;
        p0 = turns0 ? l : pieces + 2 * (l - pieces / 2);
        p1 = turns0 ? l + pieces / 2 : p0 + 1;
    }
    float2 turn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        turn[i] = make_float2(1.f, 0.f);
        const int pair = INTERLEAVED ? (i < 4 ? 4 * p0 + i : 4 * p1 + i - 4) : 8 * p0 + i;
        if (INTERLEAVED ? (i < 4 ? turns0 : turns1) : turns0) turn[i] = turn_of(position, a.inv_freq[pair], a.scale);
    }
    const int heads = a.heads_q + a.heads_k;
    for (int h = part * 8 + lane / 8; h < heads; h += share * 8) {
        const HeadRow row = head_row(a, t, h);
        const uint4 x4 = reinterpret_cast<const uint4*>(row.from)[p0], y4 = reinterpret_cast<const uint4*>(row.from)[p1];
        const uint32_t x[4] = {x4.x, x4.y, x4.z, x4.w}, y[4] = {y4.x, y4.y, y4.z, y4.w};
        uint32_t xo[4], yo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x0 = Elem<T>::lo(x[i]), x1 = Elem<T>::hi(x[i]), y0 = Elem<T>::lo(y[i]), y1 = Elem<T>::hi(y[i]);
            if (INTERLEAVED) {
                const float2 u = turn[i], v = turn[4 + i];
                xo[i] = Elem<T>::pack(x0 * u.x - x1 * u.y, x1 * u.x + x0 * u.y);
                yo[i] = Elem<T>::pack(y0 * v.x - y1 * v.y, y1 * v.x + y0 * v.y);
            } else {
                const float2 u = turn[2 * i], v = turn[2 * i + 1];
                xo[i] = Elem<T>::pack(x0 * u.x - y0 * u.y, x1 * v.x - y1 * v.y);
                yo[i] = Elem<T>::pack(y0 * u.x + x0 * u.y, y1 * v.x + x1 * v.y);
            }
            // what does not turn keeps its bits, infinities and not-a-numbers among them (times zero they would not)
            if (!turns0) xo[i] = x[i];
            if (!turns1) yo[i] = y[i];
        }
        reinterpret_cast<uint4*>(row.to)[p0] = make_uint4(xo[0], xo[1], xo[2], xo[3]);
        reinterpret_cast<uint4*>(row.to)[p1] = make_uint4(yo[0], yo[1], yo[2], yo[3]);
    }
}

// Any even R: a lane to a pair, or to two channels that pass, a wavefront to a head at a time.
template <class T, bool INTERLEAVED>
__global__ __launch_bounds__(kRotaryThreads) void rotary_pairs_kernel(RotaryArgs a, int share) {
    const int unit = blockIdx.x * kRotaryWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int t = unit / share, part = unit % share;
    if (t >= a.total) return;
    const int position = a.positions[t];
    if (position < 0) return;
    const int pairs = a.rotary_dim / 2;
    const bool turns = lane < pairs;
    const float2 turn = turns ? turn_of(position, a.inv_freq[lane], a.scale) : make_float2(1.f, 0.f);
    const int heads = a.heads_q + a.heads_k;
    for (int h = part; h < heads; h += share) {
        const HeadRow row = head_row(a, t, h);
        if (INTERLEAVED || !turns) {
            const uint32_t x = reinterpret_cast<const uint32_t*>(row.from)[lane];
            const float lo = Elem<T>::lo(x), hi = Elem<T>::hi(x);
            reinterpret_cast<uint32_t*>(row.to)[lane] = turns ? Elem<T>::pack(lo * turn.x - hi * turn.y, hi * turn.x + lo * turn.y) : x;
        } else {
            const float lo = Elem<T>::lo(row.from[lane]), hi = Elem<T>::lo(row.from[lane + pairs]);
            const uint32_t x = Elem<T>::pack(lo * turn.x - hi * turn.y, hi * turn.x + lo * turn.y);
            row.to[lane] = (uint16_t)x;
            row.to[lane + pairs] = (uint16_t)(x >> 16);
        }
    }
}

namespace {

template <class T> hipError_t launch(const RotaryArgs& a, hipStream_t stream) {
    // A launch of few rows takes as long as one wavefront does, and a lane of rotary_pairs_kernel has one angle to work out, not eight: 16 tokens of
    // 40 heads 3.0 us against 4.3 by rows, 256 tokens 4.2 against 4.7.  512 tokens are 5.7 against 5.5, 64k 329 against 247.
    const long long all = (long long)a.total * (a.heads_q + a.heads_k);
    const bool rows = a.rotary_dim % (a.interleaved ? 8 : 16) == 0 && all > 48LL * num_compute_units();
    // Wavefronts to a token: as many as it has groups of heads while there are few tokens, one when there are plenty (its angles are
    // then worked out once: 64k tokens of 40 heads 247 us, 354 with five wavefronts to each).
    const int groups = rows ? ceil_div(a.heads_q + a.heads_k, 8) : a.heads_q + a.heads_k;
    const int share = (int)std::max(1LL, std::min<long long>(groups, 8LL * num_compute_units() / a.total));
    const long long blocks = ((long long)a.total * share + kRotaryWaves - 1) / kRotaryWaves;
    const dim3 grid((unsigned)blocks), threads(kRotaryThreads);
    if (rows && a.interleaved)
        hipLaunchKernelGGL((rotary_rows_kernel<T, true>), grid, threads, 0, stream, a, share);
    else if (rows)
        hipLaunchKernelGGL((rotary_rows_kernel<T, false>), grid, threads, 0, stream, a, share);
    else if (a.interleaved)
        hipLaunchKernelGGL((rotary_pairs_kernel<T, true>), grid, threads, 0, stream, a, share);
    else
        hipLaunchKernelGGL((rotary_pairs_kernel<T, false>), grid, threads, 0, stream, a, share);
    return hipGetLastError();
}

}  // namespace

hipError_t preload_rotary_kernels() {
    hipFuncAttributes attr;
    return hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&rotary_rows_kernel<F16, false>));
}

hipError_t launch_rotary(int dtype, const RotaryArgs& a, hipStream_t stream) {
    return dtype == 0 ? launch<F16>(a, stream) : launch<BF16>(a, stream);
}

}  // namespace lserve
