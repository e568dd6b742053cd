// Queries and keys normed head by head and turned by the positions of one or several axes, in one pass and with one rounding,
//   y = w (x - m) / sqrt(mean((x - m)^2) + eps),   a' = scale (a cos - b sin), b' = scale (b cos + a sin)
// with the angle p_axis(i) f_i for pair i (m: 0, or the mean of x).  Bound: HBM, every row read once and written once.
#include <algorithm>

#include "rotary.h"

namespace lserve {

namespace {

constexpr int kRowThreads = 256, kRowWaves = kRowThreads / kWave;

// Row of head h of token t (queries first, then keys) and the weights of its norm.
struct NormedRow {
    const uint16_t* from;
    uint16_t* to;
    const float* weight;
};
__device__ __forceinline__ NormedRow normed_row(const TurnedRowsArgs& a, int t, int h) {
    const bool q = h < a.heads_q;
    const int i = q ? h : h - a.heads_q, heads = q ? a.heads_q : a.heads_k;
    const float* w = q ? a.turn.q_weight : a.turn.k_weight;
    return {(const uint16_t*)(q ? a.q : a.k) + (size_t)t * (q ? a.q_stride : a.k_stride) + i * kHeadDim,
            (uint16_t*)(q ? a.q_out : a.k_out) + ((size_t)t * heads + i) * kHeadDim, w ? w + (size_t)i * a.turn.weight_step : w};
}

// Positions of a token on its axes.
struct Places {
    int on[4];
    __device__ __forceinline__ int of(int axis) const {
        const int low = axis & 1 ? on[1] : on[0], high = axis & 1 ? on[3] : on[2];
        return axis & 2 ? high : low;
    }
};
// False: a row that is only there to fill up the batch.
__device__ __forceinline__ bool places_of(const TurnArgs& t, int token, Places& at) {
    at = {};
    if (!t.positions) return true;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < t.axes) at.on[i] = t.positions[i * t.axis_stride + token];
    return at.on[0] >= 0;
}

}  // namespace

// Eight lanes to a head, eight heads of a token at a time (rotary.h); eight angles a lane, the same for all heads.  Wavefront w of `share` to a
// token takes every share-th eight heads.
template <class T, bool INTERLEAVED>
__global__ __launch_bounds__(kRowThreads) void turned_rows_kernel(TurnedRowsArgs a, int share) {
    constexpr int kLayout = INTERLEAVED ? kInterleaved : kHalves;
    const int unit = blockIdx.x * kRowWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int t = unit / share, part = unit % share;
    if (t >= a.total) return;
    Places at;
    if (!places_of(a.turn, t, at)) return;
    const Pieces p = pieces_of<kLayout>(lane % 8, a.turn.rotary_dim);
    float2 turn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int pair = pair_of<kLayout>(p, i);
        turn[i] = make_float2(1.f, 0.f);
        if (p.turns && pair < a.turn.rotary_dim / 2) turn[i] = turn_of(at.of(axis_of(a.turn, pair)), a.turn.inv_freq[pair], a.turn.scale);
    }
    const int heads = a.heads_q + a.heads_k;
    for (int h = part * 8 + lane / 8; h < heads; h += share * 8) {
        const NormedRow row = normed_row(a, t, h);
        const uint4 x4 = reinterpret_cast<const uint4*>(row.from)[p.p0], y4 = reinterpret_cast<const uint4*>(row.from)[p.p1];
        uint32_t x[4] = {x4.x, x4.y, x4.z, x4.w}, y[4] = {y4.x, y4.y, y4.z, y4.w};
        turn_row<T, kLayout>(x, y, turn, a.turn, row.weight, p, nullptr, nullptr);
        reinterpret_cast<uint4*>(row.to)[p.p0] = make_uint4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<uint4*>(row.to)[p.p1] = make_uint4(y[0], y[1], y[2], y[3]);
    }
}

__device__ __forceinline__ float wave_sum(float x) { return rows4_sum(row16_sum(x)); }

// Any even R: a lane to a pair, or to two channels that pass, a wavefront to a head at a time.
template <class T, bool INTERLEAVED>
__global__ __launch_bounds__(kRowThreads) void turned_pairs_kernel(TurnedRowsArgs a, int share) {
    const int unit = blockIdx.x * kRowWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int t = unit / share, part = unit % share;
    if (t >= a.total) return;
    Places at;
    if (!places_of(a.turn, t, at)) return;
    const int pairs = a.turn.rotary_dim / 2;
    const bool turns = lane < pairs;
    const float2 turn = turns ? turn_of(at.of(axis_of(a.turn, lane)), a.turn.inv_freq[lane], a.turn.scale) : make_float2(1.f, 0.f);
    const int heads = a.heads_q + a.heads_k;
    const bool apart = !INTERLEAVED && turns;  // the lane's two channels are not next to each other
    const int c0 = apart ? lane : 2 * lane, c1 = apart ? lane + pairs : c0 + 1;
    for (int h = part; h < heads; h += share) {
        const NormedRow row = normed_row(a, t, h);
        uint32_t x;
        if (apart)
            x = row.from[c0] | (uint32_t)row.from[c1] << 16;
        else
            x = reinterpret_cast<const uint32_t*>(row.from)[lane];
        float lo = Elem<T>::lo(x), hi = Elem<T>::hi(x);
        if (a.turn.norm) {
            float w0 = 1.f, w1 = 1.f;
            if (row.weight) {
                w0 = row.weight[c0];
                w1 = row.weight[c1];
            }
            if (a.turn.norm == 2) {
                const float mean = wave_sum(lo + hi) * (1.f / kHeadDim);
                lo -= mean;
                hi -= mean;
            }
            const float inverse = rsqrtf(wave_sum(__builtin_fmaf(lo, lo, hi * hi)) * (1.f / kHeadDim) + a.turn.eps);
            lo = lo * inverse * w0;
            hi = hi * inverse * w1;
            x = Elem<T>::pack(lo, hi);
        }
        if (turns) {
            const float2 both = turned(lo, hi, turn);
            x = Elem<T>::pack(both.x, both.y);
        }
        if (apart) {
            row.to[c0] = (uint16_t)x;
            row.to[c1] = (uint16_t)(x >> 16);
        } else {
            reinterpret_cast<uint32_t*>(row.to)[lane] = x;
        }
    }
}

namespace {

template <class T> hipError_t launch(const TurnedRowsArgs& a, hipStream_t stream) {
    // Few rows: a lane of turned_pairs_kernel has one angle to work out, not eight, and such a launch takes as long as one wavefront does.
    const long long all = (long long)a.total * (a.heads_q + a.heads_k);
    const bool rows = (a.turn.interleaved || a.turn.rotary_dim % 16 == 0) && all > 48LL * num_compute_units();
    // Wavefronts to a token: as many as it has groups of heads while there are few tokens, one when there are plenty (its angles are then
    // worked out once).
    const int groups = rows ? ceil_div(a.heads_q + a.heads_k, 8) : a.heads_q + a.heads_k;
    const int share = (int)std::max(1LL, std::min<long long>(groups, 8LL * num_compute_units() / a.total));
    const long long blocks = ((long long)a.total * share + kRowWaves - 1) / kRowWaves;
    const dim3 grid((unsigned)blocks), threads(kRowThreads);
    if (rows && a.turn.interleaved)
        hipLaunchKernelGGL((turned_rows_kernel<T, true>), grid, threads, 0, stream, a, share);
    else if (rows)
        hipLaunchKernelGGL((turned_rows_kernel<T, false>), grid, threads, 0, stream, a, share);
    else if (a.turn.interleaved)
        hipLaunchKernelGGL((turned_pairs_kernel<T, true>), grid, threads, 0, stream, a, share);
    else
        hipLaunchKernelGGL((turned_pairs_kernel<T, false>), grid, threads, 0, stream, a, share);
    return hipGetLastError();
}

}  // namespace

hipError_t preload_norm_rotary_kernels() {
    hipFuncAttributes attr;
    return hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&turned_rows_kernel<F16, false>));
}

hipError_t launch_turned_rows(int dtype, const TurnedRowsArgs& a, hipStream_t stream) {
    return dtype == 0 ? launch<F16>(a, stream) : launch<BF16>(a, stream);
}

}  // namespace lserve
