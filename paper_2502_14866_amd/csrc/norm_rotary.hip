// Queries and keys normed head by head and turned by the positions of one or several axes, in one pass and with one rounding,
//   y = w (x - m) / sqrt(mean((x - m)^2) + eps),   a' = scale (a cos - b sin), b' = scale (b cos + a sin)
// with the angle p_axis(i) f_i for pair i (m: 0, or the mean of x).  Bound: HBM, every row read once and written once: 65536 tokens of 40 heads, 1.34 GB, 224 us
// with three axes = 6.0 TB/s, 236 with a norm = 5.7 (a copy of 671 MiB runs at 5.3); 5003 tokens of 64 heads, half of a head turning, 34 us = 4.8; 16 tokens
// 3.3 us, which is a launch, a position, an angle and a row one after the other.
#include <algorithm>

#include "rotary.h"

namespace lserve {

namespace {

constexpr int kRowThreads = 256, kRowWaves = kRowThreads / kWave;
constexpr int kMostTokens = 8;  // to a wavefront: 20 KiB of angles to a workgroup

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

// Position of a token by which a pair turns.
__device__ __forceinline__ int place_of(const TurnArgs& t, int token, int pair) { return t.positions[axis_of(t, pair) * t.axis_stride + token]; }

}  // namespace

// Eight lanes to a head, eight heads at a time (rotary.h).  A wavefront has `tokens` neighbouring tokens, or one of `share` parts of the heads of one; their
// angles are worked out one to a lane and passed round through LDS, and the next eight heads are in flight while it works on eight.
template <class T, int LAYOUT, bool NORM>
__global__ __launch_bounds__(kRowThreads) void turned_rows_kernel(TurnedRowsArgs a, int tokens, int share, int heads_inverse) {
    extern __shared__ float2 all_turns[];  // [wavefronts][tokens][kTurnRow]; behind the angles of a token, whether it is there; for kOddHalves rows in 32 bits
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int unit = blockIdx.x * kRowWaves + wave, t0 = unit / share * tokens, part = unit % share;
    if (t0 >= a.total) return;
    float2* turns = all_turns + wave * tokens * kTurnRow;
    float* room = reinterpret_cast<float*>(all_turns + kRowWaves * tokens * kTurnRow) + (wave * 8 + lane / 8) * kHeadDim;
    const Pieces p = pieces_of<LAYOUT>(lane % 8, a.turn.rotary_dim);
    const int heads = a.heads_q + a.heads_k, here = min(tokens, a.total - t0), rows = here * heads, first = part * 8 + lane / 8;
    auto token_of = [&](int j) { return tokens == 1 ? 0 : j * heads_inverse >> 16; };  // j / heads
    auto row_of = [&](int j) {
        const int held = min(j, rows - 1), t = token_of(held);
        return normed_row(a, t0 + t, held - t * heads);
    };
    uint32_t x[4], y[4], next_x[4], next_y[4];
    NormedRow row = row_of(first);
    load_pieces(row.from, 0, p, x, y);
    if (a.turn.positions) {
        for (int i = 0; i < here; ++i) {
            float2* to = turns + i * kTurnRow;
            if (lane < a.turn.rotary_dim / 2) to[turn_place<LAYOUT>(lane)] = turn_of(place_of(a.turn, t0 + i, lane), a.turn.inv_freq[lane], a.turn.scale);
            if (lane == 0) to[kHeadDim / 2].x = a.turn.positions[t0 + i] < 0 ? 0.f : 1.f;  // (a row that is only there to fill up the batch)
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    for (int j = first; j - lane / 8 < rows; j += share * 8) {
        const float2* turns_of_row = turns + token_of(min(j, rows - 1)) * kTurnRow;
        const bool there = j < rows && (!a.turn.positions || turns_of_row[kHeadDim / 2].x != 0.f);
        Weights w;  // (asked for ahead of the next rows: loads come back in order)
        if (NORM) load_weights(row.weight, p, w);
        const NormedRow next = row_of(j + share * 8);
        load_pieces(next.from, 0, p, next_x, next_y);
        float2 turn[8];
        if constexpr (LAYOUT != kOddHalves) read_turns(turns_of_row, lane % 8, turn);
        turn_row<T, LAYOUT, NORM>(x, y, turn, a.turn, row.weight != nullptr, w, p, room, turns_of_row);
        arrived(next_x, next_y);
        if (there) store_pieces(row.to, 0, p, x, y);
        row = next;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = next_x[i];
            y[i] = next_y[i];
        }
    }
}

__device__ __forceinline__ float wave_sum(float x) { return rows4_sum(row16_sum(x)); }

// Any even R: a lane to a pair, or to two channels that pass, a wavefront to a head at a time.
template <class T, bool INTERLEAVED>
__global__ __launch_bounds__(kRowThreads) void turned_pairs_kernel(TurnedRowsArgs a, int share) {
    const int unit = blockIdx.x * kRowWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int t = unit / share, part = unit % share;
    if (t >= a.total) return;
    if (a.turn.positions && a.turn.positions[t] < 0) return;
    const int pairs = a.turn.rotary_dim / 2;
    const bool turns = lane < pairs;
    const float2 turn = turns ? turn_of(place_of(a.turn, t, lane), a.turn.inv_freq[lane], a.turn.scale) : make_float2(1.f, 0.f);
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
    // Few rows: a launch takes as long as one wavefront does, and turned_pairs_kernel has no trip through LDS: 16 tokens of 40 heads 3.2 us against 3.6
    // by rows, 64 3.4 to 3.6 either way, 128 4.3 against 3.6 and 256 5.2 against 4.0 (with a norm 3.2, 3.6, 3.6, 4.7, 3.8, 5.8 and 4.1).  Halves of 20 channels,
    // whose rows pass through LDS: 500 tokens 7.7 us by pairs and 6.5 by rows, 5000 57.7 and 27.4, 60000 492 and 231.
    const int heads = a.heads_q + a.heads_k;
    const bool rows = (long long)a.total * heads > 12LL * num_compute_units();
    // Parts of a token: as many as it has groups of heads while there are few tokens.  With plenty, short wavefronts suit the memory better, long ones work
    // out fewer angles, which tells where a norm makes a group dearer.  One to five parts, us: 65536 tokens of five groups 246, 231, 235, 224, 232, with a
    // norm 243, 236, 246, 264, 272; 36000 of nine 255, 246, 241, 238, 237 (seven 227), with a norm 251, 237, 231, 234, 238; 40000 of eight 247, 238, 240,
    // 239, 233 (six 230), with a norm 242, 232, 235, 233, 244.  Tokens of few heads go several to a wavefront: 262144 of 10 heads with a norm 335 us one by
    // one, 268, 252, 271 in twos, fours, nines, without 246, 247, 255, 271; 9000 without 11.4, 10.1, 11.1, 15.9.
    const int groups = rows ? ceil_div(heads, 8) : heads;
    int share = (int)std::max(1LL, std::min<long long>(groups, 8LL * num_compute_units() / a.total)), tokens = 1;
    if (rows) {
        share = std::max(share, a.turn.norm ? (groups + 1) / 3 : groups * 4 / 5);
        if (share <= 1) tokens = (int)std::max(1LL, std::min<long long>(std::min((a.turn.norm ? 48 : 24) / heads, kMostTokens), a.total / (8LL * num_compute_units())));
    }
    const long long blocks = (((long long)a.total + tokens - 1) / tokens * share + kRowWaves - 1) / kRowWaves;
    const dim3 grid((unsigned)blocks), threads(kRowThreads);
    const int layout = a.turn.interleaved ? kInterleaved : a.turn.rotary_dim % 16 == 0 ? kHalves : kOddHalves;
    const size_t lds = sizeof(float2) * kRowWaves * tokens * kTurnRow + (layout == kOddHalves ? sizeof(float) * kRowWaves * 8 * kHeadDim : 0);
    const int heads_inverse = 65536 / heads + 1;
    auto by_rows = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, threads, lds, stream, a, tokens, share, heads_inverse); };
    if (rows && layout == kInterleaved)
        a.turn.norm ? by_rows(turned_rows_kernel<T, kInterleaved, true>) : by_rows(turned_rows_kernel<T, kInterleaved, false>);
    else if (rows && layout == kHalves)
        a.turn.norm ? by_rows(turned_rows_kernel<T, kHalves, true>) : by_rows(turned_rows_kernel<T, kHalves, false>);
    else if (rows)
        a.turn.norm ? by_rows(turned_rows_kernel<T, kOddHalves, true>) : by_rows(turned_rows_kernel<T, kOddHalves, false>);
    else if (a.turn.interleaved)
        hipLaunchKernelGGL((turned_pairs_kernel<T, true>), grid, threads, 0, stream, a, share);
    else
        hipLaunchKernelGGL((turned_pairs_kernel<T, false>), grid, threads, 0, stream, a, share);
    return hipGetLastError();
}

}  // namespace

hipError_t preload_norm_rotary_kernels() {
    hipFuncAttributes attr;
    return hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&turned_rows_kernel<F16, kHalves, false>));
}

hipError_t launch_turned_rows(int dtype, const TurnedRowsArgs& a, hipStream_t stream) {
    return dtype == 0 ? launch<F16>(a, stream) : launch<BF16>(a, stream);
}

}  // namespace lserve
