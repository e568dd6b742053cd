// New tokens on their way from a projection into the paged cache: queries normed and turned, keys normed, turned and written to their pages
// (16-bit rows or codes) with the key statistics brought up to date, values written next to them.  What it leaves in the cache is what
// lserve_append_kv would be handed the turned keys for.  Bound: HBM, every row read once, queries and pages written once.
#include <algorithm>

#include "quantize.h"
#include "rotary.h"

namespace lserve {

namespace {

constexpr int kAppendThreads = 256, kAppendWaves = kAppendThreads / kWave;

constexpr int kDppRor8 = 0x128;  // lane i <-> i ^ 8 inside each row

// Combines lanes l, l ^ 8, l ^ 16, l ^ 32, as far as `rows` (a power of two) rows of eight lanes go.
template <class Op> __device__ __forceinline__ float over_rows(float x, int rows, Op op) {
    if (rows >= 2) x = op(x, dpp_f<kDppRor8>(x));
    if (rows >= 4) {
        const unsigned u = __builtin_bit_cast(unsigned, x);
        const swap_pair_t s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        const unsigned s0 = s[0], s1 = s[1];
        x = op(__builtin_bit_cast(float, s0), __builtin_bit_cast(float, s1));
    }
    if (rows >= 8) {
        const unsigned u = __builtin_bit_cast(unsigned, x);
        const swap_pair_t s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        const unsigned s0 = s[0], s1 = s[1];
        x = op(__builtin_bit_cast(float, s0), __builtin_bit_cast(float, s1));
    }
    return x;
}

// Writes the ranges of eight channels into the statistics rows of a logical page, with what they hold taken in if it held tokens before.
template <class T>
__device__ __forceinline__ void write_range(uint4* stats, int piece, const float (&high)[8], const float (&low)[8], bool held) {
    float h[8], l[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        h[i] = high[i];
        l[i] = low[i];
    }
    if (held) {
        const uint4 om = stats[piece], on = stats[kHeadDim / 8 + piece];
        const uint32_t wm[4] = {om.x, om.y, om.z, om.w}, wn[4] = {on.x, on.y, on.z, on.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[2 * i] = fmaxf(h[2 * i], Elem<T>::lo(wm[i]));
            h[2 * i + 1] = fmaxf(h[2 * i + 1], Elem<T>::hi(wm[i]));
            l[2 * i] = fminf(l[2 * i], Elem<T>::lo(wn[i]));
            l[2 * i + 1] = fminf(l[2 * i + 1], Elem<T>::hi(wn[i]));
        }
    }
    stats[piece] = make_uint4(Elem<T>::pack(h[0], h[1]), Elem<T>::pack(h[2], h[3]), Elem<T>::pack(h[4], h[5]), Elem<T>::pack(h[6], h[7]));
    stats[kHeadDim / 8 + piece] = make_uint4(Elem<T>::pack(l[0], l[1]), Elem<T>::pack(l[2], l[3]), Elem<T>::pack(l[4], l[5]), Elem<T>::pack(l[6], l[7]));
}

// Where the rows of a KV head of a page go.
struct Slab {
    uint4 *k, *v;
    size_t page_head;  // (page, head) index inside the pool
};
__device__ __forceinline__ Slab slab_of(const LayerParams& lp, const PagedParams& kv, int b, int hk, int p, int bits) {
    const bool ring = in_stream_pool(lp, kv, hk);
    const int phys = ring ? kv.ring_table[(size_t)b * kv.ring + ring_slot(lp, p)] : kv.page_table[(size_t)b * kv.max_pages + p];
    const size_t ph = (size_t)phys * (ring ? kv.stream_heads : kv.pool_heads) + pool_rank(lp, kv, hk, ring);
    uint4 *k = reinterpret_cast<uint4*>(const_cast<void*>(ring ? kv.k_stream : kv.k_pool)),
          *v = reinterpret_cast<uint4*>(const_cast<void*>(ring ? kv.v_stream : kv.v_pool));
    return {k + ph * slab_chunks(lp.NP, bits), v + ph * slab_chunks(lp.NP, bits), ph};
}

// A lane's two pieces of a row to its slot of a slab.
template <class T, int BITS>
__device__ __forceinline__ void write_row(uint4* slab, int page_size, int slot, const Pieces& p, int l, const uint32_t (&x)[4], const uint32_t (&y)[4]) {
    const size_t row = (size_t)slot * (kHeadDim / 8);
    if constexpr (BITS == 16) {
        slab[row + p.p0] = make_uint4(x[0], x[1], x[2], x[3]);
        slab[row + p.p1] = make_uint4(y[0], y[1], y[2], y[3]);
    } else {
        uint2 u, v;
        uint32_t pair;
        quantize_pieces<T, BITS>(x, y, u, v, pair);
        if constexpr (BITS == 8) {
            reinterpret_cast<uint2*>(slab)[row + p.p0] = u;
            reinterpret_cast<uint2*>(slab)[row + p.p1] = v;
        } else {
            reinterpret_cast<uint32_t*>(slab)[row + p.p0] = u.x;
            reinterpret_cast<uint32_t*>(slab)[row + p.p1] = v.x;
        }
        if (l == 0) reinterpret_cast<uint32_t*>(slab + page_size * (kHeadDim * BITS / 128))[slot] = pair;
    }
}

// Angles of a token in LDS: what a lane reads of its eight pairs is four pieces of sixteen bytes, each next to those of the other lanes of the row;
// the rows of neighbouring tokens start in other banks.  kOddHalves: pair by pair.
constexpr int kTurnRow = 80;  // float2 to a token
template <int LAYOUT> __device__ __forceinline__ int turn_place(int pair) {
    if (LAYOUT == kOddHalves) return pair;
    const int l = LAYOUT == kHalves ? pair / 8 : pair % 32 / 4, i = LAYOUT == kHalves ? pair % 8 : pair / 32 * 4 + pair % 4;
    return i / 2 * 16 + l * 2 + i % 2;
}
__device__ __forceinline__ void read_turns(const float2* row, int l, float2 (&turn)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 two = *reinterpret_cast<const float4*>(row + i * 16 + l * 2);
        turn[2 * i] = make_float2(two.x, two.y);
        turn[2 * i + 1] = make_float2(two.z, two.w);
    }
}

template <class T> __device__ __forceinline__ void load_pieces(const void* base, size_t element, const Pieces& p, uint32_t (&x)[4], uint32_t (&y)[4]) {
    const uint4* row = reinterpret_cast<const uint4*>((const uint16_t*)base + element);
    const uint4 u = row[p.p0], v = row[p.p1];
    x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w;
    y[0] = v.x, y[1] = v.y, y[2] = v.z, y[3] = v.w;
}
__device__ __forceinline__ void store_pieces(void* base, size_t element, const Pieces& p, const uint32_t (&x)[4], const uint32_t (&y)[4]) {
    uint4* row = reinterpret_cast<uint4*>((uint16_t*)base + element);
    row[p.p0] = make_uint4(x[0], x[1], x[2], x[3]);
    row[p.p1] = make_uint4(y[0], y[1], y[2], y[3]);
}

__device__ __forceinline__ int position_of(const TurnArgs& t, int token, int place, int pair) {
    return t.positions ? t.positions[axis_of(t, pair) * t.axis_stride + token] : place;
}

// First block of sequence b: sequences get a block for every `block` tokens or part of it, and one more for a start inside of one.
__device__ __forceinline__ int first_block(const int* cu_new, int b, int block) { return cu_new[b] / block + 2 * b; }
// The sequence of a block, by 64 candidates at a time.
__device__ __forceinline__ int sequence_of(const int* cu_new, int batch, int block, int at, int lane) {
    int lo = 0, left = batch;
    while (left > 1) {
        const int step = (left + kWave - 1) / kWave, i = lane * step;
        const unsigned long long in = __ballot(i < left && first_block(cu_new, lo + min(i, left - 1), block) <= at);
        const int n = max(__popcll(in) - 1, 0) * step;
        left = min(step, left - n);
        lo += n;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

}  // namespace

// A workgroup has a block of `block` neighbouring tokens of a sequence, aligned in the sequence and at least a logical page, and works out its
// angles once, into LDS.  Its wavefronts, and those of the `share` workgroups of the block, take heads in turn: keys, values, queries; eight lanes to
// a row and eight tokens of a head at a time, so that the rows of a page are written next to each other and a logical page's
// range stays in the registers of one wavefront.
template <class T, int LAYOUT, int BITS>
__global__ __launch_bounds__(kAppendThreads) void turned_append_kernel(TurnedAppendArgs a, int block, int share) {
    extern __shared__ float2 lds[];  // [block][kTurnRow], then for kOddHalves a row of channels for every row in hand
    const LayerParams& lp = a.lp;
    const PagedParams& kv = a.kv;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int part = blockIdx.x % share, at = blockIdx.x / share;
    const int b = sequence_of(a.cu_new, kv.batch, block, at, lane);
    const int src0 = a.cu_new[b], s = a.start_pos[b], e = s + min(a.cu_new[b + 1], a.total) - src0;
    const int lo = (s / block + at - first_block(a.cu_new, b, block)) * block;
    const int t0 = max(lo, s), t1 = min(lo + block, e);
    if (t0 >= t1) return;

    const int pairs = a.turn.rotary_dim / 2;
    if (lane < pairs) {
        const double f = a.turn.inv_freq[lane];
        for (int t = t0 + wave; t < t1; t += kAppendWaves)
            lds[(t - lo) * kTurnRow + turn_place<LAYOUT>(lane)] = turn_of(position_of(a.turn, src0 + t - s, t, lane), f, a.turn.scale);
    }
    __syncthreads();

    const int l = lane % 8, r = lane / 8;
    const Pieces p = pieces_of<LAYOUT>(l, a.turn.rotary_dim);
    float* room = reinterpret_cast<float*>(lds + block * kTurnRow) + (wave * 8 + r) * kHeadDim;
    const int page = lo / lp.NP, heads_q = a.q ? lp.H : 0;
    const int rows = min(lp.NL, 8);  // of a logical page among the eight rows in hand
    auto turn_it = [&](uint32_t (&x)[4], uint32_t (&y)[4], int t, const float* weight) {
        float2 turn[8];
        const float2* row = lds + (t - lo) * kTurnRow;
        if constexpr (LAYOUT != kOddHalves) read_turns(row, l, turn);
        turn_row<T, LAYOUT>(x, y, turn, a.turn, weight, p, room, row);
    };

    for (int u = wave + kAppendWaves * part; u < 2 * lp.Hkv + heads_q; u += kAppendWaves * share) {
        if (u >= 2 * lp.Hkv) {  // queries
            const int h = u - 2 * lp.Hkv;
            const float* weight = a.turn.q_weight ? a.turn.q_weight + (size_t)h * a.turn.weight_step : nullptr;
            for (int j = 0; j < block; j += 8) {
                const int t = lo + j + r, held = min(max(t, t0), t1 - 1);
                const size_t src = (size_t)(src0 + held - s);
                uint32_t x[4], y[4];
                load_pieces<T>(a.q, src * a.q_stride + h * kHeadDim, p, x, y);
                turn_it(x, y, held, weight);
                if (t == held) store_pieces(a.q_out, (src * lp.H + h) * kHeadDim, p, x, y);
            }
            continue;
        }
        const bool is_v = u >= lp.Hkv;
        const int hk = is_v ? u - lp.Hkv : u;
        const bool streaming = (lp.streaming_mask >> hk) & 1ull;
        // bounded pool: only sink pages and those that are local once all new tokens are in
        const bool kept = !in_stream_pool(lp, kv, hk) || page < lp.sink_pages || page >= ceil_div(e, lp.NP) - lp.local_pages;
        void* dense = is_v ? a.v_out : a.k_out;
        if (!kept && !dense) continue;
        Slab slab = {};
        if (kept) slab = slab_of(lp, kv, b, hk, page, BITS);
        const float* weight = a.turn.k_weight ? a.turn.k_weight + (size_t)hk * a.turn.weight_step : nullptr;
        RowRange<T> range_x, range_y;
        for (int j = 0; j < block; j += 8) {
            const int t = lo + j + r, held = min(max(t, t0), t1 - 1);
            const bool there = t == held;
            const size_t src = (size_t)(src0 + held - s);
            uint32_t x[4], y[4];
            load_pieces<T>(is_v ? a.v : a.k, src * (is_v ? a.v_stride : a.k_stride) + hk * kHeadDim, p, x, y);
            if (!is_v) turn_it(x, y, held, weight);
            if (there) {
                if (kept) write_row<T, BITS>(is_v ? slab.v : slab.k, lp.NP, held - page * lp.NP, p, l, x, y);
                if (dense) store_pieces(dense, (src * lp.Hkv + hk) * kHeadDim, p, x, y);
            }
            if (is_v || streaming) continue;
            if (there) {
                range_x.add(make_uint4(x[0], x[1], x[2], x[3]));
                range_y.add(make_uint4(y[0], y[1], y[2], y[3]));
            }
            if ((j + 8) % lp.NL != 0 && lp.NL > 8) continue;
            // a logical page ends here, or several do
            float xh[8], xl[8], yh[8], yl[8];
            auto larger_of = [](float u, float v) { return fmaxf(u, v); };
            auto smaller_of = [](float u, float v) { return fminf(u, v); };
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                xh[i] = over_rows(range_x.largest(i), rows, larger_of);
                xl[i] = over_rows(range_x.smallest(i), rows, smaller_of);
                yh[i] = over_rows(range_y.largest(i), rows, larger_of);
                yl[i] = over_rows(range_y.smallest(i), rows, smaller_of);
            }
            const int first = t / lp.NL * lp.NL;  // of the row's logical page
            if (r % rows == 0 && first < t1 && first + lp.NL > t0) {
                uint4* stats = reinterpret_cast<uint4*>(kv.stats) + ((slab.page_head * lp.g + (first - page * lp.NP) / lp.NL) * 2) * (kHeadDim / 8);
                write_range<T>(stats, p.p0, xh, xl, first < s);
                write_range<T>(stats, p.p1, yh, yl, first < s);
            }
            range_x = RowRange<T>();
            range_y = RowRange<T>();
        }
    }
}

// At most one new token per sequence (a decode step): nothing but latency.  A wavefront has eight heads of one token, works out the token's angles, one
// to a lane, and passes them round through LDS; all loads that depend on nothing but the position go out together.
template <class T, int LAYOUT, int BITS>
__global__ __launch_bounds__(kAppendThreads) void turned_step_kernel(TurnedAppendArgs a, int groups_q, int groups_kv) {
    __shared__ float2 all_turns[kAppendWaves][kTurnRow];
    __shared__ float rooms[LAYOUT == kOddHalves ? kAppendWaves * 8 : 1][kHeadDim];
    const LayerParams& lp = a.lp;
    const PagedParams& kv = a.kv;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, l = lane % 8, r = lane / 8;
    const int groups = groups_q + 2 * groups_kv, unit = blockIdx.x * kAppendWaves + wave;
    const int b = unit / groups, group = unit % groups;
    if (b >= kv.batch) return;
    const int src = a.cu_new[b], s = a.start_pos[b];
    if (a.cu_new[b + 1] <= src || src >= a.total) return;  // no new token
    const int kind = group < groups_kv ? 0 : group < 2 * groups_kv ? 1 : 2;  // keys, values, queries
    const int heads = kind == 2 ? lp.H : lp.Hkv, h = (group - kind * groups_kv) * 8 + r;
    const bool there = h < heads;
    const int head = there ? h : 0;
    const Pieces p = pieces_of<LAYOUT>(l, a.turn.rotary_dim);
    const void* from = kind == 0 ? a.k : kind == 1 ? a.v : a.q;
    const long long stride = kind == 0 ? a.k_stride : kind == 1 ? a.v_stride : a.q_stride;
    uint32_t x[4], y[4];
    load_pieces<T>(from, (size_t)src * stride + head * kHeadDim, p, x, y);
    if (kind != 1) {
        const int pairs = a.turn.rotary_dim / 2;
        float2* turns = all_turns[wave];
        if (lane < pairs) turns[turn_place<LAYOUT>(lane)] = turn_of(position_of(a.turn, src, s, lane), a.turn.inv_freq[lane], a.turn.scale);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        float2 turn[8];
        if constexpr (LAYOUT != kOddHalves) read_turns(turns, l, turn);
        const float* weight = kind == 2 ? a.turn.q_weight : a.turn.k_weight;
        if (weight) weight += (size_t)head * a.turn.weight_step;
        turn_row<T, LAYOUT>(x, y, turn, a.turn, weight, p, rooms[LAYOUT == kOddHalves ? wave * 8 + r : 0], turns);
    }
    if (!there) return;
    void* dense = kind == 0 ? a.k_out : kind == 1 ? a.v_out : a.q_out;
    if (dense) store_pieces(dense, ((size_t)src * heads + head) * kHeadDim, p, x, y);
    if (kind == 2) return;
    // the one new token is the last of its sequence, so its page is a local one: a bounded pool always keeps it
    const int page = s / lp.NP, slot = s - page * lp.NP;
    const Slab slab = slab_of(lp, kv, b, head, page, BITS);
    write_row<T, BITS>(kind == 0 ? slab.k : slab.v, lp.NP, slot, p, l, x, y);
    if (kind == 1 || ((lp.streaming_mask >> head) & 1ull)) return;
    RowRange<T> range_x, range_y;
    range_x.add(make_uint4(x[0], x[1], x[2], x[3]));
    range_y.add(make_uint4(y[0], y[1], y[2], y[3]));
    float xh[8], xl[8], yh[8], yl[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        xh[i] = range_x.largest(i);
        xl[i] = range_x.smallest(i);
        yh[i] = range_y.largest(i);
        yl[i] = range_y.smallest(i);
    }
    const int j = slot / lp.NL;
    const bool held = slot - j * lp.NL != 0;
    uint4* stats = reinterpret_cast<uint4*>(kv.stats) + ((slab.page_head * lp.g + j) * 2) * (kHeadDim / 8);
    write_range<T>(stats, p.p0, xh, xl, held);
    write_range<T>(stats, p.p1, yh, yl, held);
}

namespace {

template <class T, int LAYOUT, int BITS> hipError_t launch(const TurnedAppendArgs& a, hipStream_t stream) {
    const dim3 threads(kAppendThreads);
    if (a.max_new == 1) {
        const int groups_q = a.q ? ceil_div(a.lp.H, 8) : 0, groups_kv = ceil_div(a.lp.Hkv, 8);
        const long long waves = (long long)a.kv.batch * (groups_q + 2 * groups_kv);
        hipLaunchKernelGGL((turned_step_kernel<T, LAYOUT, BITS>), dim3((unsigned)((waves + kAppendWaves - 1) / kAppendWaves)), threads, 0, stream, a, groups_q,
                           groups_kv);
        return hipGetLastError();
    }
    const int block = std::max(16, a.lp.NL);
    const long long blocks = a.total / block + 2LL * a.kv.batch;
    const int units = 2 * a.lp.Hkv + (a.q ? a.lp.H : 0);
    const int share = (int)std::max(1LL, std::min<long long>(ceil_div(units, kAppendWaves), 8LL * num_compute_units() / blocks));
    const size_t lds = (size_t)block * kTurnRow * sizeof(float2) + (LAYOUT == kOddHalves ? kAppendWaves * 8 * kHeadDim * sizeof(float) : 0);
    hipLaunchKernelGGL((turned_append_kernel<T, LAYOUT, BITS>), dim3((unsigned)(blocks * share)), threads, lds, stream, a, block, share);
    return hipGetLastError();
}

template <class T, int LAYOUT> hipError_t launch_bits(const TurnedAppendArgs& a, hipStream_t stream) {
    return a.kv.kv_bits == 8 ? launch<T, LAYOUT, 8>(a, stream) : a.kv.kv_bits == 4 ? launch<T, LAYOUT, 4>(a, stream) : launch<T, LAYOUT, 16>(a, stream);
}
template <class T> hipError_t launch_layout(const TurnedAppendArgs& a, hipStream_t stream) {
    if (a.turn.interleaved) return launch_bits<T, kInterleaved>(a, stream);
    return a.turn.rotary_dim % 16 == 0 ? launch_bits<T, kHalves>(a, stream) : launch_bits<T, kOddHalves>(a, stream);
}

}  // namespace

hipError_t preload_rotary_append_kernels() {
    hipFuncAttributes attr;
    return hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&turned_step_kernel<F16, kHalves, 16>));
}

hipError_t launch_turned_append(int dtype, const TurnedAppendArgs& a, hipStream_t stream) {
    return dtype == 0 ? launch_layout<F16>(a, stream) : launch_layout<BF16>(a, stream);
}

}  // namespace lserve
