// New tokens on their way from a projection into the paged cache: queries normed and turned, keys normed, turned and written to their pages
// (16-bit rows or codes) with the key statistics brought up to date, values written next to them.  The cache is left as lserve_append_kv would
// leave it, handed the turned keys.  Bound: HBM, every row read once, queries and pages written once: 65536 tokens of 32 / 8 heads, 1.62 GB
// with 16-bit pages, 300 us = 5.4 TB/s (a copy of 671 MiB runs at 5.3); eight of 512 to 8192 into 8-bit pages with dense keys and values kept, 618 MB, 120 to
// 126 us (under the profiler 118 at least, 132 in the median); 16 single tokens 4.1 us, which is a launch and the loads of a place, an angle, a row and a page
// one after the other, 4.8 into pages of codes.
#include <algorithm>

#include "quantize.h"
#include "rotary.h"

namespace lserve {

namespace {

constexpr int kAppendThreads = 256, kAppendWaves = kAppendThreads / kWave;
constexpr int kStepThreads = 256, kStepWaves = kStepThreads / kWave;

// Larger (or smaller) of eight pairs of channels, as numbers, in the type that they are in.  (What is not a number gives way: to the other, or to nothing.)
template <class T, bool LARGER> __device__ __forceinline__ uint4 further(const uint32_t (&x)[4], const uint4& y4) {
    const uint32_t y[4] = {y4.x, y4.y, y4.z, y4.w};
    uint32_t out[4];
    auto of = [](float a, float b) { return LARGER ? fmaxf(fmaxf(-INFINITY, quieted<T>(a)), b) : fminf(fminf(INFINITY, quieted<T>(a)), b); };
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = Elem<T>::pack(of(Elem<T>::lo(x[i]), Elem<T>::lo(y[i])), of(Elem<T>::hi(x[i]), Elem<T>::hi(y[i])));
    return make_uint4(out[0], out[1], out[2], out[3]);
}

// Where the rows of a KV head of a page go.
struct Slab {
    uint4 *k, *v;
    size_t page_head;  // (page, head) index inside the pool
};
// Physical pages of page p of sequence b, in the main pool and in the ring.
struct Pages {
    int main, ring;
};
__device__ __forceinline__ Pages pages_of(const LayerParams& lp, const PagedParams& kv, int b, int p) {
    // (with every head in the ring the page table may be narrower than the sequence)
    return {kv.k_stream && kv.stream_heads == lp.Hkv ? 0 : kv.page_table[(size_t)b * kv.max_pages + p],
            kv.k_stream ? kv.ring_table[(size_t)b * kv.ring + ring_slot(lp, p)] : 0};
}
__device__ __forceinline__ Slab slab_of(const LayerParams& lp, const PagedParams& kv, const Pages& pages, int hk, int bits) {
    const bool ring = in_stream_pool(lp, kv, hk);
    const int phys = ring ? pages.ring : pages.main;
    const size_t ph = (size_t)phys * (ring ? kv.stream_heads : kv.pool_heads) + pool_rank(lp, kv, hk, ring);
    uint4 *k = reinterpret_cast<uint4*>(const_cast<void*>(ring ? kv.k_stream : kv.k_pool)),
          *v = reinterpret_cast<uint4*>(const_cast<void*>(ring ? kv.v_stream : kv.v_pool));
    return {k + ph * slab_chunks(lp.NP, bits), v + ph * slab_chunks(lp.NP, bits), ph};
}

// A lane's two pieces of a row as a page of BITS keeps them, and on their way to a slot.
template <int BITS> struct Stored {
    uint2 x, y;
    uint32_t pair;
};
template <> struct Stored<16> {
    uint4 x, y;
};
template <class T, int BITS> __device__ __forceinline__ Stored<BITS> stored(const uint32_t (&x)[4], const uint32_t (&y)[4]) {
    Stored<BITS> s;
    if constexpr (BITS == 16)
        s = {make_uint4(x[0], x[1], x[2], x[3]), make_uint4(y[0], y[1], y[2], y[3])};
    else
        quantize_pieces<T, BITS>(x, y, s.x, s.y, s.pair);
    return s;
}
template <int BITS> __device__ __forceinline__ void write_row(uint4* slab, int page_size, int slot, const Pieces& p, int l, const Stored<BITS>& s) {
    const size_t row = (size_t)slot * (kHeadDim / 8);
    if constexpr (BITS == 16) {
        slab[row + p.p0] = s.x;
        slab[row + p.p1] = s.y;
    } else {
        if constexpr (BITS == 8) {
            reinterpret_cast<uint2*>(slab)[row + p.p0] = s.x;
            reinterpret_cast<uint2*>(slab)[row + p.p1] = s.y;
        } else {
            reinterpret_cast<uint32_t*>(slab)[row + p.p0] = s.x.x;
            reinterpret_cast<uint32_t*>(slab)[row + p.p1] = s.y.x;
        }
        if (l == 0) reinterpret_cast<uint32_t*>(slab + page_size * (kHeadDim * BITS / 128))[slot] = s.pair;
    }
}

// Sixteen-byte pieces of LDS for a wavefront: sixteen 16-bit rows, or (kOddHalves, at another time) eight 32-bit ones.
constexpr int kTile = 16 * kHeadDim / 8;

__device__ __forceinline__ int position_of(const TurnArgs& t, int token, int place, int pair) {
    return t.positions ? t.positions[axis_of(t, pair) * t.axis_stride + token] : place;
}

// First block of a sequence: each gets a block for every `block` tokens or part of it, and one more for a start inside of one.
__device__ __forceinline__ int first_block(int cu, int b, int block) { return cu / block + 2 * b; }
// The sequence of a block, by 64 candidates at a time, with its first row, the first row behind it and its first position.
struct Found {
    int b, cu, cu_next, start;
};
__device__ __forceinline__ Found sequence_of(const int* cu_new, const int* start_pos, int batch, int block, int at, int lane) {
    int lo = 0, left = batch;
    while (true) {
        const int step = (left + kWave - 1) / kWave, i = lo + min(lane * step, left - 1);
        const int cu = cu_new[i], cu_next = cu_new[i + 1], start = start_pos[i];
        const unsigned long long in = __ballot(lane * step < left && first_block(cu, i, block) <= at);
        const int n = max(__popcll(in) - 1, 0);
        if (step == 1)
            return {lo + n, __builtin_amdgcn_readlane(cu, n), __builtin_amdgcn_readlane(cu_next, n), __builtin_amdgcn_readlane(start, n)};
        lo += n * step;
        left = min(step, left - n * step);
    }
}

}  // namespace

// A workgroup has a block of `block` neighbouring tokens of a sequence, aligned in the sequence and at least a logical page, and works out its
// angles once, into LDS.  Its wavefronts, and those of the `share` workgroups of the block, take units in turn, eight lanes to a row and twice eight rows at
// a time: a KV head of keys or values, sixteen tokens at a time, so that the rows of a page are written next to each other; or eight heads of the queries,
// two tokens at a time.  The next sixteen rows are in flight while sixteen are worked on.
template <class T, int LAYOUT, int BITS, bool NORM>
__global__ __launch_bounds__(kAppendThreads) void turned_append_kernel(TurnedAppendArgs a, int block, int share) {
    extern __shared__ float2 lds[];  // [block][kTurnRow], then a tile for every wavefront
    const LayerParams& lp = a.lp;
    const PagedParams& kv = a.kv;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    // (workgroups go to the XCDs in turn: the parts, some of them dearer, move on by one with every block)
    const int at = blockIdx.x / share, part = (blockIdx.x + at) % share;
    const Found found = sequence_of(a.cu_new, a.start_pos, kv.batch, block, at, lane);
    const int b = found.b, src0 = found.cu, s = found.start, e = s + (min(found.cu_next, a.total) - src0);
    const int nth = s / block + at - first_block(src0, b, block);
    if ((unsigned)nth * block >= (unsigned)max(e, 0)) return;
    const int lo = nth * block;
    const int t0 = max(lo, s), t1 = lo + min(block, e - lo);  // (the block may end past 2^31)
    if (t0 >= t1) return;

    const int page = lo / lp.NP, in_page = lo - page * lp.NP;
    const Pages pages = pages_of(lp, kv, b, page);
    const int l = lane % 8, r = lane / 8;
    const Pieces p = pieces_of<LAYOUT>(l, a.turn.rotary_dim);
    const int chunks = block / 16, groups = a.q ? ceil_div(lp.H, 8) : 0, stride = kAppendWaves * share;
    const int units = 2 * lp.Hkv + groups * ceil_div(t1 - t0, 2 * chunks);  // (queries: of the tokens that there are)
    // a row: its token (held back inside the block's tokens), its head, whether it is there at all
    struct Row {
        int t, head, there;
    };
    auto row_of = [&](int u, int c, int half) {
        int t, h;
        if (u < 2 * lp.Hkv) {
            t = lo + 16 * c + 8 * half + r;
            h = u < lp.Hkv ? u : u - lp.Hkv;
        } else {
            const int i = u - 2 * lp.Hkv;
            t = t0 + min((i / groups * chunks + c) * 2 + half, t1 - t0);
            h = i % groups * 8 + r;
        }
        const int held = min(max(t, t0), t1 - 1), head = min(h, lp.H - 1);
        return Row{held, head, t == held && h == head};
    };
    auto ask = [&](int u, int c, uint32_t (&x)[2][4], uint32_t (&y)[2][4]) {
        const void* from = u >= 2 * lp.Hkv ? a.q : u >= lp.Hkv ? a.v : a.k;
        const long long apart = u >= 2 * lp.Hkv ? a.q_stride : u >= lp.Hkv ? a.v_stride : a.k_stride;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const Row row = row_of(u, c, half);
            load_pieces(from, (size_t)(src0 + (row.t - s)) * apart + row.head * kHeadDim, p, x[half], y[half]);
        }
    };
    int u = wave + kAppendWaves * part, c = 0;
    uint32_t x[2][4] = {}, y[2][4] = {}, next_x[2][4], next_y[2][4];
    if (u < units) ask(u, 0, x, y);

    const int pairs = a.turn.rotary_dim / 2;
    if (lane < pairs) {
        const double f = a.turn.inv_freq[lane];
        for (int i = t0 - lo + wave; i < t1 - lo; i += kAppendWaves)
            lds[i * kTurnRow + turn_place<LAYOUT>(lane)] = turn_of(position_of(a.turn, src0 + (lo - s) + i, lo + i, lane), f, a.turn.scale);
    }
    __syncthreads();

    uint4* tile = reinterpret_cast<uint4*>(lds + block * kTurnRow) + wave * kTile;
    float* room = reinterpret_cast<float*>(tile) + r * kHeadDim;
    float high[2] = {-INFINITY, -INFINITY}, low[2] = {INFINITY, INFINITY};  // of the lane's two channels in a logical page
    while (u < units) {
        const bool is_q = u >= 2 * lp.Hkv, is_v = !is_q && u >= lp.Hkv;
        const Row rows[2] = {row_of(u, c, 0), row_of(u, c, 1)};
        const float* weight = !NORM || is_v ? nullptr : is_q ? a.turn.q_weight : a.turn.k_weight;
        Weights w;  // (asked for ahead of the next rows: loads come back in order)
        if (weight) weight += (size_t)rows[0].head * a.turn.weight_step;
        if (NORM) load_weights(weight, p, w);
        const int next_c = c + 1 < chunks ? c + 1 : 0, next_u = next_c ? u : u + stride;
        ask(next_u < units ? next_u : u, next_u < units ? next_c : c, next_x, next_y);  // (its own once more behind its last unit: no branch)
        if (!is_v) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float2 turn[8];
                const float2* turns = lds + (rows[half].t - lo) * kTurnRow;
                if constexpr (LAYOUT != kOddHalves) read_turns(turns, l, turn);
                turn_row<T, LAYOUT, NORM>(x[half], y[half], turn, a.turn, weight != nullptr, w, p, room, turns);
            }
        }
        if (is_q) {
            arrived(next_x[0], next_y[0]);
            arrived(next_x[1], next_y[1]);
#pragma unroll
            for (int half = 0; half < 2; ++half)
                if (rows[half].there) store_pieces(a.q_out, ((size_t)(src0 + (rows[half].t - s)) * lp.H + rows[half].head) * kHeadDim, p, x[half], y[half]);
        } else {
            const int hk = is_v ? u - lp.Hkv : u;
            // bounded pool: only sink pages and those that are local once all new tokens are in
            const bool kept = !in_stream_pool(lp, kv, hk) || page < lp.sink_pages || page > (e - 1) / lp.NP - lp.local_pages;
            const bool scored = !is_v && !((lp.streaming_mask >> hk) & 1ull);
            if (scored) {
                // The rows change hands in LDS: two channels to a lane, so that a range is four registers and needs no other lane
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint4* to = tile + (8 * half + r) * (kHeadDim / 8);
                    to[p.p0] = make_uint4(x[half][0], x[half][1], x[half][2], x[half][3]);
                    to[p.p1] = make_uint4(y[half][0], y[half][1], y[half][2], y[half][3]);
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
            const Stored<BITS> first_row = stored<T, BITS>(x[0], y[0]), second_row = stored<T, BITS>(x[1], y[1]);
            arrived(next_x[0], next_y[0]);
            arrived(next_x[1], next_y[1]);
            void* dense = is_v ? a.v_out : a.k_out;
            if (dense) {
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    if (rows[half].there) store_pieces(dense, ((size_t)(src0 + (rows[half].t - s)) * lp.Hkv + hk) * kHeadDim, p, x[half], y[half]);
            }
            const Slab slab = slab_of(lp, kv, pages, hk, BITS);
            if (kept) {
                uint4* to = is_v ? slab.v : slab.k;
                if (rows[0].there) write_row<BITS>(to, lp.NP, in_page + (rows[0].t - lo), p, l, first_row);
                if (rows[1].there) write_row<BITS>(to, lp.NP, in_page + (rows[1].t - lo), p, l, second_row);
            }
            if (scored) {
                const int from = lo + 16 * c;
                uint32_t keys[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) keys[i] = reinterpret_cast<const uint32_t*>(tile)[i * (kHeadDim / 2) + lane];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int t = from + i;
                    if (t < t0 || t >= t1) continue;
                    const float first_channel = quieted<T>(Elem<T>::lo(keys[i])), second_channel = quieted<T>(Elem<T>::hi(keys[i]));
                    high[0] = fmaxf(high[0], first_channel);
                    high[1] = fmaxf(high[1], second_channel);
                    low[0] = fminf(low[0], first_channel);
                    low[1] = fminf(low[1], second_channel);
                    if ((t + 1) % lp.NL != 0 && t + 1 != t1) continue;
                    // the logical page ends here, or the new tokens do
                    const int first = t / lp.NL * lp.NL;
                    uint32_t* stats = reinterpret_cast<uint32_t*>(kv.stats) + ((slab.page_head * lp.g + (first - page * lp.NP) / lp.NL) * 2) * (kHeadDim / 2) + lane;
                    if (first < s) {  // it held tokens before
                        const uint32_t most = stats[0], least = stats[kHeadDim / 2];
                        high[0] = fmaxf(high[0], Elem<T>::lo(most));
                        high[1] = fmaxf(high[1], Elem<T>::hi(most));
                        low[0] = fminf(low[0], Elem<T>::lo(least));
                        low[1] = fminf(low[1], Elem<T>::hi(least));
                    }
                    stats[0] = Elem<T>::pack(high[0], high[1]);
                    stats[kHeadDim / 2] = Elem<T>::pack(low[0], low[1]);
                    high[0] = high[1] = -INFINITY;
                    low[0] = low[1] = INFINITY;
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (the next rows take the tile over)
            }
        }
        u = next_u;
        c = next_c;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[half][i] = next_x[half][i];
                y[half][i] = next_y[half][i];
            }
        }
    }
}

// One new token per sequence (a decode step), or a few (drafted ones that were accepted): nothing but latency.  A wavefront has eight heads of a sequence and
// takes its tokens one after the other; their angles are worked out one to a lane and passed round through LDS, and all loads that depend on nothing
// but the position go out together.  The range of a logical page stays in the lanes from token to token.
template <class T, int LAYOUT, int BITS, bool NORM>
__global__ __launch_bounds__(kStepThreads) void turned_step_kernel(TurnedAppendArgs a, int groups_q, int groups_kv) {
    __shared__ float2 all_turns[kStepWaves][kTurnRow];
    __shared__ float rooms[LAYOUT == kOddHalves ? kStepWaves * 8 : 1][kHeadDim];
    const LayerParams& lp = a.lp;
    const PagedParams& kv = a.kv;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, l = lane % 8, r = lane / 8;
    const int groups = groups_q + 2 * groups_kv, unit = blockIdx.x * kStepWaves + wave;
    const int b = unit / groups, group = unit % groups;
    if (b >= kv.batch) return;
    const int src0 = a.cu_new[b], start = a.start_pos[b], n = min(a.cu_new[b + 1], a.total) - src0;
    if (n <= 0) return;  // no new token
    const int kind = group < groups_kv ? 0 : group < 2 * groups_kv ? 1 : 2;  // keys, values, queries
    const int heads = kind == 2 ? lp.H : lp.Hkv, h = (group - kind * groups_kv) * 8 + r;
    const bool there = h < heads;
    const int head = there ? h : 0;
    const bool scored = kind == 0 && there && !((lp.streaming_mask >> head) & 1ull);
    const Pieces p = pieces_of<LAYOUT>(l, a.turn.rotary_dim);
    const long long stride = kind == 0 ? a.k_stride : kind == 1 ? a.v_stride : a.q_stride;
    const uint16_t* from = (const uint16_t*)(kind == 0 ? a.k : kind == 1 ? a.v : a.q) + (size_t)src0 * stride + head * kHeadDim;
    void* dense = kind == 0 ? a.k_out : kind == 1 ? a.v_out : a.q_out;
    float2* turns = all_turns[wave];
    const uint32_t inf = Elem<T>::pack(INFINITY, INFINITY), none = inf | 0x80008000u;
    uint4 range[4];  // of the logical page: largest of either piece, smallest
    uint32_t x[4], y[4], next_x[4], next_y[4];
    load_pieces(from, 0, p, x, y);
    for (int i = 0; i < n; ++i) {
        const int s = start + i, page = s / lp.NP, slot = s - page * lp.NP, j = slot / lp.NL;
        Slab slab = {};
        uint4* stats = nullptr;
        bool kept = true;
        if (kind != 2) {
            slab = slab_of(lp, kv, pages_of(lp, kv, b, page), head, BITS);
            // bounded pool: only sink pages and those that are local once all new tokens are in
            kept = !in_stream_pool(lp, kv, head) || page < lp.sink_pages || page > (start + (n - 1)) / lp.NP - lp.local_pages;
            if (scored) {
                stats = reinterpret_cast<uint4*>(kv.stats) + ((slab.page_head * lp.g + j) * 2) * (kHeadDim / 8);
                if (slot == j * lp.NL) {  // nothing yet: infinities of either sign
                    range[0] = range[1] = make_uint4(none, none, none, none);
                    range[2] = range[3] = make_uint4(inf, inf, inf, inf);
                } else if (i == 0) {
                    range[0] = stats[p.p0], range[1] = stats[p.p1];
                    range[2] = stats[kHeadDim / 8 + p.p0], range[3] = stats[kHeadDim / 8 + p.p1];
                }
            }
        }
        Weights w;  // (asked for ahead of the next rows: loads come back in order)
        const float* weight = !NORM || kind == 1 ? nullptr : kind == 2 ? a.turn.q_weight : a.turn.k_weight;
        if (weight) weight += (size_t)head * a.turn.weight_step;
        if (NORM) load_weights(weight, p, w);
        if (i + 1 < n) load_pieces(from, (size_t)(i + 1) * stride, p, next_x, next_y);
        if (kind != 1) {
            if (lane < a.turn.rotary_dim / 2)
                turns[turn_place<LAYOUT>(lane)] = turn_of(position_of(a.turn, src0 + i, s, lane), a.turn.inv_freq[lane], a.turn.scale);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            float2 turn[8];
            if constexpr (LAYOUT != kOddHalves) read_turns(turns, l, turn);
            turn_row<T, LAYOUT, NORM>(x, y, turn, a.turn, weight != nullptr, w, p, rooms[LAYOUT == kOddHalves ? wave * 8 + r : 0], turns);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (the next token's angles take their place)
        }
        if (there && dense) store_pieces(dense, ((size_t)(src0 + i) * heads + head) * kHeadDim, p, x, y);
        if (there && kind != 2 && kept) write_row<BITS>(kind == 0 ? slab.k : slab.v, lp.NP, slot, p, l, stored<T, BITS>(x, y));
        if (scored) {
            range[0] = further<T, true>(x, range[0]);
            range[1] = further<T, true>(y, range[1]);
            range[2] = further<T, false>(x, range[2]);
            range[3] = further<T, false>(y, range[3]);
            if (i + 1 == n || (slot + 1) % lp.NL == 0) {
                stats[p.p0] = range[0];
                stats[p.p1] = range[1];
                stats[kHeadDim / 8 + p.p0] = range[2];
                stats[kHeadDim / 8 + p.p1] = range[3];
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            x[q] = next_x[q];
            y[q] = next_y[q];
        }
    }
}

namespace {

template <class T, int LAYOUT, int BITS, bool NORM> hipError_t launch(const TurnedAppendArgs& a, hipStream_t stream) {
    // A sequence's few tokens one after the other, a microsecond each, or blocks of sixteen places with as few rows in them,
    // of which more sequences are more: one sequence of two tokens 4.9 and 5.1 us, of three 5.6 and 5.2; 64 of two 5.1 and 6.6, of
    // three 6.2 and 7.5, of four 7.4 and 7.5, of six 9.6 and 9.4; 256 of four 10.1 and 13.1, of six 13.0 and 15.1, of eight 16.0 and
    // 13.3; 500 of two 8.7 and 14.6, of eight 26.5 and 31.5, of twelve 40 and 38.
    if (a.max_new <= 2 || (a.max_new <= 8 && (a.max_new - 2) * 64 <= a.kv.batch)) {
        const int groups_q = a.q ? ceil_div(a.lp.H, 8) : 0, groups_kv = ceil_div(a.lp.Hkv, 8);
        const long long waves = (long long)a.kv.batch * (groups_q + 2 * groups_kv);
        hipLaunchKernelGGL((turned_step_kernel<T, LAYOUT, BITS, NORM>), dim3((unsigned)((waves + kStepWaves - 1) / kStepWaves)), dim3(kStepThreads), 0, stream, a, groups_q,
                           groups_kv);
        return hipGetLastError();
    }
    const int block = std::max(16, a.lp.NL);
    const long long blocks = a.total / block + 2LL * a.kv.batch;
    const int each_seq = std::min(block, ceil_div(a.total, a.kv.batch));  // tokens of a block, where sequences are alike
    const int units = 2 * a.lp.Hkv + (a.q ? ceil_div(a.lp.H, 8) * ceil_div(8 * each_seq, block) : 0);
    // Parts of a block: enough for three workgroups to a compute unit, as long as every wavefront has a unit; with plenty of blocks few, as each part works out
    // the block's angles: with a norm, or where blocks are few all the same, four units to a wavefront, else two.  Two, three, four, six and twelve parts, us:
    // 65536 tokens of 32 / 8 heads 315, 311, 309, 303, 302, with a norm 311, 301, 315, 311, 404; 8 x 512 25.9, 24.0, 24.8, 25.6, 25.6; one
    // of 512 11.9, 10.5, 9.5, 8.8, 8.4, of 2000 13.8, 14.1, 12.9, 12.7, 15.0; 20000 of 64 / 8 165, 163, 160, 159, 152; 30000 into 4-bit pages 156, 148, 154,
    // 149, 191.  (A number that leaves some wavefronts a unit more than others costs: eight parts of 48 units 321 where six took 305.)
    const long long wanted = std::max<long long>(units / ((NORM || blocks < 4 * num_compute_units() ? 4 : 2) * kAppendWaves), 3LL * num_compute_units() / blocks);
    const int most = (int)std::max(1LL, std::min<long long>(ceil_div(units, kAppendWaves), wanted));
    const int each = ceil_div(units, kAppendWaves * most), share = ceil_div(units, kAppendWaves * each);  // as many to every wavefront
    const size_t lds = (size_t)block * kTurnRow * sizeof(float2) + kAppendWaves * kTile * sizeof(uint4);
    hipLaunchKernelGGL((turned_append_kernel<T, LAYOUT, BITS, NORM>), dim3((unsigned)(blocks * share)), dim3(kAppendThreads), lds, stream, a, block, share);
    return hipGetLastError();
}

template <class T, int LAYOUT, int BITS> hipError_t launch_norm(const TurnedAppendArgs& a, hipStream_t stream) {
    return a.turn.norm ? launch<T, LAYOUT, BITS, true>(a, stream) : launch<T, LAYOUT, BITS, false>(a, stream);
}
template <class T, int LAYOUT> hipError_t launch_bits(const TurnedAppendArgs& a, hipStream_t stream) {
    return a.kv.kv_bits == 8   ? launch_norm<T, LAYOUT, 8>(a, stream)
           : a.kv.kv_bits == 4 ? launch_norm<T, LAYOUT, 4>(a, stream)
                               : launch_norm<T, LAYOUT, 16>(a, stream);
}
template <class T> hipError_t launch_layout(const TurnedAppendArgs& a, hipStream_t stream) {
    if (a.turn.interleaved) return launch_bits<T, kInterleaved>(a, stream);
    return a.turn.rotary_dim % 16 == 0 ? launch_bits<T, kHalves>(a, stream) : launch_bits<T, kOddHalves>(a, stream);
}

}  // namespace

hipError_t preload_rotary_append_kernels() {
    hipFuncAttributes attr;
    return hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&turned_step_kernel<F16, kHalves, 16, false>));
}

hipError_t launch_turned_append(int dtype, const TurnedAppendArgs& a, hipStream_t stream) {
    return dtype == 0 ? launch_layout<F16>(a, stream) : launch_layout<BF16>(a, stream);
}

}  // namespace lserve
