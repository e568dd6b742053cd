// Attention of drafted tokens (Sec. 3.6's page lists under a tree of queries) on the gfx950 matrix cores.
//
// The drafted tokens of a sequence all read the same pages of history, so the rows that meet a KV head's keys are (drafted token, query
// head of the group): n G of them.  Two products of 4 n G D operations per key against the 512 bytes of its K and V row make n G operations
// per byte, and HBM is the bound up to some two hundred rows.  A list of keys is the head's pages of history followed by tiles of 64 drafted
// tokens, whose K and V come straight from the call's tensors; who sees whom there is one bit per (row, key).
//
// A workgroup owns 32 RG rows of one (sequence, KV head) and a stretch of its list, 64 keys a step, K and V brought into LDS by direct
// loads (quantised ones through registers), two stages.  Wavefront (rg, kg) works on row block rg and, of the step's keys, on half kg (RG = 1, 2) or
// all (RG = 4).  Scores are computed transposed, S^T = K Q^T, so that a lane owns a row and the softmax stays in the lane and
// its partner; the weights are then the second operand of O^T += V^T P^T as they are (see sparse_prefill.hip).
//
// Lists are cut into pieces of equal length by what the sequences hold when the kernel runs, which the host does not know: every
// workgroup works out the cut from the lengths of the batch (TreePlan).  Pieces leave (maximum, sum, outputs) in the workspace and
// fold_trees_kernel puts them together in order.
//
// Measured, calls back to back, both kernels and what is between them (a copy of 1 GiB runs at 5.1 TB/s, a product of 8192^3 at 1216 TFLOP/s): five tokens
// each on 4 x 256k, 2.15 GB, 365 .. 381 us = 5.6 .. 5.9 TB/s; 32 sequences of 4k .. 60k under 32 KV heads, 695 MB, 133 .. 140 us = 5.0 .. 5.2 TB/s; sixteen
// each on 16 x 32k, 4096 selected, 158 MB, 47 .. 49 us, of which 6.7 are the second kernel and some 8 the start (lengths, cut, page table, first tiles);
// one conversation of 4000 tokens 14.8 us, nothing but such latencies; twenty to 64 each on 64 x 16k in 4-bit pages 209 .. 213 us = 435 .. 445 TFLOP/s: there
// the vector instructions (50 % of a SIMD's cycles: unpacking, exponentials, packing) and the matrix ones (24 %) of two wavefronts to a SIMD add up with
// the barriers between; the same in 8-bit pages 215 .. 231.
#include <algorithm>

#include "kernels.h"
#include "matrix.h"

namespace lserve {

namespace {

constexpr int kTile = 64;                        // keys of a step: a page, or drafted tokens
constexpr int kRowBytes = kHeadDim * 2;          // of a 16-bit row
constexpr int kTileBytes = kTile * kRowBytes;
constexpr int kAhead = 4;                        // operand reads in flight ahead of the products
constexpr float kSlack = 6.f;                    // a row's reference moves when a weight would pass 2^kSlack
constexpr int kBlockFloat4 = 16 * kWave;         // outputs of a block of 32 rows, as the lanes hold them
constexpr int kLeastPiece = 2;                   // list entries

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// How a launch is laid out (host).
struct TreeLaunch {
    int target;     // pieces to cut the lists into, about; 0: lists stay whole
    int exact;      // no more than that
    int row_tiles;  // of 32 RG rows, of the longest sequence
    int streams;    // streaming heads
    int slots;      // of pieces in the workspace
    int folds;      // items of fold_trees_kernel: 32 rows, 32 channels
    float4* partials;
    float2* partial_ml;
    int2* pieces;   // [batch][Hkv][row_tiles]: (first slot, pieces)
};

// What sequence b asks for.  Everything is brought inside the arrays, whatever the lengths say.
struct SeqShape {
    int start, n, len, pages;  // first drafted token, how many, tokens and pages of history
    int then;                  // pages at the time of the selection
    int dense, stream;         // list entries of a head that attends a selection (or everything), of a streaming head
    int row_tiles;
};

__device__ __forceinline__ int first_local_page(const LayerParams& lp, int len) {
    // of the first drafted token, whose own tile is that of position `len`
    return max(lp.sink_pages, len / kTile - lp.local_pages + 1);
}

__device__ __forceinline__ int pages_of(int tokens) { return (int)(((unsigned)max(tokens, 0) + kTile - 1) / kTile); }

template <int R> __device__ __forceinline__ SeqShape seq_shape(const TreeArgs& a, int b) {
    SeqShape s;
    s.start = max(a.cu_new[b], 0);
    s.n = min(min(a.cu_new[b + 1] - s.start, a.max_new), a.total_new - s.start);
    s.len = (int)min((long long)max(a.kv.seq_lens[b], 0), min((long long)a.kv.max_pages * kTile, 0x7fffffc0LL));
    s.pages = ceil_div(s.len, kTile);
    const int drafts = ceil_div(max(s.n, 0), kTile);
    s.then = a.sel_pages ? min(pages_of(a.sel_seq_len[b]), s.pages) : s.pages;
    s.dense = (a.sel_pages ? min(s.then, a.sel_stride) : s.then) + s.pages - s.then + drafts;
    s.stream = min(a.lp.sink_pages, s.pages) + max(0, s.pages - first_local_page(a.lp, s.len)) + drafts;
    s.row_tiles = s.n > 0 ? ceil_div(s.n * a.lp.group, R) : 0;
    return s;
}

// Pieces of `span` list entries, or a few more.
struct TreePlan {
    int span;
    float reciprocal;
    __device__ __forceinline__ static TreePlan of(int span) { return {span, span ? __builtin_amdgcn_rcpf((float)span) : 0.f}; }
    __device__ __forceinline__ int pieces(int entries) const { return max(1, (int)ceilf((float)entries * reciprocal - 0.01f)); }
    __device__ __forceinline__ int dense_units(const TreeArgs& a, const TreeLaunch& t, const SeqShape& s) const {
        return s.row_tiles * (a.lp.Hkv - t.streams) * pieces(s.dense);
    }
    __device__ __forceinline__ int stream_units(const TreeLaunch& t, const SeqShape& s) const { return s.row_tiles * t.streams * pieces(s.stream); }
    __device__ __forceinline__ int units(const TreeArgs& a, const TreeLaunch& t, const SeqShape& s) const {
        return dense_units(a, t, s) + stream_units(t, s);
    }
};

__device__ __forceinline__ float wave_sum(float x) { return rows4_sum(row16_sum(x)); }

// (own: the shape of sequence `lane`, which is all there is to load for batches of up to 64)
template <int R> __device__ __forceinline__ TreePlan make_plan(const TreeArgs& a, const TreeLaunch& t, const SeqShape& own) {
    if (t.target == 0) return TreePlan::of(0);
    const int lane = threadIdx.x % kWave, batch = a.kv.batch, denses = a.lp.Hkv - t.streams;
    auto total = [&](auto f) {  // of f over the sequences
        float x = f(own);
        for (int base = kWave; base < batch; base += kWave)
            if (base + lane < batch) x += f(seq_shape<R>(a, base + lane));
        return wave_sum(x);
    };
    const float work = total([&](const SeqShape& s) { return (float)s.row_tiles * ((float)t.streams * s.stream + (float)denses * s.dense); });
    // what a workgroup that is always there has to do: nothing longer than that stays in one piece
    TreePlan plan = TreePlan::of(uniform(max(kLeastPiece, (int)min(work / t.target, 1e9f) + 1)));
    // (more lists than that: half as much again, so that most stay whole.  40 sequences of 100 .. 3000 tokens 49 -> 38 us, 64 over selected 4-bit
    // pages 253 -> 217, nine of 1000 .. 2000 under 32 KV heads 51 -> 43, others within 2 %; a quarter more, or less than that, is behind in one of them)
    if (!t.exact) return TreePlan::of(plan.span + plan.span / 2);
    // as long as it takes to have no more pieces than workgroups that run at once (they are at most twice as many to begin with)
    for (int i = 0; i < 24; ++i) {
        const float count = total([&](const SeqShape& s) { return (float)plan.units(a, t, s); });
        if (uniform(count <= (float)t.target)) break;
        plan = TreePlan::of(plan.span + max(1, plan.span / 16));
    }
    return plan;
}

// The unit-th piece of the launch.
struct TreeUnit {
    int b, hk, row_tile, piece, pieces;
};
template <int R>
__device__ __forceinline__ bool find_unit(const TreeArgs& a, const TreeLaunch& t, const TreePlan& plan, const SeqShape& own, int unit, TreeUnit& u,
                                          SeqShape& shape) {
    const int lane = threadIdx.x % kWave, batch = a.kv.batch;
    if (t.target == 0) {  // plenty of lists, all whole: by arithmetic, and not all of these row tiles exist
        u.row_tile = unit % t.row_tiles;
        unit /= t.row_tiles;
        u.hk = unit % a.lp.Hkv;
        u.b = unit / a.lp.Hkv;
        u.piece = 0;
        u.pieces = 1;
        if (u.b >= batch) return false;
        shape = seq_shape<R>(a, u.b);
        return u.row_tile < shape.row_tiles;
    }
    // heads that select, of all sequences, before streaming ones: what is long starts first
    bool streaming = false;
    for (int base = 0;; base += kWave) {
        if (base >= batch) {
            if (streaming || t.streams == 0) return false;
            streaming = true;
            base = 0;
        }
        SeqShape s = own;
        if (base > 0) s = base + lane < batch ? seq_shape<R>(a, base + lane) : SeqShape{};
        const int units = streaming ? plan.stream_units(t, s) : plan.dense_units(a, t, s);
        const int upto = wave_scan(units, 0, add);
        const int all = __builtin_amdgcn_readlane(upto, kWave - 1);
        if (unit >= all) {
            unit -= all;
            continue;
        }
        const int at = __builtin_ctzll(__ballot(upto > unit));
        u.b = base + at;
        shape.start = __builtin_amdgcn_readlane(s.start, at);
        shape.n = __builtin_amdgcn_readlane(s.n, at);
        shape.len = __builtin_amdgcn_readlane(s.len, at);
        shape.pages = __builtin_amdgcn_readlane(s.pages, at);
        shape.then = __builtin_amdgcn_readlane(s.then, at);
        shape.dense = __builtin_amdgcn_readlane(s.dense, at);
        shape.stream = __builtin_amdgcn_readlane(s.stream, at);
        shape.row_tiles = __builtin_amdgcn_readlane(s.row_tiles, at);
        unit -= __builtin_amdgcn_readlane(upto - units, at);
        break;
    }
    // of a sequence: heads, then pieces, then row tiles, which read the same keys
    u.pieces = plan.pieces(streaming ? shape.stream : shape.dense);
    u.row_tile = unit % shape.row_tiles;
    unit /= shape.row_tiles;
    u.piece = unit % u.pieces;
    int rank = unit / u.pieces;
    unsigned long long heads = streaming ? a.lp.streaming_mask : ~a.lp.streaming_mask;
    for (; rank > 0; --rank) heads &= heads - 1;
    u.hk = __builtin_ctzll(heads);
    return true;
}

typedef unsigned short ushort2_t __attribute__((ext_vector_type(2)));

template <class T> struct BitsOf;
template <> struct BitsOf<F16> { static constexpr uint32_t exponent = 0x7c00u; };
template <> struct BitsOf<BF16> { static constexpr uint32_t exponent = 0x7f80u; };

// Keys' codes as operands of the layer's type, exactly, a permutation of bytes to two of them where there is a number whose low bits they can be: the
// operand is code * unit + offset, and unit and offset go into the scale and zero that its score meets in fp32.
//   fp16: a code alone is the subnormal code * 2^-24, which the matrix instructions take at its value.
//   bf16: 0x4300 and four bits are 128 + code.  Eight bits do not fit behind a power of two; they are converted.
template <class T, int BITS> struct KeyCodes;
template <int BITS> struct KeyCodes<F16, BITS> {
    static constexpr float unit = 0x1p-24f, offset = 0.f;
    static constexpr uint32_t high = 0;
};
template <> struct KeyCodes<BF16, 4> {
    static constexpr float unit = 1.f, offset = 128.f;
    static constexpr uint32_t high = 0x43434343u;
};
template <> struct KeyCodes<BF16, 8> {
    static constexpr float unit = 1.f, offset = 0.f;
    static constexpr uint32_t high = 0;
};
template <class T, int BITS> __device__ __forceinline__ uint4 codes8(uint2 codes) {
    uint32_t lo = codes.x, hi = codes.y;  // channels 0..3 and 4..7, one byte each
    if constexpr (BITS == 4) {
        hi = (codes.x >> 4) & 0x0f0f0f0fu;
        lo = codes.x & 0x0f0f0f0fu;
    }
    if constexpr (std::is_same<T, BF16>::value && BITS == 8) {
        auto pair = [](uint32_t word, int at) {  // whole numbers up to 255 are the upper halves of their fp32 numbers
            const float a = (float)(word >> (8 * at) & 0xffu), b = (float)(word >> (8 * at + 8) & 0xffu);
            return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u);
        };
        return make_uint4(pair(lo, 0), pair(lo, 2), pair(hi, 0), pair(hi, 2));
    } else {
        constexpr uint32_t high = KeyCodes<T, BITS>::high;
        return make_uint4(__builtin_amdgcn_perm(high, lo, 0x04010400u), __builtin_amdgcn_perm(high, lo, 0x04030402u),
                          __builtin_amdgcn_perm(high, hi, 0x04010400u), __builtin_amdgcn_perm(high, hi, 0x04030402u));
    }
}

__device__ __forceinline__ uint2 two_words(uint2 x) { return x; }
__device__ __forceinline__ uint2 two_words(uint32_t x) { return make_uint2(x, 0u); }
// Values of quantised pages.  As fp16 numbers in LDS, next to weights rounded to fp16, they would make the second error of that size, and fp16 has not
// the range of a scale times a code: tiny rows would lose their scale, loud ones of a bf16 layer become infinite.  So LDS has (code - kMiddle) 2^e,
// which is exact, with 2^e the power of two in the row's scale (as far as fp16 has it), and what is left of the scale, in [1, 2) as a rule, meets the
// weight in fp32 before that is rounded.  The middle of the codes and the zero go into a sum of the row's own.  (Under a bf16 layer, against values
// rounded to fp16, which a fused multiply and add makes: 64 x 16k in 4-bit pages 193 -> 209 us, 4 x 100k 121 -> 125, in 8-bit pages 217 -> 231 and 144 -> 146.)
template <int BITS> struct ValueCodes {
    static constexpr int kMiddle = 1 << (BITS - 1);
    static __device__ __forceinline__ uint32_t power(uint32_t scale_zero) {  // 2^e as fp16
        const uint32_t e = scale_zero & 0x7c00u;
        return min(max(e, 0x0400u), 0x5c00u);  // 2^-14 .. 2^8: a code times that is a number of fp16
    }
    static __device__ __forceinline__ uint4 operands(uint2 codes, uint32_t scale_zero) {
        const uint32_t e = power(scale_zero);
        const half2_t factor = __builtin_bit_cast(half2_t, e | e << 16), middle = {(_Float16)(-1024.f - kMiddle), (_Float16)(-1024.f - kMiddle)};
        uint32_t lo = codes.x, hi = codes.y;  // channels 0..3 and 4..7, one byte each
        if constexpr (BITS == 4) {
            hi = (codes.x >> 4) & 0x0f0f0f0fu;
            lo = codes.x & 0x0f0f0f0fu;
        }
        auto pair = [&](uint32_t word, uint32_t select) {  // 0x6400 and a code are 1024 + code
            const half2_t c = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, word, select)) + middle;
            return __builtin_bit_cast(uint32_t, c * factor);
        };
        return make_uint4(pair(lo, 0x04010400u), pair(lo, 0x04030402u), pair(hi, 0x04010400u), pair(hi, 0x04030402u));
    }
};

// A block of 32 output rows, O^T in the lanes ((n, half) holds channels 32 db + 8 (i / 4) + 4 half + i % 4 of row n), out through 8 KiB of LDS so
// that sixteen lanes store a row.
template <class T>
__device__ __forceinline__ void store_rows(const TreeArgs& a, const float16_t (&acc)[4], float inv, unsigned char* room, const SeqShape& s, int hk, int row0) {
    const int lane = threadIdx.x % kWave, n = lane % 32, half = lane / 32, G = a.lp.group;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4) {
            uint2 w;
            w.x = Elem<T>::pack(acc[db][4 * g4] * inv, acc[db][4 * g4 + 1] * inv);
            w.y = Elem<T>::pack(acc[db][4 * g4 + 2] * inv, acc[db][4 * g4 + 3] * inv);
            *reinterpret_cast<uint2*>(room + n * kRowBytes + k_chunk_pos(n, db * 4 + g4) * 16 + 8 * half) = w;
        }
    asm volatile("" ::: "memory");  // LDS serves a wave in order, if the compiler asks in order
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + lane / 16, row = row0 + r;
        const uint4 w = *reinterpret_cast<const uint4*>(room + r * kRowBytes + k_chunk_pos(r, lane % 16) * 16);
        if (row < s.n * G)
            *reinterpret_cast<uint4*>(a.out + ((size_t)(s.start + row / G) * a.lp.H + hk * G + row % G) * kHeadDim + lane % 16 * 8) = w;
    }
}
__device__ __forceinline__ void store_lse(const TreeArgs& a, float m, float l, const SeqShape& s, int hk, int row0) {
    const int lane = threadIdx.x % kWave, row = row0 + lane % 32, G = a.lp.group;
    if (a.lse_out && lane < 32 && row < s.n * G)
        a.lse_out[(size_t)(s.start + row / G) * a.lp.H + hk * G + row % G] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

}  // namespace

// Wavefronts of a workgroup: RG row blocks, and with few of them two that share a step's keys.
constexpr int tree_waves(int RG) { return RG == 4 ? 4 : 2 * RG; }

template <class T, int BITS, int RG>
__global__ __launch_bounds__(tree_waves(RG) * kWave, (RG == 1 ? 1 : 2)) void draft_tree_kernel(TreeArgs a, TreeLaunch t) {
    constexpr bool QUANT = BITS != 16;
    constexpr int kWaves = tree_waves(RG), KG = kWaves / RG, NB = 2 / KG, R = 32 * RG;
    constexpr int kLoads = 16 / kWaves;  // 1 KiB loads per wave, operand and step
    __shared__ __attribute__((aligned(1024))) unsigned char k_lds[2][kTileBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char v_lds[2][kTileBytes];
    __shared__ __attribute__((aligned(16))) float k_scale[QUANT ? 2 : 1][2][QUANT ? kTile : 4];  // of the keys of a stage, times the softmax scale: scale, zero
    __shared__ __attribute__((aligned(16))) float v_scale[QUANT ? 2 : 1][2][QUANT ? kTile : 4];  // of the values: what is left of the scale, middle and zero
    __shared__ float2 fold_ml[RG][32];
    __shared__ unsigned spoiled_keys[2];
    __shared__ int spoiled[2];  // does a tile that some row does not see whole hold values that are not numbers?
    __shared__ int deepest[kWaves];  // tile of the wave's rows

    const int tid = threadIdx.x, lane = tid % kWave, n = lane % 32, half = lane / 32;
    const int wave = uniform(tid / kWave), rg = wave / KG, kg = wave % KG;
    SeqShape mine = {};
    if (t.target && lane < a.kv.batch) mine = seq_shape<R>(a, lane);
    const TreePlan plan = make_plan<R>(a, t, mine);
    // Workgroup ids go round-robin over the XCDs: row tiles of a piece, which read the same keys, go to one, and its L2 has them.
    constexpr int kXcds = 8;
    const int cycle = kXcds * t.row_tiles, place = blockIdx.x % cycle;
    const int unit = (int)blockIdx.x - place + place % kXcds * t.row_tiles + place / kXcds;
    TreeUnit u;
    SeqShape s = {};
    if (!find_unit<R>(a, t, plan, mine, unit, u, s)) return;
    // (all of it comes out of lane arithmetic, and what stays in vector registers takes the addresses of the walk there with it)
    u.b = uniform(u.b), u.hk = uniform(u.hk), u.row_tile = uniform(u.row_tile), u.piece = uniform(u.piece), u.pieces = uniform(u.pieces);
    s.start = uniform(s.start), s.n = uniform(s.n), s.len = uniform(s.len), s.pages = uniform(s.pages);
    s.then = uniform(s.then), s.dense = uniform(s.dense), s.stream = uniform(s.stream);
    const int b = u.b, hk = u.hk, G = a.lp.group, rows = s.n * G;
    const bool streaming = (a.lp.streaming_mask >> hk) & 1ull;
    if (u.piece == 0 && tid == 0 && t.target) t.pieces[(b * a.lp.Hkv + hk) * t.row_tiles + u.row_tile] = make_int2(unit, u.pieces);

    // ---- the list: entries of history, then tiles of drafted tokens
    const int drafts = ceil_div(s.n, kTile);
    const bool ring = in_stream_pool(a.lp, a.kv, hk);
    const int last_page = uniform((ring ? a.stream_pages : a.kv.num_pages) - 1);  // (one number of the walk: two and a choice there cost 6 % over 4-bit pages)
    const size_t head = (size_t)b * a.lp.Hkv + hk;
    // (the first `listed` entries are named by a list or a formula, the pages from first_new on follow; a list that holds fewer than it may
    // ends in entries of nothing, so that its length need not be waited for)
    const bool selects = a.sel_pages && !streaming;
    const int named = selects ? min(a.sel_count[head], a.sel_stride) : 0;
    int listed = streaming ? min(a.lp.sink_pages, s.pages) : selects ? min(s.then, a.sel_stride) : s.pages;
    const int first_new = streaming ? first_local_page(a.lp, s.len) : s.then;
    int entries, history, e0, e1;
    auto cut = [&](int all) __attribute__((always_inline)) {
        entries = all, history = all - drafts;
        const int share = all / u.pieces, rest = all - share * u.pieces;
        e0 = uniform(u.piece * share + min(u.piece, rest)), e1 = uniform(e0 + share + (u.piece < rest ? 1 : 0));
    };
    cut(streaming ? s.stream : s.dense);
    // Entry from + lane: (position of the page, physical page) or (drafted tile, -1); a position behind the last page: nothing of it is read.
    // Lane i of every wave has entry i of a stretch of 64: reading it costs no trip to memory, and no wave waits for another.
    auto look_up = [&](int from) __attribute__((always_inline)) {
        const int e = from + lane;
        int2 w = make_int2(s.pages, 0);
        if (e < e1 && e >= history) w = make_int2(e - history, -1);
        if (e < min(e1, history)) {
            int p = e < listed ? e : first_new + (e - listed);
            if (selects && e < listed) {
                p = a.sel_pages[head * a.sel_stride + e];
                if (e >= named) p = -1;
            }
            if (p >= 0 && p < s.pages) {
                const int phys = ring ? a.kv.ring_table[(size_t)b * a.kv.ring + ring_slot(a.lp, p)] : a.kv.page_table[(size_t)b * a.kv.max_pages + p];
                w = make_int2(p, min(max(phys, 0), last_page));
            }
        }
        return w;
    };

    // ---- the wave's rows: row r is query head r % G of the group, drafted token r / G; rows past the end repeat the last
    const int row0 = u.row_tile * R + rg * 32, row = min(row0 + n, rows - 1), own = row / G, token = s.start + own;  // own: index in its sequence
    const bool wave_has_rows = row0 < rows;
    // all that depends on the row alone is requested before anything is waited for
    uint4 qreg[8];
    {
        const uint4* src = reinterpret_cast<const uint4*>(a.q + ((size_t)token * a.lp.H + hk * G + row % G) * kHeadDim);
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) qreg[kk] = src[kk * 2 + half];
    }
    const unsigned long long row_mask = a.tree_mask ? a.tree_mask[(size_t)token * a.mask_words] : 0ull;  // of the first drafted tile
    int own_tile = 0, key_tile = 0;  // of the row's position; of the position of drafted key `lane`
    if (streaming) {
        const int key = min(lane, s.n - 1);
        own_tile = max(a.positions ? a.positions[token] : s.len + own, s.len);
        key_tile = max(a.positions ? a.positions[s.start + key] : s.len + key, s.len) / kTile;
        own_tile /= kTile;
    }
    int2 stretch = look_up(e0);
    // A list may also name more pages than there are or were: one of them twice, or in any order after tokens were taken back.  Its pieces are as many
    // as those of one that does not, and longer.
    if (__builtin_expect(uniform(named) > listed, 0)) {
        cut(entries + uniform(named) - listed);
        listed = uniform(named);
        stretch = look_up(e0);
    }
    // (pinned once the first keys are on their way: left alone the loads sink into the loop, where they wait for its prefetch)
    auto pin_queries = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) asm volatile("" : "+v"(qreg[kk].x), "+v"(qreg[kk].y), "+v"(qreg[kk].z), "+v"(qreg[kk].w));
    };
    float q_sum = 0.f;  // of the row, for quantised keys: code * scale + zero

    // ---- staging: wave w brings in rows w 64 / kWaves .., four rows to a load, lane l position l % 16 of row l / 16 of them
    const size_t slab = slab_chunks(kTile, BITS) * 16;
    const unsigned char* const k_base = reinterpret_cast<const unsigned char*>(ring ? a.kv.k_stream : a.kv.k_pool) + pool_rank(a.lp, a.kv, hk, ring) * slab;
    const unsigned char* const v_base = reinterpret_cast<const unsigned char*>(ring ? a.kv.v_stream : a.kv.v_pool) + pool_rank(a.lp, a.kv, hk, ring) * slab;
    const size_t page_bytes = (size_t)(ring ? a.kv.stream_heads : a.kv.pool_heads) * slab;
    const unsigned new_row_bytes = (unsigned)a.lp.Hkv * kRowBytes;
    const size_t new_offset = ((size_t)s.start * a.lp.Hkv + hk) * kRowBytes;
    const int my_row = wave * (kTile / kWaves) + lane / 16;
    constexpr int kFroms = kLoads < 4 ? kLoads : 4;
    unsigned k_from[kFroms];
#pragma unroll
    for (int i = 0; i < kFroms; ++i) k_from[i] = (unsigned)(my_row + 4 * i) * kRowBytes + k_chunk_pos(my_row + 4 * i, lane % 16) * 16;
    const unsigned v_from = (unsigned)my_row * kRowBytes + v_chunk_pos(my_row, lane % 16) * 16;
    // rows of an entry that exist
    auto live_rows = [&](int2 w) __attribute__((always_inline)) { return w.y < 0 ? min(s.n - w.x * kTile, kTile) : min(s.len - w.x * kTile, kTile); };
    auto fetch = [&](int2 w, unsigned char* kd, unsigned char* vd) __attribute__((always_inline)) {  // 16-bit rows; those past the last one repeat it
        const int live = max(live_rows(w), 1);  // (nothing of an entry without a page is used, but the loads are counted)
        const bool drafted = w.y < 0;
        const unsigned long long offset = drafted ? new_offset + (size_t)w.x * kTile * new_row_bytes : (size_t)w.y * page_bytes;
        const unsigned long long ks = uniform64((unsigned long long)(drafted ? (const unsigned char*)a.k_new : k_base) + offset);
        const unsigned long long vs = uniform64((unsigned long long)(drafted ? (const unsigned char*)a.v_new : v_base) + offset);
        const unsigned kd_at = uniform(lds_address(kd) + wave * kLoads * 1024), vd_at = uniform(lds_address(vd) + wave * kLoads * 1024);
        if (!drafted && live == kTile) {
            // sixteen rows on the permutation of K repeats itself, four rows on that of V
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                dma_load16(ks + (unsigned)(i / 4) * (16 * kRowBytes), k_from[i % kFroms], kd_at + i * 1024);
                dma_load16(vs + (unsigned)i * (4 * kRowBytes), v_from, vd_at + i * 1024);
            }
            return;
        }
        const unsigned stride = drafted ? new_row_bytes : (unsigned)kRowBytes;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = my_row + 4 * i;
            const unsigned at = (unsigned)min(r, live - 1) * stride;
            dma_load16(ks, at + k_chunk_pos(r, lane % 16) * 16, kd_at + i * 1024);
            dma_load16(vs, at + v_chunk_pos(r, lane % 16) * 16, vd_at + i * 1024);
        }
    };
    // Quantised rows on their way through registers: per load the codes of this lane's 16-byte place (8 channels) and the (scale, zero) of its
    // V row; of the K rows one wave has all, a lane each.
    constexpr int kCodeBytes = kHeadDim * BITS / 8;  // of a row
    using Codes = typename std::conditional<BITS == 8, uint2, uint32_t>::type;
    struct Staged {
        Codes k[kLoads], v[kLoads];
        uint32_t vz[kLoads], kz, vz_all;
        bool on;
    } staged;
    staged.on = false;
    unsigned k_code[QUANT ? kFroms : 1], v_code = 0;  // from the page to the places of a full one (see k_from)
    if constexpr (QUANT) {
#pragma unroll
        for (int i = 0; i < kFroms; ++i) k_code[i] = (unsigned)(my_row + 4 * i) * kCodeBytes + k_chunk_pos(my_row + 4 * i, lane % 16) * BITS;
        v_code = (unsigned)my_row * kCodeBytes + v_chunk_pos(my_row, lane % 16) * BITS;
    }
    auto fetch_codes = [&](int2 w) __attribute__((always_inline)) {
        if constexpr (QUANT) {
            const int live = live_rows(w);
            staged.on = w.y >= 0 && live > 0;
            if (!staged.on) return;
            const unsigned long long page = (unsigned long long)w.y * page_bytes;
            const unsigned char* const kp = reinterpret_cast<const unsigned char*>(uniform64((unsigned long long)k_base + page));
            const unsigned char* const vp = reinterpret_cast<const unsigned char*>(uniform64((unsigned long long)v_base + page));
            if (live == kTile) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    staged.k[i] = *reinterpret_cast<const Codes*>(kp + (k_code[i % kFroms] + i / 4 * 16 * kCodeBytes));
                    staged.v[i] = *reinterpret_cast<const Codes*>(vp + (v_code + i * 4 * kCodeBytes));
                    staged.vz[i] = *reinterpret_cast<const uint32_t*>(vp + (kTile * kCodeBytes + (unsigned)my_row * 4 + i * 16));
                }
            } else {  // rows past the last one repeat it
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int r = my_row + 4 * i;
                    const unsigned from = (unsigned)min(r, live - 1);
                    staged.k[i] = *reinterpret_cast<const Codes*>(kp + (from * kCodeBytes + k_chunk_pos(r, lane % 16) * BITS));
                    staged.v[i] = *reinterpret_cast<const Codes*>(vp + (from * kCodeBytes + v_chunk_pos(r, lane % 16) * BITS));
                    staged.vz[i] = *reinterpret_cast<const uint32_t*>(vp + (kTile * kCodeBytes + from * 4));
                }
            }
            if (wave == 0) staged.kz = *reinterpret_cast<const uint32_t*>(kp + (kTile * kCodeBytes + (unsigned)min(lane, live - 1) * 4));
            if (wave == 1) staged.vz_all = *reinterpret_cast<const uint32_t*>(vp + (kTile * kCodeBytes + (unsigned)min(lane, live - 1) * 4));
        }
    };
    // Keys go into LDS as their codes, exactly, and meet scale and zero as scores in fp32 (rounded keys would cost the log-sum-exp three
    // digits).  Values: see ValueCodes.
    auto store_staged = [&](int stage) __attribute__((always_inline)) {
        if constexpr (QUANT) {
            if (!staged.on) return;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const unsigned to = (wave * kLoads + i) * 1024 + lane * 16;
                *reinterpret_cast<uint4*>(k_lds[stage] + to) = codes8<T, BITS>(two_words(staged.k[i]));
                *reinterpret_cast<uint4*>(v_lds[stage] + to) = ValueCodes<BITS>::operands(two_words(staged.v[i]), staged.vz[i]);
            }
            if (wave == 0) {
                const float scale = Elem<F16>::lo(staged.kz), zero = Elem<F16>::hi(staged.kz);
                k_scale[stage][0][lane] = scale / KeyCodes<T, BITS>::unit * a.lp.sm_scale_log2;
                k_scale[stage][1][lane] = (zero - KeyCodes<T, BITS>::offset * scale) * a.lp.sm_scale_log2;
            }
            if (wave == 1) {
                const float scale = Elem<F16>::lo(staged.vz_all), zero = Elem<F16>::hi(staged.vz_all);
                v_scale[stage][0][lane] = scale / Elem<F16>::lo(ValueCodes<BITS>::power(staged.vz_all));
                v_scale[stage][1][lane] = zero + scale * ValueCodes<BITS>::kMiddle;
            }
        }
    };

    int deepest_tile = 0;  // of the workgroup's rows

    // ---- softmax state and outputs of the lane's row (its keys: those of its half)
    float16_t acc[4] = {};
    float m_run = -INFINITY, l_run = 0.f, o_run = 0.f;  // (o_run: what all channels get, see ValueCodes)
    // Chunk kk of a key's row is at k_place ^ 32 kk and channels 32 db and on of a value's at v_place ^ 64 db.
    const int k_place = (kg * NB * 32 + n) * kRowBytes + k_chunk_pos(n, half) * 16;
    const int v_place = kg * NB * 32 * kRowBytes + half * 1024 + lane % 16 / 4 * kRowBytes + v_chunk_pos(lane % 16 / 4, 2 * (n / 16) + lane % 4 / 2) * 16 + 8 * (lane % 2);

    // keys of the entry that the lane's row sees, one bit each
    auto seen = [&](int2 w, int live) __attribute__((always_inline)) {
        unsigned long long bits = live >= kTile ? ~0ull : (1ull << live) - 1ull;
        if (w.y >= 0) {
            if (streaming && !(w.x < a.lp.sink_pages || w.x > own_tile - a.lp.local_pages)) bits = 0;
            return bits;
        }
        if (a.tree_mask) {
            bits &= w.x == 0 ? row_mask : a.tree_mask[(size_t)token * a.mask_words + w.x];
        } else {
            const int last = own - w.x * kTile;  // a chain: its own and those before
            bits &= last < 0 ? 0ull : last >= kTile - 1 ? ~0ull : (2ull << last) - 1ull;
        }
        if (streaming && deepest_tile >= a.lp.local_pages) {
            // a drafted key counts as a token of the tile of its position
            int tile = key_tile;
            if (w.x > 0) {
                const int key = w.x * kTile + min(lane, live - 1);
                tile = max(a.positions ? a.positions[s.start + key] : s.len + key, s.len) / kTile;
            }
            // (off for some row, if at all: the deepest is the first to lose a key)
            unsigned long long far = __ballot(lane < live && tile >= a.lp.sink_pages && tile <= deepest_tile - a.lp.local_pages);
            for (; far; far &= far - 1) {
                const int i = __builtin_ctzll(far);
                if (__builtin_amdgcn_readlane(tile, i) <= own_tile - a.lp.local_pages) bits &= ~(1ull << i);
            }
        }
        return bits;
    };

    // A value that is infinite or not a number must not reach the rows that do not see its key, and zero times it would.  Tiles that some row
    // does not see whole (drafted tokens, the last page, pages at the far end of a streaming head's window) are looked through, by each wave
    // what it has brought in itself, ahead of the barrier in front of their step.  Nearly always there is nothing; otherwise such values become
    // zeros, and are added to the rows that do see their keys one by one.
    auto ragged = [&](int2 w) __attribute__((always_inline)) {
        const int live = live_rows(w);
        return live > 0 && (live < kTile || w.y < 0 || (streaming && w.x >= a.lp.sink_pages && w.x <= deepest_tile - a.lp.local_pages));
    };
    // (Codes are numbers, and scales and zeros that are not are kept from weights of zero: this is for rows of 16 bits.)
    auto look_for_spoiled = [&](int2 w, int stage) __attribute__((always_inline)) {
        if (!ragged(w)) return;
        const uint4* const brought = reinterpret_cast<const uint4*>(v_lds[stage] + wave * kLoads * 1024) + lane;
        ushort2_t most = {0, 0};  // magnitude, as whole numbers
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint4 x = brought[i * kWave];
            const uint32_t x4[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) most = __builtin_elementwise_max(most, __builtin_bit_cast(ushort2_t, x4[c] & 0x7fff7fffu));
        }
        constexpr uint32_t exponents = BitsOf<T>::exponent;
        if (__any(most[0] >= exponents || most[1] >= exponents)) spoiled[stage] = 1;
    };
    // (together; the bits of the keys that have such values)
    auto clear_spoiled = [&](int stage) __attribute__((always_inline)) -> unsigned long long {
        constexpr uint32_t low = BitsOf<T>::exponent, high = low << 16;
        constexpr int kPieces = kTileBytes / 16 / (kWaves * kWave);
        uint4* const mine = reinterpret_cast<uint4*>(v_lds[stage]) + tid;
        __syncthreads();
        if (tid == 0) spoiled[stage] = 0;
        if (tid < 2) spoiled_keys[tid] = 0;
        __syncthreads();
#pragma clang loop unroll(disable)
        for (int i = 0; i < kPieces; ++i) {
            const int at = i * kWaves * kWave;
            const uint4 x = mine[at];
            uint32_t x4[4] = {x.x, x.y, x.z, x.w};
            bool here = false;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if ((x4[c] & low) == low) x4[c] &= 0xffff0000u, here = true;
                if ((x4[c] & high) == high) x4[c] &= 0x0000ffffu, here = true;
            }
            if (here) {
                const int key = (tid + at) / 16;
                mine[at] = make_uint4(x4[0], x4[1], x4[2], x4[3]);
                atomicOr(&spoiled_keys[key / 32], 1u << (key % 32));
            }
        }
        __syncthreads();
        return (unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane(spoiled_keys[1]) << 32 |
               (unsigned)__builtin_amdgcn_readfirstlane(spoiled_keys[0]);
    };
    // Those values, from where they came from, to the rows that do see their keys: weight times value in fp32.
    auto add_spoiled = [&](int2 w, int stage, unsigned long long bits, float off, unsigned long long keys) __attribute__((always_inline)) {
        const bool drafted = w.y < 0;
        for (keys &= (NB == 2 ? ~0ull : 0xffffffffull << (32 * kg)); keys; keys &= keys - 1) {
            const int key = __builtin_ctzll(keys), from = min(key, live_rows(w) - 1);
            float score = 0.f;
#pragma unroll
            for (int kk = 0; kk < 8; ++kk) {
                const uint4 x = *reinterpret_cast<const uint4*>(k_lds[stage] + key * kRowBytes + k_chunk_pos(key, kk * 2 + half) * 16);
                score = Elem<T>::dot2(x.x, qreg[kk].x, Elem<T>::dot2(x.y, qreg[kk].y, score));
                score = Elem<T>::dot2(x.z, qreg[kk].z, Elem<T>::dot2(x.w, qreg[kk].w, score));
                __builtin_amdgcn_sched_barrier(0);
            }
            score = halves_sum(score);
            const bool on = bits >> key & 1ull;
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(score, a.lp.sm_scale_log2, off));
            const unsigned char* const src = drafted ? (const unsigned char*)a.v_new + new_offset + ((size_t)w.x * kTile + from) * new_row_bytes
                                                     : v_base + (size_t)w.y * page_bytes + from * kRowBytes;
#pragma unroll
            for (int db = 0; db < 4; ++db)
#pragma unroll
                for (int g4 = 0; g4 < 4; ++g4) {
                    const int c = 4 * db + g4;  // eight channels, of which the lane has four
                    const uint2 x = *reinterpret_cast<const uint2*>(src + c * 16 + 8 * half);
                    const float v4[4] = {Elem<T>::lo(x.x), Elem<T>::hi(x.x), Elem<T>::lo(x.y), Elem<T>::hi(x.y)};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (on && !(fabsf(v4[i]) < INFINITY)) acc[db][4 * g4 + i] += p * v4[i];
                    __builtin_amdgcn_sched_barrier(0);
                }
        }
    };

    // (kind: std::true_type for a quantised page)
    auto work_on = [&](auto kind, int2 w, int stage, bool part, unsigned long long keys) __attribute__((always_inline)) {
        constexpr bool codes = decltype(kind)::value;
        const int live = live_rows(w);
        if (live <= 0 || !wave_has_rows) return;
        unsigned long long bits = ~0ull;
        if (part) {
            bits = seen(w, live);
            if (!__any(bits != 0)) return;
        }
        const unsigned char *ks = k_lds[stage], *vs = v_lds[stage];
        int k_at = k_place;
        // Where registers are short the eight places of a step are worked out in the step (64 x 16k tokens of 8 bits, 30 drafted: 191 us with the places
        // kept and 35 other registers in scratch, 186 us with 28; of 4 bits under 32 rows each the same).
        if constexpr (QUANT && RG == 4) asm volatile("" : "+v"(k_at));
        // (one block of keys: two chains of products, which do not wait for each other, instead of one)
        constexpr int kChains = 2 / NB;
        float16_t sc[NB], chain[NB * kChains] = {};
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
                float16_t& sum = chain[kb * kChains + kk % kChains];
                sum = Mfma<T>::run(*reinterpret_cast<const uint4*>(ks + kb * 32 * kRowBytes + (k_at ^ 32 * kk)), qreg[kk], sum);
            }
        // schedule: operand reads run four ahead of the products that consume them, and no further (registers)
        __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
        for (int i = 0; i < 8 * NB - kAhead; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
            sc[kb] = chain[kb * kChains];
            if constexpr (kChains == 2) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[kb][i] += chain[kb * kChains + 1][i];
            }
        }
        // Exponents, relative to the row's reference (0 before it has one).  The reference is not the maximum so far but one that follows it at
        // a distance of up to kSlack: weights up to 2^kSlack do no harm in any of the types, and outputs are rescaled a few times a list
        // instead of in most steps.
        const bool unset = m_run == -INFINITY;
        float off = unset ? 0.f : -m_run;
        if constexpr (codes) {
#pragma unroll
            for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                for (int g4 = 0; g4 < 4; ++g4) {
                    const int key = (kg * NB + kb) * 32 + 8 * g4 + 4 * half;
                    const float4 z = *reinterpret_cast<const float4*>(&k_scale[stage][0][key]), o = *reinterpret_cast<const float4*>(&k_scale[stage][1][key]);
                    const float z4[4] = {z.x, z.y, z.z, z.w}, o4[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[kb][4 * g4 + i] = __builtin_fmaf(sc[kb][4 * g4 + i], z4[i], __builtin_fmaf(o4[i], q_sum, off));
                }
        } else {
#pragma unroll
            for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[kb][i] = __builtin_fmaf(sc[kb][i], a.lp.sm_scale_log2, off);
        }
        if (part) {
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
                const unsigned mine = (unsigned)(bits >> (32 * (kg * NB + kb))) >> (4 * half);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!(mine >> (8 * (i / 4) + i % 4) & 1u)) sc[kb][i] = -INFINITY;
            }
        }
        float top = sc[0][0];
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[kb][i]);
        top = halves_max(top);
        const bool moves = unset ? top > -INFINITY : top > kSlack;
        if (__builtin_expect(__any(moves), 0)) {
            const float delta = moves ? top : 0.f, alpha = unset ? 0.f : __builtin_amdgcn_exp2f(-delta);
            l_run *= alpha;
            if constexpr (QUANT) o_run *= alpha;
#pragma unroll
            for (int db = 0; db < 4; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[db][i] *= alpha;
#pragma unroll
            for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[kb][i] -= delta;
            if (moves) m_run = unset ? delta : m_run + delta;
            off = m_run == -INFINITY ? 0.f : -m_run;
        }
        using V = typename std::conditional<codes, F16, T>::type;  // of the values in LDS
        uint4 pb[NB][2];
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
            float p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[i] = __builtin_amdgcn_exp2f(sc[kb][i]);
                // unrounded; the second product takes them in the layer's type, which is what its operands are (a decode step, whose second product is
                // not the matrix cores', keeps fp32 there: errors against 64 bits 2.8e-4 here, 2.1e-4 with fp32 weights; bf16 2.3e-3 and 1.7e-3)
                sum[i % 2] += p[i];
            }
            if constexpr (codes) {
#pragma unroll
                for (int g4 = 0; g4 < 4; ++g4) {
                    const int key = (kg * NB + kb) * 32 + 8 * g4 + 4 * half;
                    const float4 z = *reinterpret_cast<const float4*>(&v_scale[stage][0][key]), o = *reinterpret_cast<const float4*>(&v_scale[stage][1][key]);
                    float z4[4] = {z.x, z.y, z.z, z.w}, o4[4] = {o.x, o.y, o.z, o.w};
                    if (__builtin_expect(part, 0)) {  // a key that is not seen may have a scale or zero that is not a number
                        asm volatile("");
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            z4[i] = p[4 * g4 + i] == 0.f ? 0.f : z4[i];
                            o4[i] = p[4 * g4 + i] == 0.f ? 0.f : o4[i];
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        o_run = __builtin_fmaf(p[4 * g4 + i], o4[i], o_run);
                        p[4 * g4 + i] *= z4[i];
                    }
                }
            }
            pb[kb][0] = pack8<V>(p);
            pb[kb][1] = pack8<V>(p + 8);
        }
        l_run += sum[0] + sum[1];
        auto values = [&](int step, int db) __attribute__((always_inline)) {  // V^T operand: channel 32 db + n of the lane's eight keys of the step's sixteen
            const uint2 lo = lds_read_transposed(vs + (4 * step) * 1024 + (v_place ^ 64 * db));
            const uint2 hi = lds_read_transposed(vs + (4 * step + 2) * 1024 + (v_place ^ 64 * db));
            return make_uint4(lo.x, lo.y, hi.x, hi.y);
        };
#pragma unroll
        for (int step = 0; step < 2 * NB; ++step)
#pragma unroll
            for (int db = 0; db < 4; ++db) acc[db] = Mfma<V>::run(values(step, db), pb[step / 2][step % 2], acc[db]);
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * kAhead, 0);
#pragma unroll
        for (int i = 0; i < 8 * NB - kAhead; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
        if constexpr (!codes) {
            if (__builtin_expect(keys != 0, 0)) add_spoiled(w, stage, bits, off, keys);
        }
    };

    // ---- walk
    if (tid < 2) spoiled[tid] = 0;
    {
        const int tile = wave_scan(own_tile, 0, larger);  // (as whole numbers: tiles go up to 2^25)
        if (lane == kWave - 1) deepest[wave] = tile;
    }
    if constexpr (QUANT) {
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
            const uint32_t w[4] = {qreg[kk].x, qreg[kk].y, qreg[kk].z, qreg[kk].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) q_sum += Elem<T>::lo(w[i]) + Elem<T>::hi(w[i]);
        }
        q_sum = halves_sum(q_sum);
    }

    auto step = [&](auto kind, int2 w, int stage) __attribute__((always_inline)) {
        const bool part = ragged(w);
        unsigned long long keys = 0;
        if (!decltype(kind)::value && part && __builtin_expect(uniform(spoiled[stage]) != 0, 0)) keys = clear_spoiled(stage);
        work_on(kind, w, stage, part, keys);
    };
    auto find_deepest = [&]() __attribute__((always_inline)) {  // past a barrier
#pragma unroll
        for (int i = 0; i < kWaves; ++i) deepest_tile = max(deepest_tile, deepest[i]);
        deepest_tile = uniform(deepest_tile);
    };
    const int2 nothing = make_int2(s.pages, 0);
    // entry e of the list; asked for in order
    auto next_entry = [&](int e) __attribute__((always_inline)) {
        if (e >= e1) return nothing;
        const int i = (e - e0) % kWave;
        if (i == 0 && e > e0) stretch = look_up(e);
        return make_int2(__builtin_amdgcn_readlane(stretch.x, i), __builtin_amdgcn_readlane(stretch.y, i));
    };
    // Entry e is worked on, e + 1 on its way into LDS and, of quantised pages, e + 2 on its way into registers.  The entries of quantised pages come
    // first, and then, as all entries of 16-bit caches do, drafted tokens.
    const int coded = QUANT ? max(e0, min(history, e1)) : e0;  // the first entry of 16-bit rows
    int2 w0 = next_entry(e0), w1 = nothing, w2 = nothing;
    if constexpr (QUANT) w1 = next_entry(e0 + 1);
    if (e0 < coded) {
        fetch_codes(w0);
        store_staged(0);
        if (e0 + 1 < coded) fetch_codes(w1);
    } else if (e0 < e1) {
        fetch(w0, k_lds[0], v_lds[0]);
    }
    __syncthreads();
    find_deepest();
    pin_queries();
    if constexpr (QUANT) {
        auto turn = [&](int e, int stage) __attribute__((always_inline)) {
            w2 = next_entry(e + 2);
            if (e + 1 < coded)
                store_staged(stage ^ 1);
            else if (e + 1 < e1)
                fetch(w1, k_lds[stage ^ 1], v_lds[stage ^ 1]);
            if (e + 2 < coded) fetch_codes(w2);
            step(std::true_type{}, w0, stage);
            w0 = w1;
            w1 = w2;
            __syncthreads();
        };
        for (int e = e0; e < coded; e += 2) {
            turn(e, 0);
            if (e + 1 < coded) turn(e + 1, 1);
        }
    }
    {
        auto turn = [&](int e, int stage) __attribute__((always_inline)) {
            dma_wait();
            look_for_spoiled(w0, stage);
            __syncthreads();  // the tiles of this step are there, and those of the step before are done with
            if constexpr (!QUANT) w1 = next_entry(e + 1);
            if (e + 1 < e1) fetch(w1, k_lds[stage ^ 1], v_lds[stage ^ 1]);
            step(std::false_type{}, w0, stage);
            w0 = w1;
            if constexpr (QUANT) w1 = next_entry(e + 2);
        };
        if constexpr (QUANT) {  // one or two steps
#pragma clang loop unroll(disable)
            for (int e = coded; e < e1; ++e) turn(e, (e - e0) & 1);
        } else {
            for (int e = coded; e < e1; e += 2) {
                turn(e, 0);
                if (e + 1 < e1) turn(e + 1, 1);
            }
        }
        __syncthreads();
    }

    // ---- the two halves of the keys meet in LDS (the tiles are done with: the loop ended on a barrier)
    float l = halves_sum(l_run), m = m_run;
    if constexpr (QUANT) {
        const float o = halves_sum(o_run);
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[db][i] += o;
    }
    if constexpr (KG == 2) {
        float4* const room = reinterpret_cast<float4*>(k_lds[rg]);
        if (kg == 1) {
#pragma unroll
            for (int db = 0; db < 4; ++db)
#pragma unroll
                for (int g4 = 0; g4 < 4; ++g4)
                    room[(db * 4 + g4) * kWave + lane] = make_float4(acc[db][4 * g4], acc[db][4 * g4 + 1], acc[db][4 * g4 + 2], acc[db][4 * g4 + 3]);
            if (half == 0) fold_ml[rg][n] = make_float2(m, l);
        }
        __syncthreads();
        if (kg == 1) return;
        const float2 other = fold_ml[rg][n];
        const float m_all = fmaxf(m, other.x);
        const float f0 = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_all), f1 = other.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(other.x - m_all);
        l = l * f0 + other.y * f1;
        m = m_all;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4) {
                const float4 x = room[(db * 4 + g4) * kWave + lane];
                acc[db][4 * g4] = acc[db][4 * g4] * f0 + x.x * f1;
                acc[db][4 * g4 + 1] = acc[db][4 * g4 + 1] * f0 + x.y * f1;
                acc[db][4 * g4 + 2] = acc[db][4 * g4 + 2] * f0 + x.z * f1;
                acc[db][4 * g4 + 3] = acc[db][4 * g4 + 3] * f0 + x.w * f1;
            }
    }
    if (!wave_has_rows) return;
    if (u.pieces > 1) {  // as the lanes hold it
        const size_t block = (size_t)unit * RG + rg;
        float4* const dst = t.partials + block * kBlockFloat4;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4)
                dst[(db * 4 + g4) * kWave + lane] = make_float4(acc[db][4 * g4], acc[db][4 * g4 + 1], acc[db][4 * g4 + 2], acc[db][4 * g4 + 3]);
        if (half == 0) t.partial_ml[block * 32 + n] = make_float2(m, l);
        return;
    }
    unsigned char* const room = v_lds[rg / 2] + rg % 2 * (kTileBytes / 2);  // 8 KiB for the wave's rows
    store_rows<T>(a, acc, l == 0.f ? 0.f : 1.f / l, room, s, hk, row0);
    store_lse(a, m, l, s, hk, row0);
}

// Puts the pieces of 32 rows of a (sequence, KV head) together: a workgroup to 32 channels, its eight wavefronts take pieces in turn, and what they
// have is added in their order.  Pieces come in at the latency of memory, so that many wavefronts with a few loads each are wanted: 4 to 7 us, 4 of
// them where there is nothing to do.  2048 workgroups; with 512 a launch of whole lists is over 1 to 2 us sooner (138 -> 136, 218 -> 213 us of both
// kernels), one of pieces later (16 x 32k with 64 drafted 78 -> 85, 40 x 100 .. 3000 36 -> 41).
constexpr int kFoldWaves = 8, kFoldThreads = kFoldWaves * kWave, kFoldLanes = kWave * 17;  // a lane's sixteen sums, one place apart from the next lane's
template <class T, int RG>
__device__ __forceinline__ void fold_item(const TreeArgs& a, const TreeLaunch& t, int at, float (&sums)[kFoldWaves][kFoldLanes], float2 (&wave_ml)[kFoldWaves][32]) {
    const int tid = threadIdx.x, lane = tid % kWave, n = lane % 32, G = a.lp.group, wave = uniform(tid / kWave);
    const int db = at % 4;
    at /= 4;
    const int rg = at % RG;
    at /= RG;
    const int row_tile = at % t.row_tiles, list = at / t.row_tiles, hk = list % a.lp.Hkv, b = list / a.lp.Hkv;
    const int2 pieces = t.pieces[at];
    const SeqShape s = seq_shape<32 * RG>(a, b);
    const int row0 = (row_tile * RG + rg) * 32;
    if (row0 >= s.n * G) return;  // (what stands in `pieces` of a row tile that does not exist is of another launch)
    // (lengths that contradict each other may ask for more pieces than there is room for, and lead to no address outside it)
    if (pieces.x < 0 || pieces.y < 2 || pieces.x + (long long)(pieces.y - 1) * s.row_tiles >= t.slots) return;
    // piece i of a row tile is row_tiles (of this sequence) slots behind piece i - 1
    const size_t apart = (size_t)s.row_tiles * RG, first = (size_t)pieces.x * RG + rg;
    float m = -INFINITY, l = 0.f, o[16] = {};
    for (int i = wave; i < pieces.y; i += 4 * kFoldWaves) {  // four pieces at a time
        float2 ml[4];
        float4 x[4][4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const size_t slot = first + min(i + k * kFoldWaves, pieces.y - 1) * apart;
            ml[k] = t.partial_ml[slot * 32 + n];
            const float4* src = t.partials + slot * kBlockFloat4 + db * 4 * kWave + lane;
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4) x[k][g4] = src[g4 * kWave];
        }
        float top = m;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (i + k * kFoldWaves >= pieces.y) ml[k] = make_float2(-INFINITY, 0.f);
            top = fmaxf(top, ml[k].x);
        }
        const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        l *= alpha;
#pragma unroll
        for (int c = 0; c < 16; ++c) o[c] *= alpha;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (i + k * kFoldWaves >= pieces.y) break;
            const float f = ml[k].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[k].x - top);
            l += ml[k].y * f;
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4) {
                o[4 * g4] += x[k][g4].x * f;
                o[4 * g4 + 1] += x[k][g4].y * f;
                o[4 * g4 + 2] += x[k][g4].z * f;
                o[4 * g4 + 3] += x[k][g4].w * f;
            }
        }
        m = top;
    }
#pragma unroll
    for (int c = 0; c < 16; ++c) sums[wave][lane * 17 + c] = o[c];
    if (lane < 32) wave_ml[wave][n] = make_float2(m, l);
    __syncthreads();
    // thread: row tid / 16, channels 2 (tid % 16) and the next of the 32; lane (row, half) has channel 8 g4 + 4 half + i in place 4 g4 + i
    const int r = tid / 16, c = 2 * (tid % 16), from = (r + 32 * (c / 4 % 2)) * 17 + c / 8 * 4 + c % 4, row = row0 + r;
    float top = -INFINITY, sum = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
    for (int w = 0; w < kFoldWaves; ++w) top = fmaxf(top, wave_ml[w][r].x);
#pragma unroll
    for (int w = 0; w < kFoldWaves; ++w) {
        const float2 ml = wave_ml[w][r];
        const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
        sum += ml.y * f;
        o0 += sums[w][from] * f;
        o1 += sums[w][from + 1] * f;
    }
    if (row >= s.n * G) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const size_t head = (size_t)(s.start + row / G) * a.lp.H + hk * G + row % G;
    *reinterpret_cast<uint32_t*>(a.out + head * kHeadDim + db * 32 + c) = Elem<T>::pack(o0 * inv, o1 * inv);
    if (a.lse_out && db == 0 && c == 0) a.lse_out[head] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <class T, int RG>
__global__ __launch_bounds__(kFoldThreads) void fold_trees_kernel(TreeArgs a, TreeLaunch t) {
    __shared__ float sums[kFoldWaves][kFoldLanes];
    __shared__ float2 wave_ml[kFoldWaves][32];
    const int lane = threadIdx.x % kWave;
    // Lists that are whole leave most of the work of some launches empty: a workgroup looks at up to 64 of its items at once.
    const int own = blockIdx.x + lane * (int)gridDim.x;
    bool mine = false;
    if (own < t.folds) mine = t.pieces[own / (4 * RG)].y >= 2;
    for (unsigned long long todo = __ballot(mine); todo; todo &= todo - 1) {
        const int item = blockIdx.x + __builtin_ctzll(todo) * gridDim.x;
        fold_item<T, RG>(a, t, item, sums, wave_ml);
        __syncthreads();
    }
}
// ---- host side -----------------------------------------------------------------------------------

namespace {

struct TreeSizes {
    int RG, row_tiles, target, exact, streams;
    long long grid, folds;  // workgroups of the two kernels
    size_t pieces_bytes, ml_bytes, partial_bytes;
};

TreeSizes tree_sizes(const LayerParams& lp, int batch, int total_new, int max_new, int max_pages, int sel_stride, bool quantised) {
    TreeSizes z = {};
    // As few rows as the longest tree has (two and three times as many as it takes: 40 sequences of 100 .. 3000 tokens 36 -> 50 us with RG = 1 for 64
    // rows, 36 -> 41 with RG = 4).  Quantised pages take four wavefronts to unpack, whoever has rows: 16 x 12k tokens of 8 bits under 32 rows 82 -> 76 us
    // with RG = 2, 4 x 100k of 4 bits 134 -> 125, 64 x 500 .. 4000 of 8 bits 83 -> 76; 8 x 30k, of which 4096 selected, of 4 bits 27 -> 28.
    const long long rows = (long long)max_new * lp.group;
    z.RG = rows <= 32 && !quantised ? 1 : rows <= 64 ? 2 : 4;
    const int R = 32 * z.RG;
    z.row_tiles = (int)((rows + R - 1) / R);
    z.streams = __builtin_popcountll(lp.streaming_mask);
    // row tiles of all sequences: a part of one each, and no more than the tokens there are
    const long long tiles = std::min((long long)batch * z.row_tiles, (long long)total_new * lp.group / R + batch), lists = tiles * lp.Hkv;
    const int resident = 2 * num_compute_units();  // workgroups that run at once: 64 KiB of LDS each
    // list entries as far as the host knows: pages of the table, or of a selection (and those since, which are few)
    const int drafts = ceil_div(max_new, kTile), dense = sel_stride > 0 ? std::min(max_pages, sel_stride + 1) : max_pages;
    const int stream = std::min(max_pages, lp.sink_pages + lp.local_pages);
    const long long shortest = tiles * ((lp.Hkv - z.streams) * (long long)(dense + drafts) + z.streams * (long long)(stream + drafts)) / kLeastPiece;
    // So many lists that all stay whole: to find its piece a workgroup runs over the batch, 64 sequences at a time.  Whole and cut, trees of 4 on 8 KV heads: 600
    // x 100 .. 2000 tokens 428 and 429 us, 600 x 2000 716 and 629, 1200 x 50 .. 700 400 and 647, 4000 x 50 .. 300 800 and 3800; below the border 300 x 2000 361 and
    // 322, 150 x 2000 207 and 165.  What whole lists cost is a sequence far longer than the others, which a workgroup to a head walks alone: one of 100000
    // among 600 of 100 .. 2000 1930 and 447.
    z.target = lists >= 8LL * resident || std::max(dense, stream) + drafts <= kLeastPiece ? 0 : (int)std::min<long long>(shortest, resident);
    // Few lists are cut until the pieces all run at once, more are not searched for that (see make_plan).  Searched and not: 16 x 2000 .. 40000 tokens under 8
    // heads 149 and 153 us, 32 x 2000 .. 40000 239 and 239, 16 x 4096 selected 47.6 and 46.2; past the border 64 x 2000 .. 20000, as many lists as
    // pieces, 434 and 291, 9 x 1000 .. 20000 under 32 heads 128 and 122.  One KV head and 200 sequences, loaded anew in every round of the search, 231 and 225.
    z.exact = z.target > 0 && 2 * lists <= z.target;
    z.grid = z.target == 0 ? (long long)batch * lp.Hkv * z.row_tiles : z.target + lists;
    const long long cycle = 8LL * z.row_tiles;  // see the kernel
    z.grid = (z.grid + cycle - 1) / cycle * cycle;
    z.folds = z.target == 0 ? 0 : (long long)batch * lp.Hkv * z.row_tiles * z.RG * 4;
    if (z.target) {
        z.pieces_bytes = ((size_t)batch * lp.Hkv * z.row_tiles * sizeof(int2) + 255) / 256 * 256;
        z.ml_bytes = (size_t)z.grid * z.RG * 32 * sizeof(float2);
        z.partial_bytes = (size_t)z.grid * z.RG * kBlockFloat4 * sizeof(float4);
    }
    return z;
}

template <class T, int BITS> hipError_t launch_tree(const TreeArgs& a, void* workspace, hipStream_t stream) {
    const TreeSizes z = tree_sizes(a.lp, a.kv.batch, a.total_new, a.max_new, a.kv.max_pages, a.sel_stride, BITS != 16);
    if (z.grid > 0x7fffffffLL || z.folds > 0x7fffffffLL) return hipErrorInvalidValue;
    TreeLaunch t = {};
    t.target = z.target;
    t.exact = z.exact;
    t.row_tiles = z.row_tiles;
    t.streams = z.streams;
    t.slots = z.target ? (int)z.grid : 0;
    t.folds = (int)z.folds;
    if (z.target) {
        unsigned char* p = static_cast<unsigned char*>(workspace);
        t.pieces = reinterpret_cast<int2*>(p);
        t.partial_ml = reinterpret_cast<float2*>(p + z.pieces_bytes);
        t.partials = reinterpret_cast<float4*>(p + z.pieces_bytes + z.ml_bytes);
    }
    const dim3 grid((unsigned)z.grid), folds((unsigned)std::max<long long>(std::min<long long>(z.folds, 2048), (z.folds + kWave - 1) / kWave));
    auto launch = [&](auto blocks) {
        constexpr int RG = decltype(blocks)::value;
        hipLaunchKernelGGL((draft_tree_kernel<T, BITS, RG>), grid, dim3(tree_waves(RG) * kWave), 0, stream, a, t);
        if (z.folds) hipLaunchKernelGGL((fold_trees_kernel<T, RG>), folds, dim3(kFoldThreads), 0, stream, a, t);
    };
    if (z.RG == 4)
        launch(std::integral_constant<int, 4>{});
    else if (z.RG == 2)
        launch(std::integral_constant<int, 2>{});
    else if constexpr (BITS == 16)
        launch(std::integral_constant<int, 1>{});
    return hipGetLastError();
}

template <class T> hipError_t launch_bits(const TreeArgs& a, void* workspace, hipStream_t stream) {
    switch (a.kv.kv_bits) {
        case 8:
            return launch_tree<T, 8>(a, workspace, stream);
        case 4:
            return launch_tree<T, 4>(a, workspace, stream);
        default:
            return launch_tree<T, 16>(a, workspace, stream);
    }
}

}  // namespace

size_t tree_workspace_bytes(const LayerParams& lp, int batch, int total_new, int max_new, int max_pages, int sel_stride) {
    size_t most = 0;
    for (bool quantised : {false, true}) {  // whichever the call comes with
        const TreeSizes z = tree_sizes(lp, batch, total_new, max_new, max_pages, sel_stride, quantised);
        most = std::max(most, z.pieces_bytes + z.ml_bytes + z.partial_bytes);
    }
    return most;
}

hipError_t preload_tree_kernels() {
    hipFuncAttributes attr;
    return hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&draft_tree_kernel<F16, 16, 1>));
}

hipError_t launch_sparse_decode_tree(int dtype, const TreeArgs& a, void* workspace, hipStream_t stream) {
    return dtype == 0 ? launch_bits<F16>(a, workspace, stream) : launch_bits<BF16>(a, workspace, stream);
}

}  // namespace lserve
