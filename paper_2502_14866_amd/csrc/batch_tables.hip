// What a batch's new tokens need before its kernels run, without a trip to the host: pages off the free list, running counts,
// positions and slots (extend_tables_kernel), and the ancestors of drafted tokens (tree_masks_kernel).  Whole numbers only, some tens
// of kilobytes for a decode step: what these calls take is the time of a launch and of a few dependent loads.
#include <algorithm>

#include "kernels.h"

namespace lserve {

namespace {

constexpr int kTableThreads = 256, kTableWaves = kTableThreads / kWave;
constexpr int kTokensPerThread = 4, kTableTokens = kTableThreads * kTokensPerThread;  // tokens of a workgroup

}  // namespace

// A workgroup owns kTableTokens consecutive new tokens of the batch.  It runs over the sequences, a thread to each, with a running
// count of tokens and pages (so no workgroup waits for another, and one launch does it all), and leaves a mark for every sequence at the
// first of its tokens among its own; a maximum over the marks then tells every token its sequence.  The page of a token comes from the table
// where it was there before and from the free list where it is new: the table entries other workgroups write are not read.  Workgroup 0
// also writes what there is per sequence.
// Bound: latency, of a launch and three loads that wait for each other (lengths, then a table entry or a free page).  64 sequences of one new token
// 4.0 us; 500 prompts of 16 .. 8192 new tokens, 655 thousand in 640 workgroups and 13 MB, 8.6 us.
// With 512 threads, and so half the rounds over the sequences, 64 sequences take 1 us longer, 500 prompts 0.4, and 2000 sequences 0.2 less; lengths of
// the next round loaded ahead change nothing.
__global__ __launch_bounds__(kTableThreads) void extend_tables_kernel(ExtendArgs a) {
    __shared__ int4 marks[kTableTokens];  // at the first token of a sequence: (sequence, its first token, pages handed out before, length)
    __shared__ int owner[kTableTokens];   // index of the mark, or -1
    __shared__ int2 wave_total[2][kTableWaves];
    __shared__ int wave_mark[kTableWaves];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int page = 1 << a.page_log2;
    const bool first_one = blockIdx.x == 0;
    const int t0 = (int)blockIdx.x * kTableTokens, t1 = t0 + min(kTableTokens, a.total - t0);  // (in differences: the last tokens are next to 2^31)
    auto pages_of = [&](unsigned tokens) { return (int)min((tokens + page - 1) >> a.page_log2, (unsigned)a.max_pages); };
#pragma unroll
    for (int i = 0; i < kTokensPerThread; ++i) owner[i * kTableThreads + tid] = -1;
    int tokens = 0, pages = 0;  // of the sequences so far
    for (int base = 0, turn = 0; base < a.batch; base += kTableThreads, turn ^= 1) {
        const int b = base + tid;
        int n = 0, len = 0;
        if (b < a.batch) {
            n = max(a.new_lens[b], 0);
            len = max(a.seq_lens[b], 0);
        }
        const int fresh = pages_of((unsigned)len + (unsigned)n) - pages_of((unsigned)len);
        const int n_sum = wave_scan(n, 0, add), p_sum = wave_scan(fresh, 0, add);
        if (lane == kWave - 1) wave_total[turn][wave] = make_int2(n_sum, p_sum);
        __syncthreads();  // (of two places in turn: one barrier a round is enough; the first one also covers `owner`)
        int start = tokens + n_sum - n, handed = pages + p_sum - fresh;
#pragma unroll
        for (int i = 0; i < kTableWaves; ++i) {
            const int2 w = wave_total[turn][i];
            if (i < wave) {
                start += w.x;
                handed += w.y;
            }
            tokens += w.x;
            pages += w.y;
        }
        if (b < a.batch) {
            if (first_one) {
                a.cu_new[b] = start;
                a.new_seq_lens[b] = len + n;
            }
            const int from = max(start, t0);
            if (from < min(start + n, t1)) {
                marks[from - t0] = make_int4(b, start, handed, len);
                owner[from - t0] = from - t0;
            }
        }
        if (!first_one && tokens >= t1) break;  // (the same in all threads)
    }
    if (first_one && tid == 0) {
        a.cu_new[a.batch] = tokens;
        a.pages_taken[0] = pages;
    }
    if (t0 >= t1) return;
    __syncthreads();
    const int4 o4 = reinterpret_cast<const int4*>(owner)[tid];
    int own[kTokensPerThread] = {o4.x, o4.y, o4.z, o4.w};
#pragma unroll
    for (int i = 1; i < kTokensPerThread; ++i) own[i] = max(own[i], own[i - 1]);
    const int upto = wave_scan(own[kTokensPerThread - 1], -1, larger);
    if (lane == kWave - 1) wave_mark[wave] = upto;
    int left = __shfl_up(upto, 1);
    if (lane == 0) left = -1;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTableWaves - 1; ++i)
        if (i < wave) left = max(left, wave_mark[i]);
    int position[kTokensPerThread];
    long long slot[kTokensPerThread], ring_slot_[kTokensPerThread];
    const int ring = a.sink_pages + a.local_pages;
#pragma unroll
    for (int i = 0; i < kTokensPerThread; ++i) {
        const int t = t0 + tid * kTokensPerThread + i;
        position[i] = -1;
        slot[i] = ring_slot_[i] = -1;
        if (t >= t1 || t >= tokens) continue;
        const int4 m = marks[max(own[i], left)];
        // (unsigned, here and below: lengths that are not lengths lead to no address outside the arrays)
        const unsigned upos = (unsigned)m.w + (unsigned)(t - m.y);
        const int pos = (int)upos, p = (int)(upos >> a.page_log2), in_page = pos & (page - 1);
        const int had = pages_of((unsigned)m.w);
        position[i] = pos;
        int phys = -1;
        if (p < a.max_pages) {
            int* entry = a.page_table + (size_t)m.x * a.max_pages + p;
            if (p >= had) {
                const int index = m.z + (p - had);
                if ((unsigned)index < (unsigned)a.num_free) phys = a.free_pages[index];
                if (in_page == 0) *entry = phys;  // the first token of a new page is one of the new tokens
            } else if (a.slots) {
                phys = *entry;
            }
        }
        if (phys >= 0) slot[i] = ((long long)phys << a.page_log2) + in_page;
        if (a.ring_slots) {
            const int n = a.new_lens[m.x];
            const int last = (int)(((unsigned)m.w + (unsigned)n - 1) >> a.page_log2);  // page of the sequence's last token
            if (p < a.sink_pages || p > last - a.local_pages) {
                const int r = p < a.sink_pages ? p : a.sink_pages + (p - a.sink_pages) % a.local_pages;
                ring_slot_[i] = ((long long)a.ring_table[(size_t)m.x * ring + r] << a.page_log2) + in_page;
            }
        }
    }
    const int t = t0 + tid * kTokensPerThread;
    if (t1 - t >= kTokensPerThread) {  // 16-byte stores: `t` is a multiple of four
        if (a.positions) *reinterpret_cast<int4*>(a.positions + t) = make_int4(position[0], position[1], position[2], position[3]);
#pragma unroll
        for (int i = 0; i < kTokensPerThread; i += 2) {
            if (a.slots) *reinterpret_cast<longlong2*>(a.slots + t + i) = make_longlong2(slot[i], slot[i + 1]);
            if (a.ring_slots) *reinterpret_cast<longlong2*>(a.ring_slots + t + i) = make_longlong2(ring_slot_[i], ring_slot_[i + 1]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kTokensPerThread; ++i) {
            if (t + i >= t1) break;
            if (a.positions) a.positions[t + i] = position[i];
            if (a.slots) a.slots[t + i] = slot[i];
            if (a.ring_slots) a.ring_slots[t + i] = ring_slot_[i];
        }
    }
}

// Ancestors by doubling: before round r a node knows those of fewer than 2^r steps, and the 2^r-th of them, whose own set it takes over.  A workgroup
// to a sequence, a thread to a node, WORDS words of the set in its registers; the sets meet in LDS, read by all before they are
// written by any.  Rounds end when no node has an ancestor left (drafted trees are a handful of levels deep: two or three rounds).
// Bound: latency.  16 trees of 32 tokens 3.0 us, 256 trees of up to 200 4.6 us.
template <int WORDS>
__global__ __launch_bounds__(WORDS * 64) void tree_masks_kernel(const int* __restrict__ parents, const int* __restrict__ cu_new,
                                                                const int* __restrict__ seq_lens, int total_new, int max_new, int mask_words,
                                                                unsigned long long* __restrict__ tree_mask, int* __restrict__ positions) {
    constexpr int kNodes = WORDS * 64;
    __shared__ unsigned long long sets[WORDS][kNodes];
    __shared__ int2 up[kNodes];  // (the 2^r-th ancestor or -1, steps to the farthest known one)
    const int b = blockIdx.x, j = threadIdx.x;
    const int start = max(cu_new[b], 0), n = min(min(cu_new[b + 1] - start, max_new), total_new - start);
    if (n <= 0) return;
    const int len = seq_lens[b];
    int at = -1, depth = 0;
    if (j < n) {
        at = parents[start + j];
        if (at < 0 || at >= j) at = -1;
        depth = at >= 0 ? 1 : 0;
    }
    unsigned long long set[WORDS];
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
        set[w] = j / 64 == w ? 1ull << (j % 64) : 0ull;
        if (j < n) sets[w][j] = set[w];
    }
    up[j] = make_int2(at, depth);
    while (__syncthreads_or(at >= 0)) {
        int2 far = make_int2(-1, 0);
        if (at >= 0) {
            far = up[at];
#pragma unroll
            for (int w = 0; w < WORDS; ++w) set[w] |= sets[w][at];
        }
        __syncthreads();
        if (at >= 0) {
            at = far.x;
            depth += far.y;
            up[j] = make_int2(at, depth);
#pragma unroll
            for (int w = 0; w < WORDS; ++w) sets[w][j] = set[w];
        }
    }
    if (j >= n) return;
    positions[start + j] = len + depth;
    unsigned long long* row = tree_mask + (size_t)(start + j) * mask_words;
#pragma unroll
    for (int w = 0; w < WORDS; ++w)
        if (w < mask_words) row[w] = set[w];
    for (int w = WORDS; w < mask_words; ++w) row[w] = 0;
}

hipError_t preload_table_kernels() {
    hipFuncAttributes attr;
    return hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&extend_tables_kernel));
}

hipError_t launch_extend_tables(const ExtendArgs& a, hipStream_t stream) {
    const int grid = std::max(1, (int)(((long long)a.total + kTableTokens - 1) / kTableTokens));
    hipLaunchKernelGGL(extend_tables_kernel, dim3(grid), dim3(kTableThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_tree_masks(const int* parents, const int* cu_new, const int* seq_lens, int batch, int total_new, int max_new, int mask_words,
                             unsigned long long* tree_mask, int* positions, hipStream_t stream) {
    // a thread to a node: one wavefront, four or sixteen
#define LSERVE_MASKS(W)                                                                                                                       \
    hipLaunchKernelGGL(tree_masks_kernel<W>, dim3(batch), dim3(W * 64), 0, stream, parents, cu_new, seq_lens, total_new, max_new, mask_words, \
                       tree_mask, positions)
    if (max_new <= 64)
        LSERVE_MASKS(1);
    else if (max_new <= 256)
        LSERVE_MASKS(4);
    else
        LSERVE_MASKS(16);
#undef LSERVE_MASKS
    return hipGetLastError();
}

}  // namespace lserve
