// C ABI of the library (see include/lserve.h): host-side argument validation, translation of the
// public structs into kernel parameter blocks, and launches on the caller's stream.  No device
// memory is allocated or freed here and no state survives a call.
#include "../../include/lserve.h"

#include <cmath>
#include <iterator>
#include <limits>
#include <mutex>

#include "kernels.h"

using namespace lserve;

int lserve::num_compute_units() {
    static const int cus = [] {
        int dev = 0, n = 0;
        if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
            n <= 0) {
            (void)hipGetLastError();
            return 256;
        }
        return n;
    }();
    return cus;
}

// Scratch of lserve_sparse_decode_noalloc: the partial results the decode kernels exchange, which the other
// decode entry point keeps in the caller's workspace.  One copy per GPU for the life of the process.  In host code
// the name is only a handle: the address on a device comes from hipGetSymbolAddress (scratch_on_current_device).
constexpr size_t kScratchBytes = LSERVE_NOALLOC_SCRATCH_BYTES;
static __device__ __align__(256) unsigned char scratch[kScratchBytes];

namespace {

thread_local int g_last_hip_error = 0;

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mutex;
void* g_scratch_ptr[kMaxDevices] = {};  // device address of `scratch`, per device, once resolved

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// An array of a call, if it is given.
struct Range {
    const void* at;
    long long bytes;
};
bool meet(const Range& a, const Range& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
    return a.at && b.at && a.bytes > 0 && b.bytes > 0 && x < y + (uintptr_t)b.bytes && y < x + (uintptr_t)a.bytes;
}

// Rows of a call, `apart` bytes from one to the next.
struct Rows {
    const void* at;
    long long bytes, apart, count;
};
bool meet(const Range& a, const Rows& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
    if (!meet(a, Range{b.at, (b.count - 1) * b.apart + b.bytes})) return false;
    // the first row that does not end in front of the array
    const uintptr_t first = x < y + (uintptr_t)b.bytes ? 0 : (x - y - (uintptr_t)b.bytes) / (uintptr_t)b.apart + 1;
    return first < (uintptr_t)b.count && y + first * (uintptr_t)b.apart < x + (uintptr_t)a.bytes;
}

int fail_hip(hipError_t e) {
    g_last_hip_error = (int)e;
    return LSERVE_ERR_HIP;
}

// Address of `scratch` on the device that is current on the calling thread; resolved once per device.
int scratch_on_current_device(void** ptr) {
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return fail_hip(e);
    if (dev < 0 || dev >= kMaxDevices) return LSERVE_ERR_UNSUPPORTED;
    std::lock_guard<std::mutex> lock(g_scratch_mutex);
    if (!g_scratch_ptr[dev]) {
        void* p = nullptr;
        e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess) return fail_hip(e);
        if (!p) return fail_hip(hipErrorInvalidSymbol);
        g_scratch_ptr[dev] = p;
    }
    *ptr = g_scratch_ptr[dev];
    return LSERVE_OK;
}

// Validates the layer description and fills the kernel parameter block.
int make_layer(const lserve_attn_desc* d, LayerParams* lp) {
    if (!d || !d->kv_head_is_streaming) return LSERVE_ERR_INVALID_ARG;
    if (d->num_q_heads <= 0 || d->num_kv_heads <= 0 || d->page_size <= 0 || d->logical_page_size <= 0)
        return LSERVE_ERR_INVALID_ARG;
    if (d->sink_tokens < 0 || d->local_tokens < 1) return LSERVE_ERR_INVALID_ARG;
    if (d->page_size % d->logical_page_size != 0) return LSERVE_ERR_INVALID_ARG;
    if (!(d->sm_scale >= 0.f) || std::isinf(d->sm_scale)) return LSERVE_ERR_INVALID_ARG;
    if (d->head_dim != kHeadDim) return LSERVE_ERR_UNSUPPORTED;
    if (d->dtype != LSERVE_DTYPE_FP16 && d->dtype != LSERVE_DTYPE_BF16) return LSERVE_ERR_UNSUPPORTED;
    if (d->num_q_heads % d->num_kv_heads != 0) return LSERVE_ERR_UNSUPPORTED;
    if (d->num_kv_heads > 64 || d->num_q_heads / d->num_kv_heads > kMaxGroup) return LSERVE_ERR_UNSUPPORTED;
    if (d->page_size != 16 && d->page_size != 32 && d->page_size != 64 && d->page_size != 128)
        return LSERVE_ERR_UNSUPPORTED;
    if (d->page_size / d->logical_page_size > kMaxLogical) return LSERVE_ERR_UNSUPPORTED;
    lp->H = d->num_q_heads;
    lp->Hkv = d->num_kv_heads;
    lp->group = lp->H / lp->Hkv;
    lp->NP = d->page_size;
    lp->NL = d->logical_page_size;
    lp->g = lp->NP / lp->NL;
    lp->sink_pages = (d->sink_tokens + lp->NP - 1) / lp->NP;
    lp->local_pages = (d->local_tokens + lp->NP - 1) / lp->NP;
    lp->streaming_mask = 0;
    for (int h = 0; h < lp->Hkv; ++h)
        if (d->kv_head_is_streaming[h]) lp->streaming_mask |= 1ull << h;
    const float scale = d->sm_scale > 0.f ? d->sm_scale : 1.0f / std::sqrt((float)kHeadDim);
    lp->sm_scale_log2 = scale * 1.4426950408889634f;
    return LSERVE_OK;
}

// need_stream: the call touches streaming heads, so every one of them must live in some pool.
int make_paged(const lserve_paged_kv* kv, const LayerParams& lp, bool need_k, bool need_v, bool need_stats,
               bool need_stream, PagedParams* pp) {
    if (!kv || !kv->page_table || !kv->seq_lens) return LSERVE_ERR_INVALID_ARG;
    if (kv->batch <= 0 || kv->max_pages_per_seq <= 0 || kv->num_pages <= 0) return LSERVE_ERR_INVALID_ARG;
    if (kv->batch > 65535) return LSERVE_ERR_UNSUPPORTED;
    if ((need_k && !kv->k_pool) || (need_v && !kv->v_pool) || (need_stats && !kv->stats)) return LSERVE_ERR_INVALID_ARG;
    if (!aligned16(kv->k_pool) || !aligned16(kv->v_pool) || !aligned16(kv->stats) || !aligned16(kv->page_table) ||
        !aligned16(kv->seq_lens))
        return LSERVE_ERR_INVALID_ARG;
    pp->k_pool = kv->k_pool;
    pp->v_pool = kv->v_pool;
    pp->stats = kv->stats;
    pp->page_table = kv->page_table;
    pp->seq_lens = kv->seq_lens;
    pp->batch = kv->batch;
    pp->max_pages = kv->max_pages_per_seq;
    pp->num_pages = kv->num_pages;
    int n_stream = 0;
    for (int h = 0; h < lp.Hkv; ++h) n_stream += (int)((lp.streaming_mask >> h) & 1ull);
    const int n_dense = lp.Hkv - n_stream;
    pp->pool_heads = kv->pool_heads == 0 ? lp.Hkv : kv->pool_heads;
    if (pp->pool_heads != lp.Hkv && pp->pool_heads != n_dense) return LSERVE_ERR_INVALID_ARG;
    if ((kv->k_pool_stream == nullptr) != (kv->v_pool_stream == nullptr)) return LSERVE_ERR_INVALID_ARG;
    pp->k_stream = kv->k_pool_stream;
    pp->v_stream = kv->v_pool_stream;
    pp->ring_table = kv->ring_table;
    pp->stream_heads = n_stream;
    pp->ring = lp.sink_pages + lp.local_pages;
    if (pp->k_stream) {
        if (!kv->ring_table || kv->num_pages_stream <= 0 || n_stream == 0) return LSERVE_ERR_INVALID_ARG;
        if (!aligned16(kv->k_pool_stream) || !aligned16(kv->v_pool_stream) || !aligned16(kv->ring_table))
            return LSERVE_ERR_INVALID_ARG;
    }
    if (kv->kv_bits != 0 && kv->kv_bits != 16 && kv->kv_bits != 8 && kv->kv_bits != 4) return LSERVE_ERR_INVALID_ARG;
    pp->kv_bits = kv->kv_bits == 0 ? 16 : kv->kv_bits;
    if (pp->kv_bits != 16 && lp.NP != 64) return LSERVE_ERR_UNSUPPORTED;
    const bool main_holds_all = pp->pool_heads == lp.Hkv;
    if (need_stream && n_stream > 0 && !main_holds_all && !pp->k_stream) return LSERVE_ERR_INVALID_ARG;
    return LSERVE_OK;
}

HeadList selecting_heads(const LayerParams& lp) {
    HeadList hl;
    hl.count = 0;
    for (int h = 0; h < lp.Hkv; ++h)
        if (!((lp.streaming_mask >> h) & 1ull)) hl.idx[hl.count++] = (unsigned char)h;
    return hl;
}

bool rotary_is_fine(const lserve_rotary_desc* r) {
    return r->inv_freq && r->rotary_dim >= 2 && r->rotary_dim % 2 == 0 && r->scale >= 0.f && !std::isinf(r->scale) &&
           (r->interleaved == 0 || r->interleaved == 1) && aligned16(r->inv_freq);
}

// How heads are normed and turned; positions as they are handed over (null is fine here where `own_places` says what stands in for them).
int make_turn(const lserve_head_norm* norm, const lserve_rotary_desc* rotary, const lserve_position_axes* axes,
              const int32_t* positions, int64_t positions_stride, int total, bool own_places, TurnArgs* t) {
    if (norm) {
        if ((norm->kind != LSERVE_NORM_RMS && norm->kind != LSERVE_NORM_CENTRED) || (norm->per_head != 0 && norm->per_head != 1)) return LSERVE_ERR_INVALID_ARG;
        if (!(norm->eps >= std::numeric_limits<float>::min()) || std::isinf(norm->eps) || !aligned16(norm->q_weight) || !aligned16(norm->k_weight)) return LSERVE_ERR_INVALID_ARG;
        t->norm = norm->kind == LSERVE_NORM_RMS ? 1 : 2;
        t->weight_step = norm->per_head ? kHeadDim : 0;
        t->eps = norm->eps;
        t->q_weight = norm->q_weight;
        t->k_weight = norm->k_weight;
    }
    t->axes = 1;
    t->scale = 1.f;
    if (rotary) {
        if (!rotary_is_fine(rotary) || (!positions && !own_places)) return LSERVE_ERR_INVALID_ARG;
        if (rotary->rotary_dim > kHeadDim) return LSERVE_ERR_UNSUPPORTED;
        t->inv_freq = rotary->inv_freq;
        t->rotary_dim = rotary->rotary_dim;
        t->interleaved = rotary->interleaved;
        if (rotary->scale != 0.f) t->scale = rotary->scale;
    }
    if (axes) {
        if (axes->num_axes < 1 || !rotary || !axes->pair_axis) return LSERVE_ERR_INVALID_ARG;
        if (axes->num_axes > 4) return LSERVE_ERR_UNSUPPORTED;
        if (positions && positions_stride < total) return LSERVE_ERR_INVALID_ARG;
        for (int i = 0; i < rotary->rotary_dim / 2; ++i) {
            if (axes->pair_axis[i] >= axes->num_axes) return LSERVE_ERR_INVALID_ARG;
            t->axis_of[i / 32] |= (unsigned long long)axes->pair_axis[i] << (2 * (i % 32));
        }
        t->axes = axes->num_axes;
        t->axis_stride = positions_stride;
    }
    if (!aligned16(positions)) return LSERVE_ERR_INVALID_ARG;
    t->positions = positions;
    return LSERVE_OK;
}

// What is read of all that.
struct TurnRanges {
    Range at[4];
    TurnRanges(const LayerParams& lp, const TurnArgs& t, int total)
        : at{{t.positions, ((t.axes - 1) * t.axis_stride + total) * 4}, {t.inv_freq, t.rotary_dim * 4LL},
             {t.q_weight, (t.weight_step ? lp.H : 1) * kHeadDim * 4LL}, {t.k_weight, (t.weight_step ? lp.Hkv : 1) * kHeadDim * 4LL}} {}
};

// Rows of heads, dense where they may be written in place; `out` as handed over.
bool rows_are_fine(const void* rows, int64_t stride, int64_t row, const void* out) {
    return stride >= row && stride % 8 == 0 && !(out == rows && stride != row) && aligned16(rows) && aligned16(out);
}

// lserve_rotary_axes and lserve_norm_rotary behind their own checks.
int turned_rows(const lserve_attn_desc* desc, const LayerParams& lp, const TurnArgs& turn, const void* q, const void* k, int32_t total, int64_t q_stride,
                int64_t k_stride, void* q_out, void* k_out, void* stream) {
    if (total <= 0 || (!q && !k) || !q != !q_out || !k != !k_out) return LSERVE_ERR_INVALID_ARG;
    const int64_t q_row = (int64_t)lp.H * kHeadDim, k_row = (int64_t)lp.Hkv * kHeadDim;
    if ((q && !rows_are_fine(q, q_stride, q_row, q_out)) || (k && !rows_are_fine(k, k_stride, k_row, k_out))) return LSERVE_ERR_INVALID_ARG;
    // (outputs are whole, inputs rows that may lie apart; in place a row is read before it is written)
    const Rows q_in = {q, q_row * 2, q_stride * 2, total}, k_in = {k, k_row * 2, k_stride * 2, total};
    const Range q_to = {q_out, total * q_row * 2}, k_to = {k_out, total * k_row * 2};
    const TurnRanges read(lp, turn, total);
    for (const Range& o : {q_to, k_to}) {
        for (const Range& i : read.at)
            if (meet(o, i)) return LSERVE_ERR_INVALID_ARG;
        if ((o.at != q && meet(o, q_in)) || (o.at != k && meet(o, k_in))) return LSERVE_ERR_INVALID_ARG;
    }
    if (meet(q_to, k_to) || (q_out && q_out == k) || (k_out && k_out == q)) return LSERVE_ERR_INVALID_ARG;
    TurnedRowsArgs a = {};
    a.turn = turn;
    a.q = q;
    a.k = k;
    a.q_out = q_out;
    a.k_out = k_out;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.heads_q = q ? lp.H : 0;
    a.heads_k = k ? lp.Hkv : 0;
    a.total = total;
    const hipError_t e = launch_turned_rows(desc->dtype, a, (hipStream_t)stream);
    return e == hipSuccess ? LSERVE_OK : fail_hip(e);
}

size_t select_workspace_bytes(const LayerParams& lp, int batch, int max_pages) {
    return (size_t)batch * lp.Hkv * max_pages * sizeof(float);
}

}  // namespace

extern "C" {

int lserve_build_page_stats(const lserve_attn_desc* desc, const lserve_paged_kv* kv, const int32_t* start_pos,
                            int32_t max_tail_pages, void* stream) {
    LayerParams lp;
    PagedParams pp;
    int rc = make_layer(desc, &lp);
    if (rc) return rc;
    rc = make_paged(kv, lp, true, false, true, false, &pp);
    if (rc) return rc;
    if (pp.kv_bits != 16) return LSERVE_ERR_UNSUPPORTED;  // statistics come from 16-bit keys (lserve_append_kv)
    if (max_tail_pages < 0 || !aligned16(start_pos)) return LSERVE_ERR_INVALID_ARG;
    const int tail = (max_tail_pages == 0 || max_tail_pages > pp.max_pages) ? pp.max_pages : max_tail_pages;
    hipError_t e = launch_page_stats(desc->dtype, lp, pp, start_pos, tail, selecting_heads(lp), (hipStream_t)stream);
    return e == hipSuccess ? LSERVE_OK : fail_hip(e);
}

int lserve_append_kv(const lserve_attn_desc* desc, const lserve_paged_kv* kv, const void* k_new, const void* v_new,
                     const int32_t* cu_new, const int32_t* start_pos, int32_t max_new_per_seq, void* stream) {
    LayerParams lp;
    PagedParams pp;
    int rc = make_layer(desc, &lp);
    if (rc) return rc;
    rc = make_paged(kv, lp, true, true, selecting_heads(lp).count > 0, true, &pp);
    if (rc) return rc;
    if (!k_new || !v_new || !cu_new || !start_pos || max_new_per_seq <= 0) return LSERVE_ERR_INVALID_ARG;
    if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(cu_new) || !aligned16(start_pos)) return LSERVE_ERR_INVALID_ARG;
    hipError_t e = launch_append_kv(desc->dtype, lp, pp, k_new, v_new, cu_new, start_pos, max_new_per_seq,
                                    (hipStream_t)stream);
    return e == hipSuccess ? LSERVE_OK : fail_hip(e);
}

int lserve_select_pages(const lserve_attn_desc* desc, const lserve_paged_kv* kv, const void* q, int32_t budget_tokens,
                        const int32_t* stats_valid_len, int32_t* sel_pages, int32_t* sel_count, int32_t* sel_seq_len,
                        float* scores_out, void* workspace, size_t workspace_bytes, void* stream) {
    LayerParams lp;
    PagedParams pp;
    int rc = make_layer(desc, &lp);
    if (rc) return rc;
    rc = make_paged(kv, lp, stats_valid_len != nullptr, false, selecting_heads(lp).count > 0, false, &pp);
    if (rc) return rc;
    if (stats_valid_len && pp.kv_bits != 16) return LSERVE_ERR_UNSUPPORTED;  // no 16-bit keys to rebuild from
    if (!q || !sel_pages || !sel_count || !sel_seq_len) return LSERVE_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(stats_valid_len) || !aligned16(sel_pages) || !aligned16(sel_count) || !aligned16(sel_seq_len) ||
        !aligned16(scores_out) || !aligned16(workspace))
        return LSERVE_ERR_INVALID_ARG;
    if (budget_tokens < lp.NP) return LSERVE_ERR_INVALID_ARG;
    float* scores = scores_out;
    if (!scores) {
        if (!workspace || workspace_bytes < select_workspace_bytes(lp, pp.batch, pp.max_pages)) return LSERVE_ERR_WORKSPACE;
        scores = reinterpret_cast<float*>(workspace);
    }
    hipError_t e = launch_select_pages(desc->dtype, lp, pp, q, stats_valid_len, budget_tokens / lp.NP, sel_pages, sel_count,
                                       sel_seq_len, scores, scores_out != nullptr, selecting_heads(lp), (hipStream_t)stream);
    return e == hipSuccess ? LSERVE_OK : fail_hip(e);
}

namespace {
int prefill_impl(const lserve_attn_desc* desc, const lserve_block_mask* mask, const void* q, const void* k, const void* v,
                 const int32_t* cu_seqlens, int32_t batch, int32_t total_tokens, int32_t max_seqlen, void* out,
                 float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
    LayerParams lp;
    int rc = make_layer(desc, &lp);
    if (rc) return rc;
    if (!q || !k || !v || !cu_seqlens || !out) return LSERVE_ERR_INVALID_ARG;
    if (batch <= 0 || total_tokens <= 0 || max_seqlen <= 0 || max_seqlen > total_tokens) return LSERVE_ERR_INVALID_ARG;
    if (batch > 65535) return LSERVE_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(cu_seqlens) ||
        !aligned16(lse_out) || !aligned16(workspace))
        return LSERVE_ERR_INVALID_ARG;
    if (lp.NP != 64) return LSERVE_ERR_UNSUPPORTED;
    PrefillMaskArgs ma = {};
    size_t need = prefill_workspace_bytes(lp, total_tokens, batch);
    if (mask) {
        if (!mask->head_mask || !mask->q_tile_start || !mask->row_ptr || (mask->nnz > 0 && !mask->cols))
            return LSERVE_ERR_INVALID_ARG;
        if (mask->num_masks <= 0 || mask->rows_per_mask <= 0 || mask->nnz < 0) return LSERVE_ERR_INVALID_ARG;
        if (!aligned16(mask->head_mask) || !aligned16(mask->q_tile_start) || !aligned16(mask->row_ptr) ||
            !aligned16(mask->cols))
            return LSERVE_ERR_INVALID_ARG;
        if (max_seqlen > 65536 * 64) return LSERVE_ERR_UNSUPPORTED;  // one byte of LDS per key tile in the merge pass
        ma.head_mask = mask->head_mask;
        ma.q_tile_start = mask->q_tile_start;
        ma.row_ptr = mask->row_ptr;
        ma.cols = mask->cols;
        ma.num_masks = mask->num_masks;
        ma.rows_per_mask = mask->rows_per_mask;
        ma.nnz = mask->nnz;
        need = masked_prefill_workspace_bytes(lp, total_tokens, batch, max_seqlen, mask->num_masks, mask->nnz);
    }
    if (need > 0 && (!workspace || workspace_bytes < need)) return LSERVE_ERR_WORKSPACE;
    hipError_t e = launch_sparse_prefill(desc->dtype, lp, q, k, v, cu_seqlens, batch, total_tokens, max_seqlen, out,
                                         lse_out, workspace, mask ? &ma : nullptr, (hipStream_t)stream);
    return e == hipSuccess ? LSERVE_OK : fail_hip(e);
}
}  // namespace

int lserve_sparse_prefill(const lserve_attn_desc* desc, const void* q, const void* k, const void* v,
                          const int32_t* cu_seqlens, int32_t batch, int32_t total_tokens, int32_t max_seqlen, void* out,
                          float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
    return prefill_impl(desc, nullptr, q, k, v, cu_seqlens, batch, total_tokens, max_seqlen, out, lse_out, workspace,
                        workspace_bytes, stream);
}

int lserve_sparse_prefill_masked(const lserve_attn_desc* desc, const lserve_block_mask* mask, const void* q, const void* k,
                                 const void* v, const int32_t* cu_seqlens, int32_t batch, int32_t total_tokens,
                                 int32_t max_seqlen, void* out, float* lse_out, void* workspace, size_t workspace_bytes,
                                 void* stream) {
    if (!mask) return LSERVE_ERR_INVALID_ARG;
    return prefill_impl(desc, mask, q, k, v, cu_seqlens, batch, total_tokens, max_seqlen, out, lse_out, workspace,
                        workspace_bytes, stream);
}

namespace {
int prefill_paged_impl(const lserve_attn_desc* desc, const lserve_paged_kv* kv, const void* q, const int32_t* cu_q,
                       int32_t total_new, int32_t max_new_per_seq, int32_t max_seqlen, void* out, float* lse_out,
                       const void* workspace, void* scratch, size_t scratch_bytes, void* stream) {
    LayerParams lp;
    PagedParams pp;
    int rc = make_layer(desc, &lp);
    if (rc) return rc;
    rc = make_paged(kv, lp, true, true, false, true, &pp);
    if (rc) return rc;
    if (lp.NP != 64) return LSERVE_ERR_UNSUPPORTED;
    if (pp.pool_heads != lp.Hkv || pp.k_stream) return LSERVE_ERR_UNSUPPORTED;  // one pool holding every head
    if (pp.kv_bits != 16) return LSERVE_ERR_UNSUPPORTED;
    if (!q || !cu_q || !out) return LSERVE_ERR_INVALID_ARG;
    if (total_new <= 0 || max_new_per_seq <= 0 || max_new_per_seq > total_new || max_seqlen < max_new_per_seq)
        return LSERVE_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(cu_q) || !aligned16(out) || !aligned16(lse_out) || !aligned16(workspace) || !aligned16(scratch))
        return LSERVE_ERR_INVALID_ARG;
    hipError_t e = launch_sparse_prefill_paged(desc->dtype, lp, pp, q, nullptr, nullptr, cu_q, total_new, max_new_per_seq,
                                               max_seqlen, out, lse_out, scratch, scratch_bytes, (hipStream_t)stream);
    return e == hipSuccess ? LSERVE_OK : fail_hip(e);
}
}  // namespace

int lserve_sparse_prefill_paged(const lserve_attn_desc* desc, const lserve_paged_kv* kv, const void* q,
                                const int32_t* cu_q, int32_t total_new, int32_t max_new_per_seq, int32_t max_seqlen,
                                void* out, float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
    (void)workspace_bytes;  // none needed, none used
    return prefill_paged_impl(desc, kv, q, cu_q, total_new, max_new_per_seq, max_seqlen, out, lse_out, workspace, nullptr, 0, stream);
}

int lserve_sparse_prefill_paged_scratch(const lserve_attn_desc* desc, const lserve_paged_kv* kv, const void* q,
                                        const int32_t* cu_q, int32_t total_new, int32_t max_new_per_seq, int32_t max_seqlen,
                                        void* out, float* lse_out, void* scratch, size_t scratch_bytes, void* stream) {
    return prefill_paged_impl(desc, kv, q, cu_q, total_new, max_new_per_seq, max_seqlen, out, lse_out, nullptr, scratch,
                              scratch_bytes, stream);
}

int lserve_sparse_prefill_chunk(const lserve_attn_desc* desc, const lserve_paged_kv* kv, const void* q, const void* k_new,
                                const void* v_new, const int32_t* cu_new, int32_t total_new, int32_t max_new_per_seq,
                                void* out, float* lse_out, void* stream) {
    return lserve_sparse_prefill_chunk_scratch(desc, kv, q, k_new, v_new, cu_new, total_new, max_new_per_seq, out, lse_out,
                                               nullptr, 0, stream);
}

int lserve_sparse_prefill_chunk_scratch(const lserve_attn_desc* desc, const lserve_paged_kv* kv, const void* q,
                                        const void* k_new, const void* v_new, const int32_t* cu_new, int32_t total_new,
                                        int32_t max_new_per_seq, void* out, float* lse_out, void* scratch,
                                        size_t scratch_bytes, void* stream) {
    LayerParams lp;
    PagedParams pp;
    int rc = make_layer(desc, &lp);
    if (rc) return rc;
    rc = make_paged(kv, lp, true, true, false, true, &pp);
    if (rc) return rc;
    if (lp.NP != 64) return LSERVE_ERR_UNSUPPORTED;
    if (!q || !k_new || !v_new || !cu_new || !out) return LSERVE_ERR_INVALID_ARG;
    if (total_new <= 0 || max_new_per_seq <= 0 || max_new_per_seq > total_new) return LSERVE_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(cu_new) || !aligned16(out) ||
        !aligned16(lse_out) || !aligned16(scratch))
        return LSERVE_ERR_INVALID_ARG;
    hipError_t e = launch_sparse_prefill_paged(desc->dtype, lp, pp, q, k_new, v_new, cu_new, total_new, max_new_per_seq, 0,
                                               out, lse_out, scratch, scratch_bytes, (hipStream_t)stream);
    return e == hipSuccess ? LSERVE_OK : fail_hip(e);
}

size_t lserve_chunk_scratch_bytes(const lserve_attn_desc* desc, int32_t batch, int32_t total_new, int32_t max_new_per_seq,
                                  int32_t pages, int32_t kv_bits) {
    LayerParams lp;
    if (make_layer(desc, &lp) != LSERVE_OK || lp.NP != 64) return 0;
    if (batch <= 0 || total_new <= 0 || max_new_per_seq <= 0 || max_new_per_seq > total_new || pages <= 0) return 0;
    return chunk_scratch_bytes(lp, batch, total_new, max_new_per_seq, pages, kv_bits == 0 ? 16 : kv_bits);
}

int lserve_probe_prefill_shape(const lserve_attn_desc* desc, int32_t batch, int32_t total_rows, int32_t max_rows, int32_t pages,
                               int32_t kv_bits, int32_t* shape) {
    LayerParams lp;
    const int rc = make_layer(desc, &lp);
    if (rc) return rc;
    if (!shape || batch <= 0 || total_rows <= 0 || max_rows <= 0 || max_rows > total_rows || pages < 0) return LSERVE_ERR_INVALID_ARG;
    if (kv_bits != 0 && kv_bits != 16 && kv_bits != 8 && kv_bits != 4) return LSERVE_ERR_INVALID_ARG;
    if (lp.NP != 64) return LSERVE_ERR_UNSUPPORTED;
    int out[4];
    prefill_shape(lp, batch, total_rows, max_rows, pages, kv_bits == 0 ? 16 : kv_bits, out);
    for (int i = 0; i < 4; ++i) shape[i] = out[i];
    return LSERVE_OK;
}

int lserve_probe_prefill_plan(const lserve_attn_desc* desc, int32_t batch, int32_t total_rows, int32_t max_rows, int32_t pages,
                              int32_t kv_bits, int32_t scratch, int32_t* plan) {
    LayerParams lp;
    const int rc = make_layer(desc, &lp);
    if (rc) return rc;
    if (!plan || batch <= 0 || total_rows <= 0 || max_rows <= 0 || max_rows > total_rows || pages < 0) return LSERVE_ERR_INVALID_ARG;
    if (kv_bits != 0 && kv_bits != 16 && kv_bits != 8 && kv_bits != 4) return LSERVE_ERR_INVALID_ARG;
    if (lp.NP != 64) return LSERVE_ERR_UNSUPPORTED;
    int out[6];
    prefill_plan(lp, batch, total_rows, max_rows, pages, kv_bits == 0 ? 16 : kv_bits, scratch != 0, out);
    for (int i = 0; i < 6; ++i) plan[i] = out[i];
    return LSERVE_OK;
}

int lserve_probe_prefill_longest_first(const lserve_attn_desc* desc, int32_t batch, int32_t total_rows, int32_t max_rows, int32_t* first) {
    LayerParams lp;
    const int rc = make_layer(desc, &lp);
    if (rc) return rc;
    if (!first || batch <= 0 || total_rows <= 0 || max_rows <= 0 || max_rows > total_rows) return LSERVE_ERR_INVALID_ARG;
    if (lp.NP != 64) return LSERVE_ERR_UNSUPPORTED;
    *first = prefill_longest_first(lp, batch, total_rows, max_rows);
    return LSERVE_OK;
}

int lserve_probe_mask_walk(const lserve_attn_desc* desc, int32_t batch, int32_t total_tokens, int32_t max_seqlen,
                           int32_t num_masks, int32_t rows_per_mask, int32_t nnz, int32_t* walk) {
    LayerParams lp;
    const int rc = make_layer(desc, &lp);
    if (rc) return rc;
    if (!walk || batch <= 0 || total_tokens <= 0 || max_seqlen <= 0 || max_seqlen > total_tokens || num_masks <= 0 ||
        rows_per_mask <= 0 || nnz < 0)
        return LSERVE_ERR_INVALID_ARG;
    if (lp.NP != 64) return LSERVE_ERR_UNSUPPORTED;
    *walk = mask_walk(lp, batch, total_tokens, max_seqlen, num_masks, rows_per_mask, nnz);
    return LSERVE_OK;
}

size_t lserve_paged_prefill_workspace_bytes(const lserve_attn_desc* desc, int32_t batch, int32_t max_pages_per_seq) {
    LayerParams lp;
    if (make_layer(desc, &lp) != LSERVE_OK || batch <= 0 || max_pages_per_seq <= 0) return 0;
    return paged_prefill_workspace_bytes(lp, batch, max_pages_per_seq);
}

size_t lserve_masked_prefill_workspace_bytes(const lserve_attn_desc* desc, int32_t batch, int32_t total_tokens,
                                             int32_t max_seqlen, int32_t num_masks, int32_t nnz) {
    LayerParams lp;
    if (make_layer(desc, &lp) != LSERVE_OK) return 0;
    if (batch <= 0 || total_tokens <= 0 || max_seqlen <= 0 || num_masks <= 0 || nnz < 0) return 0;
    return masked_prefill_workspace_bytes(lp, total_tokens, batch, max_seqlen, num_masks, nnz);
}

namespace {
// Everything lserve_sparse_decode checks except the workspace.
int check_decode_args(const lserve_attn_desc* desc, const lserve_paged_kv* kv, const void* q, const int32_t* sel_pages,
                      const int32_t* sel_count, const int32_t* sel_seq_len, int32_t sel_stride, const void* out,
                      const float* lse_out, LayerParams* lp, PagedParams* pp) {
    int rc = make_layer(desc, lp);
    if (rc) return rc;
    rc = make_paged(kv, *lp, true, true, false, true, pp);
    if (rc) return rc;
    if (!q || !out) return LSERVE_ERR_INVALID_ARG;
    const bool any_selecting = selecting_heads(*lp).count > 0;
    if (any_selecting && (!sel_pages || !sel_count || !sel_seq_len || sel_stride <= 0)) return LSERVE_ERR_INVALID_ARG;
    if (sel_stride < 0) return LSERVE_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(out) || !aligned16(sel_pages) || !aligned16(sel_count) || !aligned16(sel_seq_len) ||
        !aligned16(lse_out))
        return LSERVE_ERR_INVALID_ARG;
    // the launch plan numbers the nominal index-table entries of the whole batch with 32-bit integers
    if ((long long)pp->batch * decode_nominal_entries(*lp, sel_stride) > 0x7fffffffLL) return LSERVE_ERR_UNSUPPORTED;
    return LSERVE_OK;
}
}  // namespace

int lserve_sparse_decode(const lserve_attn_desc* desc, const lserve_paged_kv* kv, const void* q,
                         const int32_t* sel_pages, const int32_t* sel_count, const int32_t* sel_seq_len,
                         int32_t sel_stride, void* out, float* lse_out, void* workspace, size_t workspace_bytes,
                         void* stream) {
    LayerParams lp;
    PagedParams pp;
    int rc = check_decode_args(desc, kv, q, sel_pages, sel_count, sel_seq_len, sel_stride, out, lse_out, &lp, &pp);
    if (rc) return rc;
    if (!aligned16(workspace)) return LSERVE_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < decode_workspace_bytes(lp, pp.batch, sel_stride)) return LSERVE_ERR_WORKSPACE;
    hipError_t e = launch_sparse_decode(desc->dtype, lp, pp, q, sel_pages, sel_count, sel_seq_len, sel_stride, out,
                                        lse_out, workspace, (hipStream_t)stream);
    return e == hipSuccess ? LSERVE_OK : fail_hip(e);
}

int lserve_sparse_decode_noalloc(const lserve_attn_desc* desc, const lserve_paged_kv* kv, const void* q,
                                 const int32_t* sel_pages, const int32_t* sel_count, const int32_t* sel_seq_len,
                                 int32_t sel_stride, void* out, float* lse_out, void* stream) {
    LayerParams lp;
    PagedParams pp;
    int rc = check_decode_args(desc, kv, q, sel_pages, sel_count, sel_seq_len, sel_stride, out, lse_out, &lp, &pp);
    if (rc) return rc;
    if (decode_workspace_bytes(lp, pp.batch, sel_stride) > kScratchBytes) return LSERVE_ERR_WORKSPACE;
    void* ws = nullptr;
    rc = scratch_on_current_device(&ws);
    if (rc) return rc;
    // The arrival counters at the start of the scratch are zero when the device image is loaded and every launch
    // leaves them at zero; the kernels write every partial they later read.
    hipError_t e = launch_sparse_decode(desc->dtype, lp, pp, q, sel_pages, sel_count, sel_seq_len, sel_stride, out,
                                        lse_out, ws, (hipStream_t)stream);
    return e == hipSuccess ? LSERVE_OK : fail_hip(e);
}

int lserve_extend_tables(const lserve_attn_desc* desc, const lserve_paged_kv* kv, const int32_t* new_lens, const int32_t* free_pages,
                         int32_t num_free, int32_t total_new, int32_t* cu_new, int32_t* new_seq_lens, int32_t* pages_taken,
                         int32_t* positions, int64_t* slots, int64_t* ring_slots, void* stream) {
    LayerParams lp;
    const int rc = make_layer(desc, &lp);
    if (rc) return rc;
    if (!kv || !kv->page_table || !kv->seq_lens || kv->batch <= 0 || kv->max_pages_per_seq <= 0) return LSERVE_ERR_INVALID_ARG;
    if (kv->batch > 65535) return LSERVE_ERR_UNSUPPORTED;
    if (!new_lens || num_free < 0 || (num_free > 0 && !free_pages) || total_new < 0 || !cu_new || !new_seq_lens || !pages_taken)
        return LSERVE_ERR_INVALID_ARG;
    if (ring_slots && !kv->ring_table) return LSERVE_ERR_INVALID_ARG;
    // what one workgroup writes others still read the lengths, the free list and the tables for
    const long long batch = kv->batch, total = total_new;
    const Range in[] = {{kv->seq_lens, batch * 4}, {new_lens, batch * 4}, {free_pages, num_free * 4LL},
                        {ring_slots ? kv->ring_table : nullptr, batch * (lp.sink_pages + lp.local_pages) * 4}};
    const Range out[] = {{cu_new, (batch + 1) * 4}, {new_seq_lens, batch * 4}, {pages_taken, 4}, {kv->page_table, batch * kv->max_pages_per_seq * 4},
                         {positions, total * 4}, {slots, total * 8}, {ring_slots, total * 8}};
    for (const Range& o : out) {
        for (const Range& i : in)
            if (meet(o, i)) return LSERVE_ERR_INVALID_ARG;
        for (const Range& other : out)
            if (&other != &o && meet(o, other)) return LSERVE_ERR_INVALID_ARG;
    }
    if (!aligned16(kv->page_table) || !aligned16(kv->seq_lens) || !aligned16(kv->ring_table) || !aligned16(new_lens) ||
        (reinterpret_cast<uintptr_t>(free_pages) & 3u) != 0 || !aligned16(cu_new) || !aligned16(new_seq_lens) || !aligned16(pages_taken) || !aligned16(positions) ||
        !aligned16(slots) || !aligned16(ring_slots))
        return LSERVE_ERR_INVALID_ARG;
    ExtendArgs a = {};
    a.page_table = const_cast<int*>(kv->page_table);  // device memory of the caller's, which only this call writes
    a.seq_lens = kv->seq_lens;
    a.new_lens = new_lens;
    a.free_pages = free_pages;
    a.ring_table = kv->ring_table;
    a.cu_new = cu_new;
    a.new_seq_lens = new_seq_lens;
    a.pages_taken = pages_taken;
    a.positions = positions;
    a.slots = (long long*)slots;
    a.ring_slots = (long long*)ring_slots;
    a.batch = kv->batch;
    a.max_pages = kv->max_pages_per_seq;
    a.num_free = num_free;
    a.total = total_new;
    a.page_log2 = __builtin_ctz((unsigned)lp.NP);
    a.sink_pages = lp.sink_pages;
    a.local_pages = lp.local_pages;
    const hipError_t e = launch_extend_tables(a, (hipStream_t)stream);
    return e == hipSuccess ? LSERVE_OK : fail_hip(e);
}

int lserve_rotary(const lserve_attn_desc* desc, const lserve_rotary_desc* rotary, const void* q, const void* k, const int32_t* positions,
                  int32_t total, int64_t q_stride, int64_t k_stride, void* q_out, void* k_out, void* stream) {
    LayerParams lp;
    const int rc = make_layer(desc, &lp);
    if (rc) return rc;
    if (!rotary || !rotary_is_fine(rotary) || !positions || total <= 0 || (!q && !k) || !q != !q_out || !k != !k_out) return LSERVE_ERR_INVALID_ARG;
    if (rotary->rotary_dim > kHeadDim) return LSERVE_ERR_UNSUPPORTED;
    const int64_t q_row = (int64_t)lp.H * kHeadDim, k_row = (int64_t)lp.Hkv * kHeadDim;
    if (q && (q_stride < q_row || q_stride % 8 != 0 || (q_out == q && q_stride != q_row))) return LSERVE_ERR_INVALID_ARG;
    if (k && (k_stride < k_row || k_stride % 8 != 0 || (k_out == k && k_stride != k_row))) return LSERVE_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out) || !aligned16(positions)) return LSERVE_ERR_INVALID_ARG;
    // (outputs are whole, inputs rows that may lie apart; in place a row is read before it is written)
    const Rows q_in = {q, q_row * 2, q_stride * 2, total}, k_in = {k, k_row * 2, k_stride * 2, total};
    const Range q_to = {q_out, total * q_row * 2}, k_to = {k_out, total * k_row * 2}, at = {positions, total * 4LL},
                freq = {rotary->inv_freq, rotary->rotary_dim * 4LL};
    for (const Range& o : {q_to, k_to})
        if (meet(o, at) || meet(o, freq) || (o.at != q && meet(o, q_in)) || (o.at != k && meet(o, k_in))) return LSERVE_ERR_INVALID_ARG;
    if (meet(q_to, k_to) || (q_out && q_out == k) || (k_out && k_out == q)) return LSERVE_ERR_INVALID_ARG;
    RotaryArgs a = {};
    a.q = q;
    a.k = k;
    a.q_out = q_out;
    a.k_out = k_out;
    a.positions = positions;
    a.inv_freq = rotary->inv_freq;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.heads_q = q ? lp.H : 0;
    a.heads_k = k ? lp.Hkv : 0;
    a.total = total;
    a.rotary_dim = rotary->rotary_dim;
    a.interleaved = rotary->interleaved;
    a.scale = rotary->scale == 0.f ? 1.f : rotary->scale;
    const hipError_t e = launch_rotary(desc->dtype, a, (hipStream_t)stream);
    return e == hipSuccess ? LSERVE_OK : fail_hip(e);
}

int lserve_rotary_frequencies(const lserve_rotary_scaling* s, double* inv_freq, float* scale) {
    if (!s || !inv_freq || !scale || s->rotary_dim < 2 || s->rotary_dim % 2 != 0) return LSERVE_ERR_INVALID_ARG;
    if (s->rotary_dim > kHeadDim || s->kind < LSERVE_ROTARY_NONE || s->kind > LSERVE_ROTARY_RAMP) return LSERVE_ERR_UNSUPPORTED;
    const bool stretched = s->kind != LSERVE_ROTARY_NONE, by_turns = s->kind == LSERVE_ROTARY_WAVELENGTH || s->kind == LSERVE_ROTARY_RAMP;
    if (!(s->base > 1.0) || std::isinf(s->base)) return LSERVE_ERR_INVALID_ARG;
    if (stretched && (!(s->factor >= 1.0) || std::isinf(s->factor))) return LSERVE_ERR_INVALID_ARG;
    if (by_turns && (!(s->original_positions > 0.0) || std::isinf(s->original_positions) || !(s->low > 0.0) || !(s->high > s->low) ||
                     std::isinf(s->high)))
        return LSERVE_ERR_INVALID_ARG;
    const double kTurn = 6.283185307179586476925, R = s->rotary_dim;
    // index (not a whole number) of the pair that turns n times over the original positions
    auto index_of = [&](double n) { return R * std::log(s->original_positions / (n * kTurn)) / (2.0 * std::log(s->base)); };
    double first = 0.0, last = 0.0;
    if (s->kind == LSERVE_ROTARY_RAMP) {
        first = std::fmax(std::floor(index_of(s->high)), 0.0);
        last = std::fmin(std::ceil(index_of(s->low)), R - 1.0);
    }
    for (int i = 0; i < s->rotary_dim / 2; ++i) {
        const double f = std::pow(s->base, -2.0 * i / R);
        double kept = 1.0;  // share of the frequency as it is; the rest is f / factor
        if (s->kind == LSERVE_ROTARY_LINEAR) kept = 0.0;
        if (s->kind == LSERVE_ROTARY_WAVELENGTH) kept = (s->original_positions * f / kTurn - s->low) / (s->high - s->low);
        if (s->kind == LSERVE_ROTARY_RAMP) kept = 1.0 - (i - first) / std::fmax(last - first, 0.001);
        kept = std::fmin(std::fmax(kept, 0.0), 1.0);
        inv_freq[i] = kept == 1.0 ? f : f * kept + f / s->factor * (1.0 - kept);
    }
    *scale = s->kind == LSERVE_ROTARY_RAMP ? (float)(0.1 * std::log(s->factor) + 1.0) : 1.f;
    return LSERVE_OK;
}

int lserve_rotary_axes(const lserve_attn_desc* desc, const lserve_rotary_desc* rotary, const lserve_position_axes* axes, const void* q, const void* k,
                       const int32_t* positions, int64_t positions_stride, int32_t total, int64_t q_stride, int64_t k_stride, void* q_out,
                       void* k_out, void* stream) {
    LayerParams lp;
    int rc = make_layer(desc, &lp);
    if (rc) return rc;
    if (!rotary || !axes) return LSERVE_ERR_INVALID_ARG;
    TurnArgs turn = {};
    rc = make_turn(nullptr, rotary, axes, positions, positions_stride, total, false, &turn);
    return rc ? rc : turned_rows(desc, lp, turn, q, k, total, q_stride, k_stride, q_out, k_out, stream);
}

int lserve_norm_rotary(const lserve_attn_desc* desc, const lserve_head_norm* norm, const lserve_rotary_desc* rotary, const lserve_position_axes* axes,
                       const void* q, const void* k, const int32_t* positions, int64_t positions_stride, int32_t total, int64_t q_stride,
                       int64_t k_stride, void* q_out, void* k_out, void* stream) {
    LayerParams lp;
    int rc = make_layer(desc, &lp);
    if (rc) return rc;
    if (!norm) return LSERVE_ERR_INVALID_ARG;
    TurnArgs turn = {};
    rc = make_turn(norm, rotary, axes, positions, positions_stride, total, false, &turn);
    return rc ? rc : turned_rows(desc, lp, turn, q, k, total, q_stride, k_stride, q_out, k_out, stream);
}

int lserve_rotary_append_kv(const lserve_attn_desc* desc, const lserve_paged_kv* kv, const lserve_head_norm* norm, const lserve_rotary_desc* rotary,
                            const lserve_position_axes* axes, const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride,
                            int64_t v_stride, const int32_t* positions, int64_t positions_stride, const int32_t* cu_new, const int32_t* start_pos,
                            int32_t total_new, int32_t max_new_per_seq, void* q_out, void* k_out, void* v_out, void* stream) {
    TurnedAppendArgs a = {};
    int rc = make_layer(desc, &a.lp);
    if (rc) return rc;
    const int selecting = selecting_heads(a.lp).count;
    rc = make_paged(kv, a.lp, true, true, selecting > 0, true, &a.kv);
    if (rc) return rc;
    if (!k || !v || !q != !q_out || !cu_new || !start_pos || total_new <= 0 || max_new_per_seq <= 0) return LSERVE_ERR_INVALID_ARG;
    rc = make_turn(norm, rotary, axes, positions, positions_stride, total_new, true, &a.turn);
    if (rc) return rc;
    const int64_t q_row = (int64_t)a.lp.H * kHeadDim, k_row = (int64_t)a.lp.Hkv * kHeadDim;
    if ((q && !rows_are_fine(q, q_stride, q_row, q_out)) || !rows_are_fine(k, k_stride, k_row, k_out) || !rows_are_fine(v, v_stride, k_row, v_out))
        return LSERVE_ERR_INVALID_ARG;
    if (!aligned16(cu_new) || !aligned16(start_pos)) return LSERVE_ERR_INVALID_ARG;
    // what one workgroup writes others still read rows, places and tables for
    const long long batch = a.kv.batch, total = total_new, slab = 16LL * (long long)slab_chunks(a.lp.NP, a.kv.kv_bits);
    const Rows rows[] = {{q, q_row * 2, q_stride * 2, total}, {k, k_row * 2, k_stride * 2, total}, {v, k_row * 2, v_stride * 2, total}};
    const TurnRanges read(a.lp, a.turn, total_new);
    const Range in[] = {read.at[0], read.at[1], read.at[2], read.at[3], {cu_new, (batch + 1) * 4}, {start_pos, batch * 4},
                        {kv->page_table, batch * a.kv.max_pages * 4}, {a.kv.k_stream ? kv->ring_table : nullptr, batch * a.kv.ring * 4}};
    // (a layer whose heads are all in the bounded pool writes nothing of the main one)
    const bool main_used = !a.kv.k_stream || a.kv.stream_heads < a.lp.Hkv;
    const long long main = main_used ? (long long)a.kv.num_pages * a.kv.pool_heads : 0, bounded = (long long)kv->num_pages_stream * a.kv.stream_heads;
    const Range written[] = {{q_out, total * q_row * 2}, {k_out, total * k_row * 2}, {v_out, total * k_row * 2}, {kv->k_pool, main * slab},
                             {kv->v_pool, main * slab}, {a.kv.k_stream, bounded * slab}, {a.kv.v_stream, bounded * slab},
                             {selecting > 0 ? kv->stats : nullptr, main * a.lp.g * 4 * kHeadDim}};
    for (const Range& o : written) {
        if (!o.at) continue;
        for (const Range& i : in)
            if (meet(o, i)) return LSERVE_ERR_INVALID_ARG;
        for (const Rows& i : rows) {
            const bool in_place = o.at && o.at == i.at && ((&i == &rows[0] && &o == &written[0]) || (&i == &rows[1] && &o == &written[1]));
            if (!in_place && i.at && meet(o, i)) return LSERVE_ERR_INVALID_ARG;
        }
        for (const Range* other = &o + 1; other != std::end(written); ++other)
            if (meet(o, *other)) return LSERVE_ERR_INVALID_ARG;
    }
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_out = q_out;
    a.k_out = k_out;
    a.v_out = v_out;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.cu_new = cu_new;
    a.start_pos = start_pos;
    a.total = total_new;
    a.max_new = max_new_per_seq;
    const hipError_t e = launch_turned_append(desc->dtype, a, (hipStream_t)stream);
    return e == hipSuccess ? LSERVE_OK : fail_hip(e);
}

int lserve_tree_masks(const int32_t* parents, const int32_t* cu_new, const int32_t* seq_lens, int32_t batch, int32_t total_new,
                      int32_t max_new_per_seq, int32_t mask_words, uint64_t* tree_mask, int32_t* positions, void* stream) {
    if (!parents || !cu_new || !seq_lens || !tree_mask || !positions) return LSERVE_ERR_INVALID_ARG;
    if (batch <= 0 || total_new <= 0 || max_new_per_seq <= 0 || max_new_per_seq > total_new || mask_words < (max_new_per_seq + 63) / 64)
        return LSERVE_ERR_INVALID_ARG;
    if (batch > 65535 || max_new_per_seq > kMaxTreeNodes) return LSERVE_ERR_UNSUPPORTED;
    if (!aligned16(parents) || !aligned16(cu_new) || !aligned16(seq_lens) || !aligned16(tree_mask) || !aligned16(positions))
        return LSERVE_ERR_INVALID_ARG;
    // (positions may take the parents' place: a workgroup has read all of its own before it writes any)
    const Range in[] = {{positions == parents ? nullptr : parents, total_new * 4LL}, {cu_new, (batch + 1LL) * 4}, {seq_lens, batch * 4LL}};
    const Range mask = {tree_mask, (long long)total_new * mask_words * 8}, at = {positions, total_new * 4LL};
    for (const Range& i : in)
        if (meet(mask, i) || meet(at, i)) return LSERVE_ERR_INVALID_ARG;
    if (meet(mask, at)) return LSERVE_ERR_INVALID_ARG;
    const hipError_t e = launch_tree_masks(parents, cu_new, seq_lens, batch, total_new, max_new_per_seq, mask_words,
                                           (unsigned long long*)tree_mask, positions, (hipStream_t)stream);
    return e == hipSuccess ? LSERVE_OK : fail_hip(e);
}

int lserve_sparse_decode_tree(const lserve_attn_desc* desc, const lserve_paged_kv* kv, const void* q, const void* k_new, const void* v_new,
                              const int32_t* cu_new, const uint64_t* tree_mask, int32_t mask_words, const int32_t* positions,
                              const int32_t* sel_pages, const int32_t* sel_count, const int32_t* sel_seq_len, int32_t sel_stride,
                              int32_t total_new, int32_t max_new_per_seq, void* out, float* lse_out, void* workspace,
                              size_t workspace_bytes, void* stream) {
    TreeArgs a = {};
    int rc = make_layer(desc, &a.lp);
    if (rc) return rc;
    rc = make_paged(kv, a.lp, true, true, false, true, &a.kv);
    if (rc) return rc;
    if (a.lp.NP != 64) return LSERVE_ERR_UNSUPPORTED;
    if (!q || !k_new || !v_new || !cu_new || !out) return LSERVE_ERR_INVALID_ARG;
    if (total_new <= 0 || max_new_per_seq <= 0 || max_new_per_seq > total_new || !tree_mask != !positions) return LSERVE_ERR_INVALID_ARG;
    if (tree_mask && mask_words < (max_new_per_seq + 63) / 64) return LSERVE_ERR_INVALID_ARG;
    if (!sel_pages != !sel_count || !sel_pages != !sel_seq_len || (sel_pages ? sel_stride <= 0 : sel_stride != 0)) return LSERVE_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(cu_new) || !aligned16(tree_mask) || !aligned16(positions) ||
        !aligned16(sel_pages) || !aligned16(sel_count) || !aligned16(sel_seq_len) || !aligned16(out) || !aligned16(lse_out) ||
        !aligned16(workspace))
        return LSERVE_ERR_INVALID_ARG;
    if (max_new_per_seq > kMaxTreeNodes) return LSERVE_ERR_UNSUPPORTED;
    const size_t need = tree_workspace_bytes(a.lp, a.kv.batch, total_new, max_new_per_seq, a.kv.max_pages, sel_stride);
    if (need > 0 && (!workspace || workspace_bytes < need)) return LSERVE_ERR_WORKSPACE;
    // what one workgroup writes others still read their rows, keys and lists for
    const long long batch = a.kv.batch, total = total_new, row = 2LL * kHeadDim, lists = batch * a.lp.Hkv * 4;
    const Range in[] = {{q, total * a.lp.H * row}, {k_new, total * a.lp.Hkv * row}, {v_new, total * a.lp.Hkv * row}, {cu_new, (batch + 1) * 4},
                        {tree_mask, total * mask_words * 8}, {positions, total * 4}, {sel_pages, lists * sel_stride}, {sel_count, lists},
                        {sel_seq_len, batch * 4}, {kv->seq_lens, batch * 4}, {kv->page_table, batch * a.kv.max_pages * 4},
                        {a.kv.k_stream ? kv->ring_table : nullptr, batch * a.kv.ring * 4}};
    const Range written[] = {{out, total * a.lp.H * row}, {lse_out, total * a.lp.H * 4}, {workspace, (long long)need}};
    for (const Range& o : written) {
        for (const Range& i : in)
            if (meet(o, i)) return LSERVE_ERR_INVALID_ARG;
        for (const Range& other : written)
            if (&other != &o && meet(o, other)) return LSERVE_ERR_INVALID_ARG;
    }
    a.q = (const uint16_t*)q;
    a.k_new = (const uint16_t*)k_new;
    a.v_new = (const uint16_t*)v_new;
    a.cu_new = cu_new;
    a.positions = positions;
    a.tree_mask = (const unsigned long long*)tree_mask;
    a.sel_pages = sel_pages;
    a.sel_count = sel_count;
    a.sel_seq_len = sel_seq_len;
    a.mask_words = mask_words;
    a.sel_stride = sel_stride;
    a.total_new = total_new;
    a.max_new = max_new_per_seq;
    a.stream_pages = kv->num_pages_stream;
    a.out = (uint16_t*)out;
    a.lse_out = lse_out;
    const hipError_t e = launch_sparse_decode_tree(desc->dtype, a, workspace, (hipStream_t)stream);
    return e == hipSuccess ? LSERVE_OK : fail_hip(e);
}

size_t lserve_tree_workspace_bytes(const lserve_attn_desc* desc, int32_t batch, int32_t total_new, int32_t max_new_per_seq,
                                   int32_t max_pages_per_seq, int32_t sel_stride) {
    LayerParams lp;
    if (make_layer(desc, &lp) != LSERVE_OK || lp.NP != 64) return 0;
    if (batch <= 0 || batch > 65535 || total_new <= 0 || max_new_per_seq <= 0 || max_new_per_seq > total_new ||
        max_new_per_seq > kMaxTreeNodes || max_pages_per_seq <= 0 || sel_stride < 0)
        return 0;
    return tree_workspace_bytes(lp, batch, total_new, max_new_per_seq, max_pages_per_seq, sel_stride);
}

int lserve_probe_decode_read(const lserve_attn_desc* desc, const lserve_paged_kv* kv, const int32_t* sel_pages,
                             const int32_t* sel_count, const int32_t* sel_seq_len, int32_t sel_stride, void* stream) {
    LayerParams lp;
    PagedParams pp;
    int rc = make_layer(desc, &lp);
    if (rc) return rc;
    rc = make_paged(kv, lp, true, true, false, true, &pp);
    if (rc) return rc;
    const bool any_selecting = selecting_heads(lp).count > 0;
    if (any_selecting && (!sel_pages || !sel_count || !sel_seq_len || sel_stride <= 0)) return LSERVE_ERR_INVALID_ARG;
    if (sel_stride < 0 || !aligned16(sel_pages) || !aligned16(sel_count) || !aligned16(sel_seq_len)) return LSERVE_ERR_INVALID_ARG;
    if ((long long)pp.batch * lp.Hkv > 65535) return LSERVE_ERR_UNSUPPORTED;  // one grid row per (sequence, KV head)
    hipError_t e = launch_decode_read_probe(lp, pp, sel_pages, sel_count, sel_seq_len, sel_stride, (hipStream_t)stream);
    return e == hipSuccess ? LSERVE_OK : fail_hip(e);
}

size_t lserve_workspace_bytes(int which_call, const lserve_attn_desc* desc, int32_t batch, int32_t max_pages_per_seq,
                              int32_t sel_stride_or_budget_pages, int32_t total_tokens) {
    LayerParams lp;
    if (make_layer(desc, &lp) != LSERVE_OK) return 0;
    switch (which_call) {
        case LSERVE_CALL_SELECT_PAGES:
            return batch > 0 && max_pages_per_seq > 0 ? select_workspace_bytes(lp, batch, max_pages_per_seq) : 0;
        case LSERVE_CALL_SPARSE_PREFILL:
            return batch > 0 && total_tokens > 0 ? prefill_workspace_bytes(lp, total_tokens, batch) : 0;
        case LSERVE_CALL_SPARSE_DECODE:
            return batch > 0 && sel_stride_or_budget_pages >= 0
                       ? decode_workspace_bytes(lp, batch, sel_stride_or_budget_pages)
                       : 0;
        default:
            return 0;
    }
}

int lserve_init(void) {
    void* ws = nullptr;
    const int rc = scratch_on_current_device(&ws);
    if (rc) return rc;
    hipError_t e = preload_stats_kernels();
    if (e == hipSuccess) e = preload_select_kernels();
    if (e == hipSuccess) e = preload_prefill_kernels();
    if (e == hipSuccess) e = preload_decode_kernels();
    if (e == hipSuccess) e = preload_table_kernels();
    if (e == hipSuccess) e = preload_rotary_kernels();
    if (e == hipSuccess) e = preload_norm_rotary_kernels();
    if (e == hipSuccess) e = preload_rotary_append_kernels();
    if (e == hipSuccess) e = preload_tree_kernels();
    return e == hipSuccess ? LSERVE_OK : fail_hip(e);
}

const char* lserve_strerror(int code) {
    switch (code) {
        case LSERVE_OK:
            return "success";
        case LSERVE_ERR_INVALID_ARG:
            return "invalid argument (null or misaligned pointer, non-positive size, bad page sizes or budget)";
        case LSERVE_ERR_UNSUPPORTED:
            return "unsupported configuration (head_dim, dtype, head counts or page size)";
        case LSERVE_ERR_WORKSPACE:
            return "workspace missing or too small";
        case LSERVE_ERR_HIP:
            return "a HIP call failed (see lserve_last_hip_error)";
        default:
            return "unknown error code";
    }
}

int lserve_last_hip_error(void) { return g_last_hip_error; }

}  // extern "C"
