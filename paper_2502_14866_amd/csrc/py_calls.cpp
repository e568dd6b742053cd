// The calls of a decode step and those on new tokens, marshalled natively.  A step of a small batch is some ten microseconds of GPU work a call, and
// through ctypes a call was five microseconds of Python before its launch: the struct of the cache built field by field, an
// address and a check per tensor, twelve arguments converted.  Arguments are the binding's own objects; what is passed on
// is what ctypes passed on (see binding.py), and the return value is the library's.  The library is not linked: its entry points are
// handed over by address (bind), since the binding may load another build of it.
#include <torch/csrc/autograd/python_variable.h>

#include <c10/core/impl/VirtualGuardImpl.h>

#include <exception>
#include <initializer_list>

#include "../../include/lserve.h"

namespace {

decltype(&lserve_append_kv) append_kv;
decltype(&lserve_select_pages) select_pages;
decltype(&lserve_sparse_decode) sparse_decode;
decltype(&lserve_extend_tables) extend_tables;
decltype(&lserve_tree_masks) tree_masks;
decltype(&lserve_rotary) rotary;
decltype(&lserve_sparse_decode_tree) sparse_decode_tree;

struct PythonError {};  // the interpreter's error is set

const at::Tensor* tensor_or_null(PyObject* o) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "lserve binding takes tensors, not %.100s", Py_TYPE(o)->tp_name);
        throw PythonError();
    }
    return &THPVariable_Unpack(o);
}

template <class P = void> P* address(const at::Tensor* t) {
    if (!t) return nullptr;
    if (!t->is_contiguous()) {
        PyErr_SetString(PyExc_ValueError, "lserve binding takes contiguous tensors");
        throw PythonError();
    }
    return static_cast<P*>(t->data_ptr());
}
template <class P = void> P* address(PyObject* o) { return address<P>(tensor_or_null(o)); }

// What the library cannot see from an address: a tensor's type, how many elements of it are read or written, its device.
struct Wanted {
    const at::Tensor* t;
    at::ScalarType type;
    int64_t least;
};
[[noreturn]] void refuse(const char* where, const std::string& why) {
    PyErr_Format(PyExc_ValueError, "%s: %s", where, why.c_str());
    throw PythonError();
}
void check(const char* where, std::initializer_list<Wanted> wanted) {
    const at::Tensor* first = nullptr;
    for (const Wanted& w : wanted) {
        if (!w.t) continue;
        if (w.t->scalar_type() != w.type) refuse(where, std::string("a tensor of ") + c10::toString(w.t->scalar_type()) + " where " + c10::toString(w.type) + " is taken");
        if (w.t->numel() < w.least)
            refuse(where, "a tensor of " + std::to_string(w.t->numel()) + " elements where " + std::to_string(w.least) + " are read or written");
        if (first && w.t->device() != first->device()) refuse(where, "tensors on " + first->device().str() + " and " + w.t->device().str());
        if (!first) first = w.t;
    }
    if (first && first->device().is_cuda()) {
        const c10::Device now = c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice();
        if (first->device() != now) refuse(where, "tensors on " + first->device().str() + " while device " + now.str() + " is current");
    }
}
constexpr at::ScalarType kInt = at::kInt, kLong = at::kLong, kFloat = at::kFloat, kDouble = at::kDouble;
at::ScalarType type_of(const lserve_attn_desc* d) { return d->dtype == LSERVE_DTYPE_BF16 ? at::kBFloat16 : at::kHalf; }

// (the low bits, as ctypes takes them)
unsigned long long number(PyObject* o) {
    const unsigned long long x = PyLong_AsUnsignedLongLongMask(o);
    if (x == (unsigned long long)-1 && PyErr_Occurred()) throw PythonError();
    return x;
}
int32_t number32(PyObject* o) { return (int32_t)number(o); }

// A Python object's attribute, held while in use.
struct Attribute {
    PyObject* o;
    Attribute(PyObject* of, PyObject* name) : o(PyObject_GetAttr(of, name)) {
        if (!o) throw PythonError();
    }
    ~Attribute() { Py_DECREF(o); }
    Attribute(const Attribute&) = delete;
};

enum { kKPool, kVPool, kStats, kPageTable, kSeqLens, kPoolHeads, kKStream, kVStream, kRingTable, kBits, kNames };
PyObject* names[kNames];

// binding.PagedKV as lserve_paged_kv.  (The tensors stay alive: the caller holds the object.)
lserve_paged_kv paged(PyObject* kv) {
    const Attribute k(kv, names[kKPool]), v(kv, names[kVPool]), st(kv, names[kStats]), table(kv, names[kPageTable]), lens(kv, names[kSeqLens]),
        heads(kv, names[kPoolHeads]), ks(kv, names[kKStream]), vs(kv, names[kVStream]), ring(kv, names[kRingTable]), bits(kv, names[kBits]);
    const at::Tensor *kt = tensor_or_null(k.o), *vt = tensor_or_null(v.o), *stt = tensor_or_null(st.o), *tt = tensor_or_null(table.o),
                     *kst = tensor_or_null(ks.o);
    const at::Tensor* sized = stt ? stt : vt ? vt : kt;
    if (!tt) {
        PyErr_SetString(PyExc_TypeError, "PagedKV.page_table is None");
        throw PythonError();
    }
    lserve_paged_kv p = {};
    p.k_pool = address(kt);
    p.v_pool = address(vt);
    p.stats = address(stt);
    p.page_table = address<int32_t>(tt);
    p.seq_lens = address<int32_t>(lens.o);
    p.batch = (int32_t)tt->size(0);
    p.max_pages_per_seq = (int32_t)tt->size(1);
    p.num_pages = sized ? (int32_t)sized->size(0) : 0;
    p.pool_heads = number32(heads.o);
    p.k_pool_stream = address(kst);
    p.v_pool_stream = address(vs.o);
    p.ring_table = address<int32_t>(ring.o);
    p.num_pages_stream = kst ? (int32_t)kst->size(0) : 0;
    p.kv_bits = number32(bits.o);
    return p;
}

const lserve_attn_desc* description(PyObject* o) { return reinterpret_cast<const lserve_attn_desc*>((uintptr_t)number(o)); }
void* stream_handle(PyObject* o) { return reinterpret_cast<void*>((uintptr_t)number(o)); }

// Other threads may run while the library is at work (a launch waits where the queue is full).
struct WithoutLock {
    PyThreadState* state = PyEval_SaveThread();
    ~WithoutLock() { PyEval_RestoreThread(state); }
};

template <class F> PyObject* call(Py_ssize_t given, Py_ssize_t wanted, F f) {
    if (given != wanted) return PyErr_Format(PyExc_TypeError, "%zd arguments instead of %zd", given, wanted);
    try {
        const int rc = f();
        return PyLong_FromLong(rc);
    } catch (const PythonError&) {
        return nullptr;
    } catch (const std::exception& e) {
        return PyErr_Format(PyExc_RuntimeError, "%s", e.what());
    }
}

PyObject* py_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 8, [&] {
        const lserve_attn_desc* desc = description(a[0]);
        const lserve_paged_kv kv = paged(a[1]);
        const void *k = address(a[2]), *v = address(a[3]);
        const int32_t *cu = address<int32_t>(a[4]), *start = address<int32_t>(a[5]), longest = number32(a[6]);
        void* stream = stream_handle(a[7]);
        const WithoutLock w;
        return append_kv(desc, &kv, k, v, cu, start, longest, stream);
    });
}

PyObject* py_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 11, [&] {
        const lserve_attn_desc* desc = description(a[0]);
        const lserve_paged_kv kv = paged(a[1]);
        const at::Tensor* ws = tensor_or_null(a[9]);
        const void* q = address(a[2]);
        const int32_t budget = number32(a[3]), *valid = address<int32_t>(a[4]);
        int32_t *pages = address<int32_t>(a[5]), *count = address<int32_t>(a[6]), *len = address<int32_t>(a[7]);
        float* scores = address<float>(a[8]);
        void *workspace = address(ws), *stream = stream_handle(a[10]);
        const size_t bytes = ws ? ws->nbytes() : 0;
        const WithoutLock w;
        return select_pages(desc, &kv, q, budget, valid, pages, count, len, scores, workspace, bytes, stream);
    });
}

PyObject* py_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 10, [&] {
        const lserve_attn_desc* desc = description(a[0]);
        const lserve_paged_kv kv = paged(a[1]);
        const at::Tensor *sel = tensor_or_null(a[3]), *ws = tensor_or_null(a[8]);
        const void* q = address(a[2]);
        const int32_t *pages = address<int32_t>(sel), *count = address<int32_t>(a[4]), *len = address<int32_t>(a[5]);
        const int32_t stride = sel ? (int32_t)sel->size(-1) : 0;
        void *out = address(a[6]), *workspace = address(ws), *stream = stream_handle(a[9]);
        float* lse = address<float>(a[7]);
        const size_t bytes = ws ? ws->nbytes() : 0;
        const WithoutLock w;
        return sparse_decode(desc, &kv, q, pages, count, len, stride, out, lse, workspace, bytes, stream);
    });
}

struct Held {  // a tensor of a PagedKV that is checked
    Attribute o;
    const at::Tensor* t;
    Held(PyObject* kv, int name) : o(kv, names[name]), t(tensor_or_null(o.o)) {}
};

// Entries of a sequence in the ring table of the two-way cache.
int64_t ring_of(const lserve_attn_desc* d) {
    if (d->page_size <= 0) return 0;
    const int64_t page = d->page_size;
    return (d->sink_tokens + page - 1) / page + (d->local_tokens + page - 1) / page;
}

PyObject* py_extend(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 12, [&] {
        const char* where = "lserve_extend_tables";
        const lserve_attn_desc* desc = description(a[0]);
        const lserve_paged_kv kv = paged(a[1]);
        const Held table(a[1], kPageTable), now(a[1], kSeqLens), ring_table(a[1], kRingTable);
        const at::Tensor *fresh = tensor_or_null(a[2]), *pages = tensor_or_null(a[3]), *cu = tensor_or_null(a[4]), *lens = tensor_or_null(a[5]),
                         *taken = tensor_or_null(a[6]), *pos = tensor_or_null(a[7]), *slots = tensor_or_null(a[8]), *ring = tensor_or_null(a[9]);
        const int64_t batch = kv.batch, total = PyLong_AsLongLong(a[10]);
        if (total == -1 && PyErr_Occurred()) throw PythonError();
        check(where, {{table.t, kInt, 0}, {now.t, kInt, batch}, {ring_table.t, kInt, 0}, {fresh, kInt, batch}, {pages, kInt, 0},
                      {cu, kInt, batch + 1}, {lens, kInt, batch}, {taken, kInt, 1}, {pos, kInt, total}, {slots, kLong, total}, {ring, kLong, total}});
        if (ring && ring_table.t && ring_table.t->numel() < batch * ring_of(desc))
            refuse(where, "a ring table of " + std::to_string(ring_table.t->numel()) + " entries for " + std::to_string(batch) + " sequences of " +
                              std::to_string(ring_of(desc)));
        const int32_t* p_fresh = address<int32_t>(fresh);
        const int32_t *p_pages = address<int32_t>(pages), num_free = pages ? (int32_t)pages->numel() : 0;
        int32_t *p_cu = address<int32_t>(cu), *p_lens = address<int32_t>(lens), *p_taken = address<int32_t>(taken), *p_pos = address<int32_t>(pos);
        int64_t *p_slots = address<int64_t>(slots), *p_ring = address<int64_t>(ring);
        void* stream = stream_handle(a[11]);
        const WithoutLock w;
        return extend_tables(desc, &kv, p_fresh, p_pages, num_free, (int32_t)total, p_cu, p_lens, p_taken, p_pos, p_slots, p_ring, stream);
    });
}

PyObject* py_masks(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 7, [&] {
        const at::Tensor *parents = tensor_or_null(a[0]), *cu = tensor_or_null(a[1]), *lens = tensor_or_null(a[2]), *mask = tensor_or_null(a[4]),
                         *pos = tensor_or_null(a[5]);
        const int64_t total = parents ? parents->numel() : 0, batch = cu ? cu->numel() - 1 : 0, words = mask && mask->dim() ? mask->size(-1) : 0;
        check("lserve_tree_masks", {{parents, kInt, 1}, {cu, kInt, 2}, {lens, kInt, batch}, {mask, kLong, total * words}, {pos, kInt, total}});
        const int32_t *p_parents = address<int32_t>(parents), *p_cu = address<int32_t>(cu), *p_lens = address<int32_t>(lens), longest = number32(a[3]);
        uint64_t* p_mask = address<uint64_t>(mask);
        int32_t* p_pos = address<int32_t>(pos);
        void* stream = stream_handle(a[6]);
        const WithoutLock w;
        return tree_masks(p_parents, p_cu, p_lens, (int32_t)batch, (int32_t)total, longest, (int32_t)words, p_mask, p_pos, stream);
    });
}

// Address of [total][heads][dim] whose rows may lie apart, and how far.
const void* rows(const at::Tensor* t, int64_t heads, int64_t dim, const char* what, int64_t* stride) {
    *stride = 0;
    if (!t) return nullptr;
    if (t->dim() != 3 || t->size(1) != heads || t->size(2) != dim || t->stride(2) != 1 || t->stride(1) != dim)
        refuse("lserve_rotary", std::string(what) + " is [total][" + std::to_string(heads) + "][" + std::to_string(dim) + "], heads next to each other");
    *stride = t->size(0) > 1 ? t->stride(0) : heads * dim;
    return t->data_ptr();
}

PyObject* py_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 9, [&] {
        const lserve_attn_desc* desc = description(a[0]);
        const lserve_rotary_desc* rot = reinterpret_cast<const lserve_rotary_desc*>((uintptr_t)number(a[1]));
        const at::Tensor *freq = tensor_or_null(a[2]), *q = tensor_or_null(a[3]), *k = tensor_or_null(a[4]), *pos = tensor_or_null(a[5]),
                         *qo = tensor_or_null(a[6]), *ko = tensor_or_null(a[7]);
        const int64_t dim = desc->head_dim, hq = desc->num_q_heads, hkv = desc->num_kv_heads, total = pos ? pos->numel() : 0;
        int64_t q_stride, k_stride;
        const void *p_q = rows(q, hq, dim, "q", &q_stride), *p_k = rows(k, hkv, dim, "k", &k_stride);
        const at::ScalarType t = type_of(desc);
        check("lserve_rotary", {{pos, kInt, 1}, {freq, kDouble, rot->rotary_dim <= dim ? rot->rotary_dim / 2 : 0}, {q, t, total * hq * dim}, {qo, t, total * hq * dim},
                                {k, t, total * hkv * dim}, {ko, t, total * hkv * dim}});
        const int32_t* p_pos = address<int32_t>(pos);
        void *p_qo = address(qo), *p_ko = address(ko), *stream = stream_handle(a[8]);
        const WithoutLock w;
        return rotary(desc, rot, p_q, p_k, p_pos, (int32_t)total, q_stride, k_stride, p_qo, p_ko, stream);
    });
}

PyObject* py_tree(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 16, [&] {
        const char* where = "lserve_sparse_decode_tree";
        const lserve_attn_desc* desc = description(a[0]);
        const lserve_paged_kv kv = paged(a[1]);
        const Held table(a[1], kPageTable), now(a[1], kSeqLens), ring_table(a[1], kRingTable), k_pool(a[1], kKPool), v_pool(a[1], kVPool),
            k_stream(a[1], kKStream), v_stream(a[1], kVStream);
        const at::Tensor *q = tensor_or_null(a[2]), *k = tensor_or_null(a[3]), *v = tensor_or_null(a[4]), *cu = tensor_or_null(a[5]),
                         *out = tensor_or_null(a[7]), *lse = tensor_or_null(a[8]), *mask = tensor_or_null(a[9]), *pos = tensor_or_null(a[10]),
                         *sel = tensor_or_null(a[11]), *count = tensor_or_null(a[12]), *len = tensor_or_null(a[13]), *ws = tensor_or_null(a[14]);
        const int64_t dim = desc->head_dim, hq = desc->num_q_heads, hkv = desc->num_kv_heads, batch = kv.batch, total = q && q->dim() ? q->size(0) : 0;
        const int64_t words = mask && mask->dim() ? mask->size(-1) : 0, stride = sel && sel->dim() ? sel->size(-1) : 0;
        const at::ScalarType t = type_of(desc);
        // of one head's rows in a page; a number of bits that is neither is the library's to refuse
        const bool rows16 = kv.kv_bits == 0 || kv.kv_bits == 16, codes = kv.kv_bits == 8 || kv.kv_bits == 4;
        const int64_t slab = rows16 ? desc->page_size * dim : codes ? 8 * dim * kv.kv_bits + 256 : 0;
        auto kind = [&](const Held& pool) { return rows16 ? t : codes || (pool.t && pool.t->scalar_type() == at::kByte) ? at::kByte : t; };
        int64_t streams = 0;
        for (int64_t h = 0; k_stream.t && h < hkv; ++h) streams += desc->kv_head_is_streaming[h] != 0;
        // (a layer whose heads are all in the bounded pool reads nothing of the main one)
        const int64_t pool = streams < hkv ? kv.num_pages * (kv.pool_heads ? kv.pool_heads : hkv) * slab : 0, bounded = kv.num_pages_stream * streams * slab;
        check(where, {{q, t, total * hq * dim}, {k, t, total * hkv * dim}, {v, t, total * hkv * dim}, {out, t, total * hq * dim}, {lse, kFloat, total * hq},
                      {cu, kInt, batch + 1}, {now.t, kInt, batch}, {table.t, kInt, 0}, {k_pool.t, kind(k_pool), pool}, {v_pool.t, kind(v_pool), pool},
                      {k_stream.t, kind(k_stream), bounded}, {v_stream.t, kind(v_stream), bounded},
                      {ring_table.t, kInt, k_stream.t ? batch * ring_of(desc) : 0}, {mask, kLong, total * words},
                      {pos, kInt, total}, {sel, kInt, batch * hkv * stride}, {count, kInt, batch * hkv}, {len, kInt, batch}, {ws, ws ? ws->scalar_type() : t, 0}});
        const void *p_q = address(q), *p_k = address(k), *p_v = address(v);
        const int32_t *p_cu = address<int32_t>(cu), longest = number32(a[6]), *p_pos = address<int32_t>(pos), *p_sel = address<int32_t>(sel),
                      *p_count = address<int32_t>(count), *p_len = address<int32_t>(len);
        const uint64_t* p_mask = address<uint64_t>(mask);
        void *p_out = address(out), *p_ws = address(ws), *stream = stream_handle(a[15]);
        float* p_lse = address<float>(lse);
        const size_t bytes = ws ? ws->nbytes() : 0;
        const WithoutLock w;
        return sparse_decode_tree(desc, &kv, p_q, p_k, p_v, p_cu, p_mask, (int32_t)words, p_pos, p_sel, p_count, p_len, (int32_t)stride, (int32_t)total,
                                  longest, p_out, p_lse, p_ws, bytes, stream);
    });
}

PyObject* py_bind_new(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 4, [&] {
        extend_tables = reinterpret_cast<decltype(extend_tables)>((uintptr_t)number(a[0]));
        tree_masks = reinterpret_cast<decltype(tree_masks)>((uintptr_t)number(a[1]));
        rotary = reinterpret_cast<decltype(rotary)>((uintptr_t)number(a[2]));
        sparse_decode_tree = reinterpret_cast<decltype(sparse_decode_tree)>((uintptr_t)number(a[3]));
        return 0;
    });
}

PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 3, [&] {
        append_kv = reinterpret_cast<decltype(append_kv)>((uintptr_t)number(a[0]));
        select_pages = reinterpret_cast<decltype(select_pages)>((uintptr_t)number(a[1]));
        sparse_decode = reinterpret_cast<decltype(sparse_decode)>((uintptr_t)number(a[2]));
        return 0;
    });
}

#define LSERVE_FASTCALL(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL
PyMethodDef methods[] = {
    {"bind", LSERVE_FASTCALL(py_bind), "addresses of lserve_append_kv, lserve_select_pages, lserve_sparse_decode"},
    {"append", LSERVE_FASTCALL(py_append), "desc address, kv, k_new, v_new, cu_new, start_pos, max_new_per_seq, stream"},
    {"select", LSERVE_FASTCALL(py_select),
     "desc address, kv, q, budget_tokens, stats_valid_len, sel_pages, sel_count, sel_seq_len, scores_out, workspace, stream"},
    {"decode", LSERVE_FASTCALL(py_decode), "desc address, kv, q, sel_pages, sel_count, sel_seq_len, out, lse_out, workspace, stream"},
    {"bind_new", LSERVE_FASTCALL(py_bind_new), "addresses of lserve_extend_tables, lserve_tree_masks, lserve_rotary, lserve_sparse_decode_tree"},
    {"extend", LSERVE_FASTCALL(py_extend),
     "desc address, kv, new_lens, free_pages, cu_new, new_seq_lens, pages_taken, positions, slots, ring_slots, total_new, stream"},
    {"masks", LSERVE_FASTCALL(py_masks), "parents, cu_new, seq_lens, max_new_per_seq, tree_mask, positions, stream"},
    {"rotary", LSERVE_FASTCALL(py_rotary), "desc address, rotary address, inv_freq, q, k, positions, q_out, k_out, stream"},
    {"tree", LSERVE_FASTCALL(py_tree),
     "desc address, kv, q, k_new, v_new, cu_new, max_new_per_seq, out, lse_out, tree_mask, positions, sel_pages, sel_count, sel_seq_len, workspace, stream"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "native marshalling of the calls of a decode step and on new tokens", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
    constexpr const char* spelled[kNames] = {"k_pool", "v_pool", "stats", "page_table", "seq_lens",
                                             "pool_heads", "k_pool_stream", "v_pool_stream", "ring_table", "kv_bits"};
    for (int i = 0; i < kNames; ++i)
        if (!(names[i] = PyUnicode_InternFromString(spelled[i]))) return nullptr;
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", LSERVE_TORCH) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
