// The per-call work of binding.py's draft and verify functions in native code: looking the tensors over,
// filling the C structures, allocating the outputs and making the call.  In Python these cost more than
// the kernels of a small batch (config 1, 4096 trees: spechub_draft and spechub_verify 37 us of host time a
// pair for 12 us of kernels; here 15).
//
// kv_append(), tree_attention() and kv_commit() do the same for the key-value cache (a call of Python and ctypes takes 14 to
// 20 us, as long as the kernels of a serving batch; here 5).
//
// They take what the Python functions were given and return the outputs, or an MDSD_E_*
// code (a negative int) for the caller to raise, or None for anything out of the ordinary (a tensor
// subclass, a wrong shape, type or layout): the caller then goes its own way, which raises the error.
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <utility>

#include "mdsd.h"

namespace {

// what a call is about, from the first arguments of draft() and verify()
struct Rows {
    mdsd_problem pb;
    int64_t B, N, V;
    at::Tensor draft;
};

const at::Tensor* tensor_of(PyObject* o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

bool is_rows(const at::Tensor& t)
{
    return t.is_cuda() && t.dim() == 3 && t.stride(2) == 1 && t.stride(0) == t.size(1) * t.stride(1) &&
           (t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16);
}

// a contiguous device tensor of this type and shape
const at::Tensor* plain(PyObject* o, at::ScalarType type, at::IntArrayRef shape)
{
    const at::Tensor* t = tensor_of(o);
    return t && t->is_cuda() && t->scalar_type() == type && t->is_contiguous() && t->sizes() == shape ? t : nullptr;
}

bool number(PyObject* o, int32_t& v)
{
    if (!PyLong_CheckExact(o)) return false;
    const long l = PyLong_AsLong(o);
    if ((l == -1 && PyErr_Occurred()) || l != (int32_t)l) {
        PyErr_Clear();
        return false;
    }
    v = (int32_t)l;
    return true;
}
bool number(PyObject* o, float& v)
{
    if (!PyFloat_CheckExact(o)) return false;  // (an integer temperature goes the other way)
    v = (float)PyFloat_AS_DOUBLE(o);
    return true;
}

// args: target or None, draft, kind, k, depth, temp_target, temp_draft, first_child or None, draft_stats or None
constexpr int kRowArgs = 9;
bool rows_of(PyObject* const* a, Rows& r)
{
    mdsd_problem& p = r.pb;
    p = mdsd_problem{};
    const at::Tensor* draft = tensor_of(a[1]);
    if (!draft || !is_rows(*draft)) return false;
    r.draft = *draft;
    r.B = draft->size(0);
    r.N = draft->size(1);
    r.V = draft->size(2);
    if (r.B > INT32_MAX || r.N > INT32_MAX || r.V > INT32_MAX) return false;
    p.ld_t = draft->stride(1);
    if (a[0] != Py_None) {
        const at::Tensor* target = tensor_of(a[0]);
        if (!target || !is_rows(*target) || target->sizes() != draft->sizes() ||
            target->scalar_type() != draft->scalar_type())
            return false;
        p.target = target->data_ptr();
        p.ld_t = target->stride(1);
    }
    p.draft = draft->data_ptr();
    p.ld_d = draft->stride(1);
    p.dtype = draft->scalar_type() == at::kFloat ? MDSD_FP32 : MDSD_BF16;
    p.B = (int32_t)r.B;
    p.N = (int32_t)r.N;
    p.V = (int32_t)r.V;
    if (!number(a[2], p.kind) || !number(a[3], p.k) || !number(a[4], p.depth) || !number(a[5], p.temp_target) ||
        !number(a[6], p.temp_draft))
        return false;
    if (a[7] != Py_None) {
        const at::Tensor* t = plain(a[7], at::kInt, {r.N});
        if (!t) return false;
        p.first_child = (const int32_t*)t->data_ptr();
    }
    if (a[8] != Py_None) {
        const at::Tensor* t = plain(a[8], at::kFloat, {r.B, r.N, 4});
        if (!t) return false;
        p.draft_stats = (mdsd_row_stats*)t->data_ptr();
    }
    return true;
}

bool stream_of(PyObject* o, void*& stream)
{
    stream = PyLong_AsVoidPtr(o);
    if (!PyErr_Occurred()) return true;
    PyErr_Clear();
    return false;
}

// the outputs of a call; given up with everything in it wherever the call does not come to its end
struct Outputs {
    PyObject* dict = PyDict_New();
    Outputs()
    {
        if (!dict) throw std::bad_alloc();
    }
    Outputs(const Outputs&) = delete;
    ~Outputs() { Py_XDECREF(dict); }

    // a new output under `name`; its data pointer
    void* add(const char* name, at::IntArrayRef shape, const at::TensorOptions& options)
    {
        at::Tensor t = at::empty(shape, options);
        void* data = t.data_ptr();
        PyObject* o = THPVariable_Wrap(std::move(t));
        const bool ok = o && PyDict_SetItemString(dict, name, o) == 0;
        Py_XDECREF(o);
        if (!ok) throw std::bad_alloc();
        return data;
    }
    // what a call that the library answered with `rc` returns
    PyObject* answer(int rc)
    {
        return rc == MDSD_OK ? std::exchange(dict, nullptr) : PyLong_FromLong(rc);
    }
};

template <class F>
PyObject* guarded(F f)
{
    try {
        return f();
    } catch (const std::exception&) {  // an allocation that failed: torch reports it on the other way
        if (PyErr_Occurred()) return nullptr;
        Py_RETURN_NONE;
    }
}

// draft(method, stream, <rows>, u)
PyObject* draft(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        int32_t method;
        void* stream;
        Rows r;
        if (n != 2 + kRowArgs + 1 || !number(a[0], method) || !stream_of(a[1], stream) || !rows_of(a + 2, r))
            Py_RETURN_NONE;
        const at::Tensor* u = plain(a[2 + kRowArgs], at::kFloat, {r.B, r.N, r.pb.k});
        if (!u) Py_RETURN_NONE;
        Outputs out;
        const at::TensorOptions ints = r.draft.options().dtype(at::kInt);
        int32_t* tokens = (int32_t*)out.add("tokens", {r.B, r.N}, ints);
        int32_t* flags = (int32_t*)out.add("flags", {r.B, r.N}, ints);
        int32_t* hub = method == 0 ? (int32_t*)out.add("hub", {r.B, r.N}, ints) : nullptr;
        const float* up = (const float*)u->data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS;
        rc = method == 0   ? spechub_draft(&r.pb, up, tokens, hub, flags, nullptr, 0, stream)
             : method == 1 ? rrs_draft(&r.pb, up, tokens, flags, nullptr, 0, stream)
                           : rrsw_draft(&r.pb, up, tokens, flags, nullptr, 0, stream);
        Py_END_ALLOW_THREADS;
        return out.answer(rc);
    });
}

// verify(method, stream, <rows>, tokens, u, resid_mass, flags, resid_prob, walk)
PyObject* verify(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        int32_t method;
        void* stream;
        Rows r;
        if (n != 2 + kRowArgs + 6 || !number(a[0], method) || !stream_of(a[1], stream) || a[2] == Py_None ||
            !rows_of(a + 2, r))
            Py_RETURN_NONE;
        a += 2 + kRowArgs;
        const at::Tensor *tokens = plain(a[0], at::kInt, {r.B, r.N}),
                         *u = plain(a[1], at::kFloat, {r.B, r.N, (int64_t)r.pb.k + 1});
        if (!tokens || !u || r.pb.depth < 0) Py_RETURN_NONE;
        for (int i = 2; i < 6; ++i)
            if (!PyBool_Check(a[i])) Py_RETURN_NONE;
        Outputs out;
        mdsd_result res = {};
        const at::TensorOptions ints = r.draft.options().dtype(at::kInt), floats = ints.dtype(at::kFloat);
        res.outcome = (int32_t*)out.add("outcome", {r.B, r.N}, ints);
        res.token = (int32_t*)out.add("token", {r.B, r.N}, ints);
        if (a[2] == Py_True) res.resid_mass = (float*)out.add("resid_mass", {r.B, r.N}, floats);
        if (a[3] == Py_True) res.flags = (int32_t*)out.add("flags", {r.B, r.N}, ints);
        if (a[4] == Py_True) res.resid_prob = (float*)out.add("resid_prob", {r.B, r.N, r.V}, floats);
        if (a[5] == Py_True) {
            res.accept_depth = (int32_t*)out.add("accept_depth", {r.B}, ints);
            res.emitted = (int32_t*)out.add("emitted", {r.B, r.pb.depth}, ints);
        }
        const int32_t* tp = (const int32_t*)tokens->data_ptr();
        const float* up = (const float*)u->data_ptr();
        decltype(&spechub_verify) call[] = {spechub_verify,      rrs_verify,      rrsw_verify,
                                            spechub_verify_path, rrs_verify_path, rrsw_verify_path};
        if (method < 0 || method > 5) Py_RETURN_NONE;
        int rc;
        Py_BEGIN_ALLOW_THREADS;
        rc = call[method](&r.pb, tp, up, &res, nullptr, 0, stream);
        Py_END_ALLOW_THREADS;
        return out.answer(rc);
    });
}

// ---------------------------------------------------------------- the key-value cache
// what a cache call is about: device, cache (k, v, table, lengths, k_scales or None, v_scales or None), tree (k, depth, first_child or
// None, counts or None)
constexpr int kCacheArgs = 11, kPagesArgs = 7;  // without a tree
struct CacheCall {
    mdsd_kv_cache c;
    mdsd_tree t;
    mdsd_kv_scales s;
    bool four;  // in 4 bits
    const at::Tensor* k;
    at::ScalarType type;  // of vectors; of a cache in 4 bits, as the first of them has it
    int64_t B;
    int32_t device;

    bool here(const at::Tensor& x) const { return x.is_cuda() && x.device().index() == device; }
    // a contiguous tensor of this type and shape on the call's device, or None: nullptr; `ok` says whether it is either
    void* optional(PyObject* o, at::ScalarType type, at::IntArrayRef shape, bool& ok) const
    {
        if (o == Py_None) return nullptr;
        const at::Tensor* x = plain(o, type, shape);
        if (!x || !here(*x)) ok = false;
        return ok ? x->data_ptr() : nullptr;
    }
    static int32_t dtype_of(at::ScalarType x) { return x == at::kFloat ? MDSD_FP32 : x == at::kBFloat16 ? MDSD_BF16 : MDSD_FP16; }
    const mdsd_kv_scales* scales() const { return four ? &s : nullptr; }
    // a stride, 0 where there is one element, whose stride may be anything
    static int64_t ld(const at::Tensor& x, int axis) { return x.size(axis) == 1 ? 0 : x.stride(axis); }

    bool cache_of(PyObject* const* a)
    {
        c = mdsd_kv_cache{};
        if (!number(a[0], device)) return false;
        k = tensor_of(a[1]);
        const at::Tensor *v = tensor_of(a[2]), *table = tensor_of(a[3]);
        if (!k || !v || !table || !here(*k) || !here(*v) || !here(*table)) return false;
        const auto held = k->scalar_type();
        four = a[5] != Py_None;
        if (k->dim() != 5 || v->dim() != 5 || k->stride(4) != 1 || v->stride(4) != 1 || v->scalar_type() != held || k->sizes() != v->sizes()) return false;
        if (four != (a[6] != Py_None) || (four ? held != at::kByte : held != at::kFloat && held != at::kBFloat16 && held != at::kHalf))
            return false;
        type = held;
        for (int i = 0; i < 4; ++i)
            if (ld(*k, i) != ld(*v, i)) return false;
        for (int i = 0; i < 5; ++i)
            if (k->size(i) > INT32_MAX) return false;
        if (four) {
            const at::Tensor *ks = tensor_of(a[5]), *vs = tensor_of(a[6]);
            if (!ks || !vs || !here(*ks) || !here(*vs) || ks->scalar_type() != at::kByte || vs->scalar_type() != at::kByte || ks->dim() != 5 ||
                vs->dim() != 5 || ks->sizes() != vs->sizes() || k->size(4) % 16 || ks->size(4) * 16 != k->size(4) || k->size(4) > MDSD_MAX_DIM)
                return false;
            for (int i = 0; i < 4; ++i)
                if (ks->size(i) != k->size(i) || 16 * ld(*ks, i) != ld(*k, i) || ld(*vs, i) != ld(*ks, i)) return false;
            if (ks->size(4) != 1 && (ks->stride(4) != 1 || vs->stride(4) != 1)) return false;
            s = mdsd_kv_scales{ks->data_ptr(), vs->data_ptr(), MDSD_BF16};
        }
        if (table->dim() != 2 || table->scalar_type() != at::kInt || table->stride(1) != 1 || table->size(0) > INT32_MAX ||
            table->size(1) > INT32_MAX)
            return false;
        B = table->size(0);
        const at::Tensor* lengths = plain(a[4], at::kInt, {B});
        if (!lengths || !here(*lengths)) return false;
        c.k = k->data_ptr();
        c.v = v->data_ptr();
        const int each = four ? 2 : 1;  // elements
        c.ld_layer = each * ld(*k, 0);
        c.ld_page = each * ld(*k, 1);
        c.ld_slot = each * ld(*k, 2);
        c.ld_head = each * ld(*k, 3);
        c.dtype = four ? MDSD_FP4 : dtype_of(held);
        c.layers = (int32_t)k->size(0);
        c.pages = (int32_t)k->size(1);
        c.page_size = (int32_t)k->size(2);
        c.heads = (int32_t)k->size(3);
        c.dim = each * (int32_t)k->size(4);
        c.table_pages = (int32_t)table->size(1);
        c.table = (const int32_t*)table->data_ptr();
        c.ld_table = B > 1 ? table->stride(0) : table->size(1);
        c.lengths = (const int32_t*)lengths->data_ptr();
        return true;
    }
    bool tree_of(PyObject* const* a, int64_t N)
    {
        t = mdsd_tree{};
        bool ok = N <= INT32_MAX && number(a[7], t.k) && number(a[8], t.depth);
        t.B = (int32_t)B;
        t.N = (int32_t)N;
        t.first_child = ok ? (const int32_t*)optional(a[9], at::kInt, {N}, ok) : nullptr;
        t.counts = ok ? (const int32_t*)optional(a[10], at::kInt, {B}, ok) : nullptr;
        return ok;
    }
    // vectors [B, N, heads, dim]; N = -1: not known yet
    bool heads_of(const at::Tensor* x, mdsd_heads& h, int64_t& N)
    {
        if (four && x && type == at::kByte) {  // the first vector
            type = x->scalar_type();
            if (type != at::kFloat && type != at::kBFloat16 && type != at::kHalf) return false;
            s.dtype = dtype_of(type);
        }
        if (!x || !here(*x) || x->dim() != 4 || x->stride(3) != 1 || x->scalar_type() != type || x->size(0) != B ||
            x->size(3) != c.dim || x->size(2) > INT32_MAX || (N >= 0 && x->size(1) != N))
            return false;
        N = x->size(1);
        h.p = x->data_ptr();
        h.ld_tree = ld(*x, 0);
        h.ld_node = ld(*x, 1);
        h.ld_head = ld(*x, 2);
        h.heads = (int32_t)x->size(2);
        return true;
    }
};

PyObject* answer(int rc, PyObject* given, at::Tensor made)
{
    if (rc != MDSD_OK) return PyLong_FromLong(rc);
    if (made.defined()) return THPVariable_Wrap(std::move(made));
    Py_INCREF(given);
    return given;
}

// kv_append(stream, <cache and tree>, k, v, q or None, inv_freq or None, layer, neighbours, out or None, flags or None, positions or
// None, axis_of or None, k_out or None, v_out or None):
// the turned queries, False without any
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        void* stream;
        CacheCall call;
        if (n != 1 + kCacheArgs + 12 || !stream_of(a[0], stream) || !call.cache_of(a + 1)) Py_RETURN_NONE;
        PyObject* const* const b = a + 1 + kCacheArgs;
        mdsd_heads k, v, q, q_out;
        int64_t N = -1;
        int32_t layer;
        if (!call.heads_of(tensor_of(b[0]), k, N) || !call.heads_of(tensor_of(b[1]), v, N) || !call.tree_of(a + 1, N) ||
            !number(b[4], layer) || !PyBool_Check(b[5]))
            Py_RETURN_NONE;
        const at::Tensor* inv_freq = nullptr;
        if (b[3] != Py_None && (!(inv_freq = tensor_of(b[3])) || !plain(b[3], at::kFloat, {inv_freq->numel()}) ||
                                !call.here(*inv_freq) || inv_freq->numel() > MDSD_MAX_DIM))
            Py_RETURN_NONE;
        bool ok = true;
        int32_t* flags = (int32_t*)call.optional(b[7], at::kInt, {call.B}, ok);
        at::Tensor made;
        if (b[2] != Py_None) {
            const at::Tensor* from = tensor_of(b[2]);
            if (!ok || !call.heads_of(from, q, N)) Py_RETURN_NONE;
            if (b[6] == Py_None) made = call.t.counts ? at::zeros_like(*from) : at::empty_like(*from);
            if (!call.heads_of(b[6] == Py_None ? &made : tensor_of(b[6]), q_out, N)) Py_RETURN_NONE;
        }
        if (!ok) Py_RETURN_NONE;
        const bool queries = b[2] != Py_None;
        mdsd_rotary r = {};
        r.inv_freq = inv_freq ? (const float*)inv_freq->data_ptr() : nullptr;
        r.rot = inv_freq ? 2 * (int32_t)inv_freq->numel() : 0;
        r.style = b[5] == Py_True ? MDSD_ROTATE_NEIGHBOURS : MDSD_ROTATE_HALVES;
        if (b[8] != Py_None) {
            const at::Tensor* x = tensor_of(b[8]);
            if (!x || x->scalar_type() != at::kInt || !x->is_contiguous() || !call.here(*x) || (x->dim() != 2 && x->dim() != 3) ||
                x->size(0) > INT32_MAX || x->size(1) != call.B || (x->dim() == 3 && x->size(2) != N))
                Py_RETURN_NONE;
            r.positions = (const int32_t*)x->data_ptr();
            r.axes = (int32_t)x->size(0);
            r.per_node = x->dim() == 3;
            r.ld_tree = r.per_node ? N : 1;
            r.ld_axis = call.B * r.ld_tree;
        }
        if (b[9] != Py_None) {
            if (!r.positions) Py_RETURN_NONE;
            r.axis_of = (const uint8_t*)call.optional(b[9], at::kByte, {r.rot / 2}, ok);
        }
        mdsd_heads k_out, v_out;
        if ((b[10] != Py_None && !call.heads_of(tensor_of(b[10]), k_out, N)) || (b[11] != Py_None && !call.heads_of(tensor_of(b[11]), v_out, N)) || !ok)
            Py_RETURN_NONE;
        int rc;
        Py_BEGIN_ALLOW_THREADS;
        rc = mdsd_kv_append_at(&call.c, call.scales(), layer, &call.t, &k, &v, queries ? &q : nullptr, queries ? &q_out : nullptr, &r,
                               b[10] != Py_None ? &k_out : nullptr, b[11] != Py_None ? &v_out : nullptr, flags, stream);
        Py_END_ALLOW_THREADS;
        return answer(rc, queries ? b[6] : Py_False, std::move(made));
    });
}

// tree_attention(stream, <cache and tree>, q, layer, scale or None, shared, shared_pages or None, longest, out or None,
// flags or None, workspace or None, lse or None): the results
PyObject* tree_attention(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        void* stream;
        CacheCall call;
        if (n != 1 + kCacheArgs + 10 || !stream_of(a[0], stream) || !call.cache_of(a + 1)) Py_RETURN_NONE;
        PyObject* const* const b = a + 1 + kCacheArgs;
        mdsd_heads q, out;
        int64_t N = -1;
        int32_t layer, shared, longest;
        float scale;
        const at::Tensor* from = tensor_of(b[0]);
        if (!call.heads_of(from, q, N) || !call.tree_of(a + 1, N) || !number(b[1], layer) || !number(b[3], shared) || !number(b[5], longest))
            Py_RETURN_NONE;
        if (b[2] == Py_None)
            scale = (float)(1.0 / std::sqrt((double)call.c.dim));
        else if (!number(b[2], scale))
            Py_RETURN_NONE;
        const int32_t* pages = nullptr;
        if (b[4] != Py_None) {
            const at::Tensor* x = tensor_of(b[4]);
            if (!x || !plain(b[4], at::kInt, {x->numel()}) || !call.here(*x) || x->numel() * call.c.page_size < shared) Py_RETURN_NONE;
            pages = (const int32_t*)x->data_ptr();
        } else if (shared) {
            if ((int64_t)call.c.table_pages * call.c.page_size < shared) Py_RETURN_NONE;
            pages = call.c.table;  // the first sequence's
        }
        bool ok = true;
        int32_t* flags = (int32_t*)call.optional(b[7], at::kInt, {call.B}, ok);
        float* lse = ok ? (float*)call.optional(b[9], at::kFloat, {call.B, N, (int64_t)q.heads}, ok) : nullptr;
        if (!ok) Py_RETURN_NONE;
        at::Tensor made, scratch;
        if (b[6] == Py_None) made = call.t.counts ? at::zeros_like(*from) : at::empty_like(*from);
        if (!call.heads_of(b[6] == Py_None ? &made : tensor_of(b[6]), out, N)) Py_RETURN_NONE;
        const at::Tensor* ws = nullptr;
        if (b[8] != Py_None) {
            ws = tensor_of(b[8]);
            if (!ws || !plain(b[8], at::kByte, {ws->numel()}) || !call.here(*ws)) Py_RETURN_NONE;
        } else if (const size_t size = mdsd_tree_attention_lse_workspace_bytes(&call.c, call.scales(), &call.t, q.heads, shared, longest)) {
            scratch = at::empty({(int64_t)size}, from->options().dtype(at::kByte));
            ws = &scratch;
        }
        int rc;
        Py_BEGIN_ALLOW_THREADS;
        rc = mdsd_tree_attention_lse(&call.c, call.scales(), layer, &call.t, &q, &out, scale, pages, shared, longest, lse, flags,
                                     ws ? ws->data_ptr() : nullptr, ws ? (size_t)ws->numel() : 0, stream);
        Py_END_ALLOW_THREADS;
        return answer(rc, b[6], std::move(made));
    });
}

// kv_commit(stream, <cache and tree>, outcome, accept_depth, out or None, flags or None): the new lengths
PyObject* kv_commit(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        void* stream;
        CacheCall call;
        if (n != 1 + kCacheArgs + 4 || !stream_of(a[0], stream) || !call.cache_of(a + 1)) Py_RETURN_NONE;
        PyObject* const* const b = a + 1 + kCacheArgs;
        const at::Tensor* outcome = tensor_of(b[0]);
        if (!outcome || outcome->dim() != 2 || !plain(b[0], at::kInt, {call.B, outcome->size(1)}) || !call.here(*outcome) ||
            !call.tree_of(a + 1, outcome->size(1)))
            Py_RETURN_NONE;
        bool ok = b[1] != Py_None;
        const int32_t* accepted = ok ? (const int32_t*)call.optional(b[1], at::kInt, {call.B}, ok) : nullptr;
        int32_t* flags = ok ? (int32_t*)call.optional(b[3], at::kInt, {call.B}, ok) : nullptr;
        if (!ok) Py_RETURN_NONE;
        at::Tensor made;
        int32_t* lengths;
        if (b[2] == Py_None) {
            made = at::empty({call.B}, outcome->options());
            lengths = (int32_t*)made.data_ptr();
        } else {
            lengths = (int32_t*)call.optional(b[2], at::kInt, {call.B}, ok);
        }
        if (!ok) Py_RETURN_NONE;
        int rc;
        Py_BEGIN_ALLOW_THREADS;
        rc = call.four ? mdsd_kv4_commit(&call.c, &call.s, &call.t, (const int32_t*)outcome->data_ptr(), accepted, lengths, flags, stream)
                       : mdsd_kv_commit(&call.c, &call.t, (const int32_t*)outcome->data_ptr(), accepted, lengths, flags, stream);
        Py_END_ALLOW_THREADS;
        return answer(rc, b[2], std::move(made));
    });
}

// [B, slots] float32 with unit stride, rows that do not overlap
float* weights_of(const CacheCall& call, PyObject* o, int64_t slots, int64_t& ld)
{
    const at::Tensor* x = tensor_of(o);
    if (!x || !call.here(*x) || x->scalar_type() != at::kFloat || x->dim() != 2 || x->size(0) != call.B || x->size(1) != slots ||
        (slots != 1 && x->stride(1) != 1) || (call.B > 1 && x->stride(0) < slots))
        return nullptr;
    ld = call.B > 1 ? x->stride(0) : slots;
    return (float*)x->data_ptr();
}

// kv_weigh(stream, <cache and tree>, q, lse, weights or None, layer, scale or None, outcome or None, accept_depth or None, out, flags or
// None): the sums
PyObject* kv_weigh(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        void* stream;
        CacheCall call;
        if (n != 1 + kCacheArgs + 9 || !stream_of(a[0], stream) || !call.cache_of(a + 1)) Py_RETURN_NONE;
        PyObject* const* const b = a + 1 + kCacheArgs;
        mdsd_heads q;
        int64_t N = -1, ld_weights = 0, ld_out = 0;
        int32_t layer;
        float scale;
        if (!call.heads_of(tensor_of(b[0]), q, N) || !call.tree_of(a + 1, N) || !number(b[3], layer)) Py_RETURN_NONE;
        if (b[4] == Py_None)
            scale = (float)(1.0 / std::sqrt((double)call.c.dim));
        else if (!number(b[4], scale))
            Py_RETURN_NONE;
        const at::Tensor* to = tensor_of(b[7]);
        if (!to || to->dim() != 2 || to->size(1) < 1 || to->size(1) > INT32_MAX || call.B < 1) Py_RETURN_NONE;
        float* const out = weights_of(call, b[7], to->size(1), ld_out);
        const float* const weights = b[2] == Py_None ? nullptr : weights_of(call, b[2], to->size(1), ld_weights);
        bool ok = out && (weights || b[2] == Py_None) && b[1] != Py_None;
        const float* lse = ok ? (const float*)call.optional(b[1], at::kFloat, {call.B, N, (int64_t)q.heads}, ok) : nullptr;
        const int32_t* outcome = ok ? (const int32_t*)call.optional(b[5], at::kInt, {call.B, N}, ok) : nullptr;
        const int32_t* accepted = ok ? (const int32_t*)call.optional(b[6], at::kInt, {call.B}, ok) : nullptr;
        int32_t* flags = ok ? (int32_t*)call.optional(b[8], at::kInt, {call.B}, ok) : nullptr;
        if (!ok) Py_RETURN_NONE;
        int rc;
        Py_BEGIN_ALLOW_THREADS;
        rc = mdsd_kv_weigh(&call.c, call.scales(), layer, &call.t, &q, lse, scale, outcome, accepted, weights, ld_weights, out, ld_out,
                           (int32_t)to->size(1), flags, stream);
        Py_END_ALLOW_THREADS;
        return answer(rc, b[7], at::Tensor());
    });
}

// kv_evict(stream, <cache>, weights, budget, first, recent, out or None, kept or None, weights_out or None, flags or None): the new
// lengths, and what was kept
PyObject* kv_evict(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        void* stream;
        CacheCall call;
        if (n != 1 + kPagesArgs + 8 || !stream_of(a[0], stream) || !call.cache_of(a + 1)) Py_RETURN_NONE;
        PyObject* const* const b = a + 1 + kPagesArgs;
        int32_t budget, first, recent;
        int64_t ld_weights = 0, ld_out = 0;
        const at::Tensor* from = tensor_of(b[0]);
        if (!from || from->dim() != 2 || from->size(1) < 1 || from->size(1) > INT32_MAX || call.B < 1 || !number(b[1], budget) || budget < 1 ||
            !number(b[2], first) || !number(b[3], recent))
            Py_RETURN_NONE;
        const int64_t slots = from->size(1);
        const float* const weights = weights_of(call, b[0], slots, ld_weights);
        float* const to = b[6] == Py_None ? nullptr : weights_of(call, b[6], slots, ld_out);
        bool ok = weights && (to || b[6] == Py_None);
        int32_t* lengths = ok ? (int32_t*)call.optional(b[4], at::kInt, {call.B}, ok) : nullptr;
        int32_t* kept = ok ? (int32_t*)call.optional(b[5], at::kInt, {call.B, (int64_t)budget}, ok) : nullptr;
        int32_t* flags = ok ? (int32_t*)call.optional(b[7], at::kInt, {call.B}, ok) : nullptr;
        if (!ok) Py_RETURN_NONE;
        at::Tensor made[2];
        const auto ints = from->options().dtype(at::kInt);
        if (!lengths) lengths = (int32_t*)(made[0] = at::empty({call.B}, ints)).data_ptr();
        if (!kept) kept = (int32_t*)(made[1] = at::empty({call.B, (int64_t)budget}, ints)).data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS;
        rc = mdsd_kv_evict(&call.c, call.scales(), (int32_t)call.B, weights, ld_weights, (int32_t)slots, budget, first, recent, lengths, kept,
                           to, ld_out, flags, stream);
        Py_END_ALLOW_THREADS;
        if (rc != MDSD_OK) return PyLong_FromLong(rc);
        PyObject* const both = PyTuple_New(2);
        if (!both) return nullptr;
        PyTuple_SET_ITEM(both, 0, answer(rc, b[4], std::move(made[0])));
        PyTuple_SET_ITEM(both, 1, answer(rc, b[5], std::move(made[1])));
        return both;
    });
}

PyMethodDef methods[] = {
    {"kv_weigh", (PyCFunction)(void (*)(void))kv_weigh, METH_FASTCALL, nullptr},
    {"kv_evict", (PyCFunction)(void (*)(void))kv_evict, METH_FASTCALL, nullptr},
    {"kv_append", (PyCFunction)(void (*)(void))kv_append, METH_FASTCALL, nullptr},
    {"tree_attention", (PyCFunction)(void (*)(void))tree_attention, METH_FASTCALL, nullptr},
    {"kv_commit", (PyCFunction)(void (*)(void))kv_commit, METH_FASTCALL, nullptr},
    {"draft", (PyCFunction)(void (*)(void))draft, METH_FASTCALL, nullptr},
    {"verify", (PyCFunction)(void (*)(void))verify, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host(void) { return PyModule_Create(&module); }
