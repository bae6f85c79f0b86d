// Argument marshalling of the calls that a serving loop makes, as a CPython module: what binding.py does with ctypes, without a Python
// object for every pointer.  A call here answers the plain case -- tensors of exactly torch's own classes, structs of the binding's
// own classes or of classes that pack like them, numbers that struct.pack and ctypes would take, the current stream or a stream's handle -- and returns None for everything else
// (other classes, a wrong dtype, device or layout, a tensor missing), before anything has been launched: binding.py then takes its own path,
// which raises what it raised before.  What is refused is refused without an exception, at the first argument that is not plain.
// A step of one layer (append and attention, 10.5 us on the device) took 14.2 us of host time, 6.3 of them in the library.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <dlfcn.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "rows.h"
#include "vector.h"

namespace {

#define ENTRY_POINTS(X) \
    X(vector_score) X(vector_route) X(vector_route_layer) X(vector_compact) X(vector_compact_layer) X(vector_append) X(vector_decode_attn) \
        X(vector_decode_attn_layer) X(vector_decode_attn_static) X(vector_block_tables) X(vector_compact_q4) X(vector_append_q4) X(vector_read_q4) \
        X(vector_decode_attn_q4) X(vector_q4_tile_bytes) X(vector_compact_q8) X(vector_append_q8) X(vector_read_q8) X(vector_decode_attn_q8) X(vector_q8_tile_bytes) \
        X(vector_norm_rope)
#define POINTER(name) decltype(&::name) p_##name = nullptr;
ENTRY_POINTS(POINTER)

// A class of the binding, and what makes up the packed form that ctypes is given: a class derived from it is read like it where these
// members are still the base's.
struct Class {
    static constexpr int MEMBERS = 2;
    PyTypeObject* type = nullptr;
    PyObject* name[MEMBERS] = {};
    PyObject* member[MEMBERS] = {};
    bool covers(PyObject* o) const {
        if (Py_TYPE(o) == type) return true;
        if (!PyType_IsSubtype(Py_TYPE(o), type)) return false;
        for (int i = 0; i < MEMBERS; ++i)
            if (name[i]) {
                PyObject* m = PyObject_GetAttr((PyObject*)Py_TYPE(o), name[i]);
                Py_XDECREF(m);
                if (m != member[i]) return false;
            }
        return true;
    }
    bool set(PyObject* t, const char* first, const char* second = nullptr) {
        Py_INCREF(t);
        type = (PyTypeObject*)t;
        const char* const names[MEMBERS] = {first, second};
        for (int i = 0; i < MEMBERS; ++i)
            if (names[i] && (!(name[i] = PyUnicode_InternFromString(names[i])) || !(member[i] = PyObject_GetAttr(t, name[i])))) return false;
        return true;
    }
};
Class shape_class, budget_class, cache_class, q4_cache_class;
enum Name { BATCH, N_LAYERS, N_Q_HEADS, N_KV_HEADS, HEAD_DIM, DTYPE, WINDOW, POOL_KERNEL, SM_SCALE, ROPE_ENABLED, ROPE_THETA, N_TOKENS,
            N_BUDGET_PAIRS, N_A, N_POOL, N_APX, N_RET, N_EVICT, RET_K, RET_V, APX_K, RET_POS, APX_POS,
            RET_PAGES, APX_PAGES, RET_TABLE, APX_TABLE, RET_LEN, APX_LEN, NAMES };
const char* const spelled[NAMES] = {"batch", "n_layers", "n_q_heads", "n_kv_heads", "head_dim", "dtype", "window", "pool_kernel", "sm_scale",
                                    "rope_enabled", "rope_theta", "n_tokens", "n_budget_pairs", "n_a", "n_pool", "n_apx", "n_ret",
                                    "n_evict", "ret_k", "ret_v", "apx_k", "ret_pos", "apx_pos", "ret_pages", "apx_pages", "ret_table", "apx_table", "ret_len",
                                    "apx_len"};
PyObject* name[NAMES];

struct Ref {                                            // an owned reference, or none
    PyObject* o;
    explicit Ref(PyObject* p) : o(p) {}
    ~Ref() { Py_XDECREF(o); }
    Ref(const Ref&) = delete;
};
struct Workspace { void* p = nullptr; size_t n = 0; };
struct Out { void* p = nullptr; int32_t type = 0; };
at::ScalarType type_of(const vector_shape& s) { return s.dtype == VECTOR_BF16 ? at::kBFloat16 : at::kFloat; }

// Reads a call's arguments.  `plain` turns false at the first one that is not: what is read from then on is nothing and means nothing.
struct Reader {
    bool plain = true;
    int here = -1;                                      // the device that tensors have to lie on, where the call asks for it
    void on_current_device() { here = c10::cuda::current_device(); }
    bool need(bool holds) { return plain = plain && holds; }
    PyObject* attr(PyObject* o, Name n) {               // new, or null
        PyObject* v = plain ? PyObject_GetAttr(o, name[n]) : nullptr;
        need(v);
        return v;
    }
    int64_t integer(PyObject* o) {                      // an argument: ctypes takes an int
        if (!need(o && PyLong_Check(o))) return 0;
        int over = 0;
        const long long v = PyLong_AsLongLongAndOverflow(o, &over);
        need(!over);
        return v;
    }
    int32_t integer32(PyObject* o) {
        const int64_t v = integer(o);
        need(v == (int32_t)v);
        return (int32_t)v;
    }
    int64_t field(PyObject* o, Name n) {                // a struct's field: struct.pack takes whatever is an index
        const Ref v(attr(o, n));
        if (!plain || PyLong_Check(v.o)) return integer(v.o);
        if (!need(PyIndex_Check(v.o))) return 0;
        const Ref i(PyNumber_Index(v.o));
        return need(i.o) ? integer(i.o) : 0;
    }
    int32_t field32(PyObject* o, Name n) {
        const int64_t v = field(o, n);
        need(v == (int32_t)v);
        return (int32_t)v;
    }
    float number(PyObject* o, Name n) {                 // whatever is a float, an integer too
        const Ref v(attr(o, n));
        if (!plain) return 0.f;
        const double x = PyFloat_AsDouble(v.o);
        need(!PyErr_Occurred() && std::isfinite((float)x));
        return (float)x;
    }
    const at::Tensor* tensor(PyObject* o) { return need(o && THPVariable_CheckExact(o)) ? &THPVariable_Unpack(o) : nullptr; }
    void* device(PyObject* o, at::ScalarType type) {
        const at::Tensor* t = tensor(o);
        return t && need(t->is_cuda() && t->is_contiguous() && t->scalar_type() == type && (here < 0 || t->get_device() == here)) ? t->data_ptr() : nullptr;
    }
    void* optional(PyObject* o, at::ScalarType type) { return o == Py_None ? nullptr : device(o, type); }
    // A tensor of n elements at least; null where there are none to have.
    void* sized(PyObject* o, at::ScalarType type, int64_t n) {
        if (n == 0) return nullptr;
        void* p = device(o, type);
        return plain && need(tensor(o)->numel() >= n) ? p : nullptr;
    }
    int32_t* ints(PyObject* o, int64_t n) { return (int32_t*)sized(o, at::kInt, n); }
    int32_t* optional_ints(PyObject* o, int64_t n) { return o == Py_None ? nullptr : ints(o, n); }
    int64_t numel(PyObject* o) {
        const at::Tensor* t = o == Py_None ? nullptr : tensor(o);
        return t ? t->numel() : 0;
    }
    Workspace workspace(PyObject* o) {
        Workspace w;
        w.p = optional(o, at::kByte);
        if (plain && o != Py_None) w.n = (size_t)tensor(o)->numel();
        return w;
    }
    Out output(PyObject* o) {
        Out out;
        const at::Tensor* t = tensor(o);
        if (!t || !need(t->scalar_type() == at::kFloat || t->scalar_type() == at::kBFloat16)) return out;
        out.type = t->scalar_type() == at::kBFloat16 ? VECTOR_BF16 : VECTOR_F32;
        out.p = device(o, t->scalar_type());
        return out;
    }
    void* stream(PyObject* o) {                         // None, the current one, or a handle
        if (!plain) return nullptr;
        if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
        if (!need(PyLong_CheckExact(o))) return nullptr;
        void* p = PyLong_AsVoidPtr(o);
        need(!PyErr_Occurred());
        return p;
    }
    vector_shape shape(PyObject* o) {
        vector_shape s = {};
        if (!need(shape_class.covers(o))) return s;
        s.batch = field32(o, BATCH);
        s.n_layers = field32(o, N_LAYERS);
        s.n_q_heads = field32(o, N_Q_HEADS);
        s.n_kv_heads = field32(o, N_KV_HEADS);
        s.head_dim = field32(o, HEAD_DIM);
        s.dtype = field32(o, DTYPE);
        s.window = field32(o, WINDOW);
        s.pool_kernel = field32(o, POOL_KERNEL);
        s.sm_scale = number(o, SM_SCALE);
        s.rope_enabled = field32(o, ROPE_ENABLED);
        s.rope_theta = number(o, ROPE_THETA);
        return s;
    }
    vector_budget budget(PyObject* o) {
        vector_budget b = {};
        if (!need(budget_class.covers(o))) return b;
        b.n_tokens = field(o, N_TOKENS);
        b.n_budget_pairs = field(o, N_BUDGET_PAIRS);
        b.n_a = field(o, N_A);
        b.n_pool = field(o, N_POOL);
        b.n_apx = field(o, N_APX);
        b.n_ret = field(o, N_RET);
        b.n_evict = field(o, N_EVICT);
        return b;
    }
    vector_cache cache(PyObject* o) {
        vector_cache c = {};
        if (!need(cache_class.covers(o))) return c;
        const Ref rk(attr(o, RET_K)), rv(attr(o, RET_V)), ak(attr(o, APX_K)), rp(attr(o, RET_POS)), ap(attr(o, APX_POS));
        const at::Tensor *trk = tensor(rk.o), *trv = tensor(rv.o), *tak = tensor(ak.o), *trp = tensor(rp.o), *tap = tensor(ap.o);
        if (!plain || !need(trk->dim() >= 2 && tak->dim() >= 2)) return c;
        c.ret_k = trk->data_ptr();
        c.ret_v = trv->data_ptr();
        c.apx_k = tak->data_ptr();
        c.ret_pos = (decltype(c.ret_pos))trp->data_ptr();
        c.apx_pos = (decltype(c.apx_pos))tap->data_ptr();
        c.cap_ret = trk->size(1);
        c.cap_apx = tak->size(1);
        c.n_ret = field(o, N_RET);
        c.n_apx = field(o, N_APX);
        return c;
    }
    // Rows of `width` neighbouring elements: contiguous ones, or those that rows.h finds.
    struct Rows { void* p = nullptr; int64_t stride = 0; };
    Rows rows(PyObject* o, at::ScalarType type, int64_t count, int64_t width) {
        Rows r;
        const at::Tensor* t = tensor(o);
        if (!t || !need(t->is_cuda() && t->scalar_type() == type && (here < 0 || t->get_device() == here) && width > 0 && t->numel() == count * width)) return r;
        r.p = t->data_ptr();
        r.stride = width;
        if (!t->is_contiguous()) need(vec::row_distance(t->sizes().data(), t->strides().data(), (int)t->dim(), width, &r.stride));
        return r;
    }
    vector_q4_cache q8_cache(PyObject* o, const vector_shape& s) { return q4_cache(o, s, true, p_vector_q8_tile_bytes, VECTOR_Q8_PAGE_ROWS); }
    // attends: with the tables and lengths, which of the 4-bit cache's calls attention alone reads.
    vector_q4_cache q4_cache(PyObject* o, const vector_shape& s, bool attends, size_t (*tile_bytes)(const vector_shape*) = p_vector_q4_tile_bytes, int page_rows = VECTOR_PAGE_ROWS) {
        vector_q4_cache c = {};
        if (!plain || !need(q4_cache_class.covers(o))) return c;
        const int64_t LH = (int64_t)s.n_layers * s.n_kv_heads, tile = (int64_t)tile_bytes(&s);
        auto pages = [&](Name n, int64_t bytes, int64_t* count) -> void* {
            const Ref r(attr(o, n));
            void* p = plain ? device(r.o, at::kByte) : nullptr;
            if (!plain) return nullptr;
            const at::Tensor* t = tensor(r.o);
            if (!need(t->dim() == 3 && t->size(1) == LH && t->size(2) == bytes)) return nullptr;
            *count = t->size(0);
            return p;
        };
        c.ret_pages = pages(RET_PAGES, 2 * tile, &c.n_ret_pages);
        c.apx_pages = pages(APX_PAGES, tile, &c.n_apx_pages);
        auto positions = [&](Name n, int64_t count) -> int32_t* {
            const Ref r(attr(o, n));
            return plain ? optional_ints(r.o, count * LH * page_rows) : nullptr;
        };
        c.ret_pos = positions(RET_POS, c.n_ret_pages);
        c.apx_pos = positions(APX_POS, c.n_apx_pages);
        auto tables = [&](Name n, Name len, const int32_t** table, const int32_t** lens, int32_t* width) {
            const Ref r(attr(o, n)), l(attr(o, len));
            if (!plain) return;
            *table = (int32_t*)device(r.o, at::kInt);
            if (!plain || !need(tensor(r.o)->dim() == 2 && tensor(r.o)->size(0) >= s.batch && tensor(r.o)->size(1) <= 0x7fffffffLL)) return;
            *width = (int32_t)tensor(r.o)->size(1);
            *lens = ints(l.o, s.batch);
        };
        if (attends) {
            tables(RET_TABLE, RET_LEN, &c.ret_table, &c.ret_len, &c.ret_width);
            tables(APX_TABLE, APX_LEN, &c.apx_table, &c.apx_len, &c.apx_width);
        }
        return c;
    }
};
int64_t units_of(const vector_shape& s) { return (int64_t)s.batch * s.n_layers * s.n_kv_heads; }

// What `call` returns as a Python integer; None where the plain case does not hold.
template <typename F>
PyObject* plain(Py_ssize_t given, Py_ssize_t wanted, F call) {
    if (given != wanted) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return nullptr; }
    Reader r;
    long rc = 0;
    try {
        rc = call(r);
    } catch (const std::exception&) {                   // torch's refusals: a tensor without storage, say
        r.plain = false;
    }
    if (r.plain) return PyLong_FromLong(rc);
    PyErr_Clear();
    Py_RETURN_NONE;
}
// The library runs without the interpreter's lock, as it does under ctypes; nothing runs where the plain case does not hold.
template <typename F>
long run(const Reader& r, F f) {
    long rc = 0;
    if (!r.plain) return rc;
    Py_BEGIN_ALLOW_THREADS
    rc = (long)f();
    Py_END_ALLOW_THREADS
    return rc;
}

#define METHOD(name) PyObject* name(PyObject*, PyObject* const* a, Py_ssize_t n)
METHOD(score) {                                         // shape, Q_obs, K, N, scores, raw_out, ws, stream
    return plain(n, 8, [&](Reader& r) {
        const vector_shape s = r.shape(a[0]);
        void *q = r.device(a[1], type_of(s)), *k = r.device(a[2], type_of(s));
        const int64_t N = r.integer(a[3]);
        float *out = (float*)r.device(a[4], at::kFloat), *raw = (float*)r.optional(a[5], at::kFloat);
        const Workspace w = r.workspace(a[6]);
        void* st = r.stream(a[7]);
        return run(r, [&] { return p_vector_score(&s, q, k, N, out, raw, w.p, w.n, st); });
    });
}
template <typename Fn>
long route_with(Fn fn, Reader& r, PyObject* const* a) { // shape, budget, scores, K, V, W, tier, ret_idx, apx_idx, eps_out, pool_idx_out, ws, stream
    const vector_shape s = r.shape(a[0]);
    const vector_budget b = r.budget(a[1]);
    const at::ScalarType type = type_of(s);
    const float* scores = (const float*)r.device(a[2], at::kFloat);
    void *k = r.device(a[3], type), *v = r.device(a[4], type), *w = r.device(a[5], type);
    uint8_t* tier = (uint8_t*)r.device(a[6], at::kByte);
    int32_t *ret = (int32_t*)r.device(a[7], at::kInt), *apx = (int32_t*)r.device(a[8], at::kInt);
    float* eps = (float*)r.optional(a[9], at::kFloat);
    int32_t* pool = (int32_t*)r.optional(a[10], at::kInt);
    const Workspace ws = r.workspace(a[11]);
    void* st = r.stream(a[12]);
    return run(r, [&] { return fn(&s, &b, scores, k, v, w, tier, ret, apx, eps, pool, ws.p, ws.n, st); });
}
METHOD(route) { return plain(n, 13, [&](Reader& r) { return route_with(p_vector_route, r, a); }); }
METHOD(route_layer) { return plain(n, 13, [&](Reader& r) { return route_with(p_vector_route_layer, r, a); }); }
template <typename Fn>
long compact_with(Fn fn, Reader& r, PyObject* const* a) {      // shape, budget, K, V, ret_idx, apx_idx, cache, stream
    const vector_shape s = r.shape(a[0]);
    const vector_budget b = r.budget(a[1]);
    void *k = r.device(a[2], type_of(s)), *v = r.device(a[3], type_of(s));
    const int32_t *ret = (const int32_t*)r.device(a[4], at::kInt), *apx = (const int32_t*)r.device(a[5], at::kInt);
    const vector_cache c = r.cache(a[6]);
    void* st = r.stream(a[7]);
    return run(r, [&] { return fn(&s, &b, k, v, ret, apx, &c, st); });
}
METHOD(compact) { return plain(n, 8, [&](Reader& r) { return compact_with(p_vector_compact, r, a); }); }
METHOD(compact_layer) { return plain(n, 8, [&](Reader& r) { return compact_with(p_vector_compact_layer, r, a); }); }
METHOD(decode_attn) {                                   // shape, q, cache, W, out, mode, ws, stream
    return plain(n, 8, [&](Reader& r) {
        const vector_shape s = r.shape(a[0]);
        void* q = r.device(a[1], type_of(s));
        const vector_cache c = r.cache(a[2]);
        void* W = r.device(a[3], type_of(s));
        const Out out = r.output(a[4]);
        const int32_t mode = r.integer32(a[5]);
        const Workspace w = r.workspace(a[6]);
        void* st = r.stream(a[7]);
        return run(r, [&] { return p_vector_decode_attn(&s, q, &c, W, out.p, out.type, mode, w.p, w.n, st); });
    });
}
METHOD(decode_attn_layer) {                             // shape, q, cache, W_layer, out, ws, stream
    return plain(n, 7, [&](Reader& r) {
        const vector_shape s = r.shape(a[0]);
        void* q = r.device(a[1], type_of(s));
        const vector_cache c = r.cache(a[2]);
        void* W = r.device(a[3], type_of(s));
        const Out out = r.output(a[4]);
        const Workspace w = r.workspace(a[5]);
        void* st = r.stream(a[6]);
        return run(r, [&] { return p_vector_decode_attn_layer(&s, q, &c, W, out.p, out.type, w.p, w.n, st); });
    });
}
METHOD(decode_attn_static) {                            // shape, q, cache, W, out, mode, stream
    return plain(n, 7, [&](Reader& r) {
        const vector_shape s = r.shape(a[0]);
        void* q = r.device(a[1], type_of(s));
        const vector_cache c = r.cache(a[2]);
        void* W = r.device(a[3], type_of(s));
        const Out out = r.output(a[4]);
        const int32_t mode = r.integer32(a[5]);
        void* st = r.stream(a[6]);
        return run(r, [&] { return p_vector_decode_attn_static(&s, q, &c, W, out.p, out.type, mode, st); });
    });
}
METHOD(append) {                                        // shape, cache, k_new, v_new, pos, stream
    return plain(n, 6, [&](Reader& r) {
        const vector_shape s = r.shape(a[0]);
        const vector_cache c = r.cache(a[1]);
        void *k = r.device(a[2], type_of(s)), *v = r.device(a[3], type_of(s));
        const int32_t pos = r.integer32(a[4]);
        void* st = r.stream(a[5]);
        return run(r, [&] { return p_vector_append(&s, &c, k, v, pos, st); });
    });
}
// Compressor.append's own conditions on top: plain rows of the shape's size on the current device, room for one more, and not what the
// entry point refuses (rows off a 16-byte boundary): those rows are assigned.
METHOD(append_rows) {                                   // shape, cache, k_new, v_new, pos
    return plain(n, 5, [&](Reader& r) {
        const vector_shape s = r.shape(a[0]);
        const vector_cache c = r.cache(a[1]);
        r.need((PyObject*)Py_TYPE(a[2]) == THPVariableClass && (PyObject*)Py_TYPE(a[3]) == THPVariableClass);
        const Ref rk(r.attr(a[1], RET_K)), rv(r.attr(a[1], RET_V)), rp(r.attr(a[1], RET_POS));
        const at::Tensor *trk = r.tensor(rk.o), *trv = r.tensor(rv.o), *trp = r.tensor(rp.o), *tk = r.tensor(a[2]), *tv = r.tensor(a[3]);
        if (!r.plain || !r.need(trk->dim() == 3 && tk->dim() == 2 && tv->dim() == 2)) return 0L;
        const int64_t U = trk->size(0), cap = trk->size(1), d = trk->size(2);
        const bool rows = tk->size(0) == U && tk->size(1) == d && tv->size(0) == U && tv->size(1) == d && d == s.head_dim &&
                          U == (int64_t)s.batch * s.n_layers * s.n_kv_heads;
        const int dev = c10::cuda::current_device();
        const bool here = tk->get_device() == dev && tv->get_device() == dev && trk->get_device() == dev && trv->get_device() == dev;
        r.need(rows && here && c.n_ret < cap && trv->nbytes() == trk->nbytes() && trk->is_contiguous() && trv->is_contiguous() &&
               trp->numel() == U * cap && !tk->requires_grad() && !tv->requires_grad());
        void *k = r.device(a[2], type_of(s)), *v = r.device(a[3], type_of(s));
        const int32_t pos = r.integer32(a[4]);
        void* st = r.stream(Py_None);
        const long rc = run(r, [&] { return p_vector_append(&s, &c, k, v, pos, st); });
        r.need(rc != VECTOR_ERR_SHAPE);
        return rc;
    });
}
METHOD(block_tables) {                                  // lengths, added, page_rows, table, free, n_free, new_lengths, new_n_free, first_row, row_start, slots, stream
    return plain(n, 12, [&](Reader& r) {
        const int32_t* table = (const int32_t*)r.device(a[3], at::kInt);
        const at::Tensor* t = r.tensor(a[3]);
        if (!r.plain || !r.need(t->dim() == 2 && t->size(0) <= 0x7fffffffLL && t->size(1) <= 0x7fffffffLL)) return 0L;
        const int64_t B = t->size(0), width = t->size(1), n_slots = r.numel(a[10]);
        const int32_t *lengths = r.ints(a[0], B), *added = r.ints(a[1], B), *n_free = r.ints(a[5], 1);
        const int32_t page_rows = r.integer32(a[2]);
        int32_t* stack = (int32_t*)r.device(a[4], at::kInt);
        const int64_t cap = r.plain ? r.tensor(a[4])->numel() : 0;
        r.need(cap <= 0x7fffffffLL);
        int32_t *new_lengths = r.ints(a[6], B), *new_n_free = r.ints(a[7], 1), *first = r.ints(a[8], B), *start = r.ints(a[9], B + 1), *slots = r.ints(a[10], n_slots);
        void* st = r.stream(a[11]);
        return run(r, [&] {
            return p_vector_block_tables((int32_t)B, lengths, added, page_rows, (int32_t*)table, (int32_t)width, stack, (int32_t)cap, n_free, new_lengths, new_n_free, first, start,
                                         slots, n_slots, st);
        });
    });
}
METHOD(compact_q4) {                                    // shape, budget, K, V, ret_idx, apx_idx, cache, ret_slots, apx_slots, stream
    return plain(n, 10, [&](Reader& r) {
        const vector_shape s = r.shape(a[0]);
        const vector_budget b = r.budget(a[1]);
        const int64_t U = units_of(s), rows = U * b.n_tokens * s.head_dim;
        void *k = r.sized(a[2], type_of(s), rows), *v = r.sized(a[3], type_of(s), rows);
        const int32_t *ri = r.ints(a[4], U * b.n_ret), *ai = r.ints(a[5], U * b.n_apx);
        const vector_q4_cache c = r.q4_cache(a[6], s, false);
        const int32_t *rs = r.ints(a[7], s.batch * b.n_ret), *as = r.ints(a[8], s.batch * b.n_apx);
        void* st = r.stream(a[9]);
        return run(r, [&] { return p_vector_compact_q4(&s, &b, k, v, ri, ai, &c, rs, as, st); });
    });
}
METHOD(append_q4) {                                     // shape, cache, k_new, v_new, row_start, slots, pos, stream
    return plain(n, 8, [&](Reader& r) {
        const vector_shape s = r.shape(a[0]);
        const vector_q4_cache c = r.q4_cache(a[1], s, false);
        const int64_t rows = units_of(s) * s.head_dim;
        void *k = r.sized(a[2], type_of(s), rows), *v = r.sized(a[3], type_of(s), rows);
        const int32_t *start = r.optional_ints(a[4], (int64_t)s.batch + 1), *slots = (const int32_t*)r.device(a[5], at::kInt), *pos = r.optional_ints(a[6], s.batch);
        const int64_t n_slots = r.plain ? r.tensor(a[5])->numel() : 0;
        void* st = r.stream(a[7]);
        return run(r, [&] { return p_vector_append_q4(&s, &c, k, v, start, slots, n_slots, pos, st); });
    });
}
METHOD(read_q4) {                                       // shape, cache, ret_slots, ret_k, ret_v, apx_slots, apx_k, stream
    return plain(n, 8, [&](Reader& r) {
        const vector_shape s = r.shape(a[0]);
        const vector_q4_cache c = r.q4_cache(a[1], s, false);
        if (!r.need(s.batch > 0)) return 0L;
        const int64_t n_ret = r.numel(a[2]) / s.batch, n_apx = r.numel(a[5]) / s.batch, d = units_of(s) * s.head_dim;
        const int32_t *rs = r.ints(a[2], s.batch * n_ret), *as = r.ints(a[5], s.batch * n_apx);
        void *rk = r.sized(a[3], type_of(s), n_ret * d), *rv = r.sized(a[4], type_of(s), n_ret * d), *ak = r.sized(a[6], type_of(s), n_apx * d);
        void* st = r.stream(a[7]);
        return run(r, [&] { return p_vector_read_q4(&s, &c, rs, n_ret, rk, rv, as, n_apx, ak, st); });
    });
}
METHOD(decode_attn_q4) {                                // shape, q, cache, W, out, ws, stream
    return plain(n, 7, [&](Reader& r) {
        const vector_shape s = r.shape(a[0]);
        if (!r.need(s.n_kv_heads > 0)) return 0L;
        const int64_t rows = units_of(s) * (s.n_q_heads / s.n_kv_heads) * s.head_dim;
        void* q = r.sized(a[1], type_of(s), rows);
        const vector_q4_cache c = r.q4_cache(a[2], s, true);
        void* W = r.sized(a[3], type_of(s), (int64_t)s.n_layers * s.n_kv_heads * s.head_dim * s.head_dim);
        const Out out = r.output(a[4]);
        r.need(r.numel(a[4]) >= rows);
        const Workspace w = r.workspace(a[5]);
        void* st = r.stream(a[6]);
        return run(r, [&] { return p_vector_decode_attn_q4(&s, q, &c, W, out.p, out.type, w.p, w.n, st); });
    });
}
METHOD(compact_q8) {                                    // shape, budget, K, V, ret_idx, apx_idx, cache, stream
    return plain(n, 8, [&](Reader& r) {
        r.on_current_device();
        const vector_shape s = r.shape(a[0]);
        const vector_budget b = r.budget(a[1]);
        const int64_t U = units_of(s), rows = U * b.n_tokens * s.head_dim;
        void *k = r.sized(a[2], type_of(s), rows), *v = r.sized(a[3], type_of(s), rows);
        const int32_t *ri = r.ints(a[4], U * b.n_ret), *ai = r.ints(a[5], U * b.n_apx);
        const vector_q8_cache c = r.q8_cache(a[6], s);
        void* st = r.stream(a[7]);
        return run(r, [&] { return p_vector_compact_q8(&s, &b, k, v, ri, ai, &c, st); });
    });
}
METHOD(append_q8) {                                     // shape, cache, k_new, v_new, first_row, pos, rotate, stream
    return plain(n, 8, [&](Reader& r) {
        r.on_current_device();
        const vector_shape s = r.shape(a[0]);
        const vector_q8_cache c = r.q8_cache(a[1], s);
        const int64_t width = (int64_t)s.n_layers * s.n_kv_heads * s.head_dim, each = width * s.batch;
        if (!r.need(each > 0 && width > 0 && PyBool_Check(a[6]))) return 0L;
        const int64_t rows = r.numel(a[2]) / each;
        for (PyObject* o : {a[2], a[3]}) {               // several tokens have to show their order
            const at::Tensor* t = r.tensor(o);
            r.need(t && (rows <= 1 || (t->dim() >= 2 && ((t->size(0) == s.batch && t->size(1) == rows) || (t->dim() == 2 && t->size(0) == s.batch * rows && t->size(1) == width)))));
        }
        const Reader::Rows k = r.rows(a[2], type_of(s), s.batch * rows, width), v = r.rows(a[3], type_of(s), s.batch * rows, width);
        const int32_t *first = r.ints(a[4], s.batch), *pos = r.optional_ints(a[5], s.batch * rows);
        r.need(a[5] == Py_None || r.numel(a[5]) == s.batch * rows);
        const int32_t rotate = a[6] == Py_True;
        void* st = r.stream(a[7]);
        return run(r, [&] { return p_vector_append_q8(&s, &c, k.p, k.stride, v.p, v.stride, rows, first, pos, rotate, st); });
    });
}
METHOD(read_q8) {                                       // shape, cache, ret_k, ret_v, apx_k, stream
    return plain(n, 6, [&](Reader& r) {
        r.on_current_device();
        const vector_shape s = r.shape(a[0]);
        const vector_q8_cache c = r.q8_cache(a[1], s);
        const int64_t each = units_of(s) * s.head_dim;
        if (!r.need(each > 0)) return 0L;
        const int64_t n_ret = r.numel(a[2]) / each, n_apx = r.numel(a[4]) / each;
        r.need(r.numel(a[2]) % each == 0 && r.numel(a[3]) == r.numel(a[2]) && (a[3] == Py_None) == (a[2] == Py_None) && r.numel(a[4]) % each == 0);
        void *rk = r.sized(a[2], type_of(s), n_ret * each), *rv = r.sized(a[3], type_of(s), n_ret * each), *ak = r.sized(a[4], type_of(s), n_apx * each);
        void* st = r.stream(a[5]);
        return run(r, [&] { return p_vector_read_q8(&s, &c, n_ret, rk, rv, n_apx, ak, st); });
    });
}
METHOD(decode_attn_q8) {                                // shape, q, cache, W, out, ws, stream
    return plain(n, 7, [&](Reader& r) {
        r.on_current_device();
        const vector_shape s = r.shape(a[0]);
        if (!r.need(s.n_kv_heads > 0)) return 0L;
        const int64_t rows = units_of(s) * (s.n_q_heads / s.n_kv_heads) * s.head_dim;
        void* q = r.sized(a[1], type_of(s), rows);
        const vector_q8_cache c = r.q8_cache(a[2], s);
        void* W = r.sized(a[3], type_of(s), (int64_t)s.n_layers * s.n_kv_heads * s.head_dim * s.head_dim);
        const Out out = r.output(a[4]);
        r.need(r.numel(a[4]) >= rows);
        const Workspace w = r.workspace(a[5]);
        void* st = r.stream(a[6]);
        return run(r, [&] { return p_vector_decode_attn_q8(&s, q, &c, W, out.p, out.type, w.p, w.n, st); });
    });
}
METHOD(norm_rope) {                                     // shape, n_tokens, q, k, v, q_out, k_out, v_out, q_weight, k_weight, pos, q_first, eps, stream
    return plain(n, 14, [&](Reader& r) {
        r.on_current_device();
        const vector_shape s = r.shape(a[0]);
        const int64_t N = r.integer(a[1]), first = r.integer(a[11]), BL = (int64_t)s.batch * s.n_layers, d = s.head_dim;
        if (!r.need(s.batch > 0 && s.n_layers > 0 && s.n_q_heads > 0 && s.n_kv_heads > 0 && d > 0 && N > 0 && N <= (1 << 30) && first >= 0 && first <= N && PyFloat_Check(a[12]))) return 0L;
        const at::ScalarType type = type_of(s);
        Reader::Rows in[3];
        void* out[3] = {};
        for (int i = 0; i < 3 && r.plain; ++i)
            if (a[2 + i] != Py_None) {
                const int64_t heads = i == 0 ? s.n_q_heads : s.n_kv_heads;
                in[i] = r.rows(a[2 + i], type, BL * N, heads * d);
                out[i] = r.sized(a[5 + i], type, BL * heads * (i == 0 ? N - first : N) * d);
            }
        void* weight[2];
        for (int i = 0; i < 2; ++i) weight[i] = a[8 + i] == Py_None ? nullptr : r.sized(a[8 + i], type, s.n_layers * d);
        const int32_t* pos = r.optional_ints(a[10], s.batch * N);
        r.need(a[10] == Py_None || r.numel(a[10]) == s.batch * N);
        const float eps = (float)PyFloat_AsDouble(a[12]);
        void* st = r.stream(a[13]);
        return run(r, [&] {
            return p_vector_norm_rope(&s, N, in[0].p, in[0].stride, weight[0], first, out[0], in[1].p, in[1].stride, weight[1], out[1], in[2].p, in[2].stride, out[2], pos, eps, st);
        });
    });
}
// The library's entry points, by the handle of the library that ctypes has loaded, and the classes of the structs.
METHOD(bind) {
    if (n != 5 || !PyLong_Check(a[0]) || !PyType_Check(a[1]) || !PyType_Check(a[2]) || !PyType_Check(a[3]) || !PyType_Check(a[4])) {
        PyErr_SetString(PyExc_TypeError, "bind(handle, Shape, Budget, Cache, Q4Cache)");
        return nullptr;
    }
    void* handle = PyLong_AsVoidPtr(a[0]);
#define RESOLVE(name)                                                                                             \
    p_##name = (decltype(p_##name))dlsym(handle, #name);                                                          \
    if (!p_##name) { PyErr_SetString(PyExc_ImportError, "libvector.so does not export " #name); return nullptr; }
    ENTRY_POINTS(RESOLVE)
    if (!shape_class.set(a[1], "_p", "torch_dtype") || !budget_class.set(a[2], "_p") || !cache_class.set(a[3], "_p") || !q4_cache_class.set(a[4], "_p"))
        return nullptr;
    Py_RETURN_NONE;
}

#define ROW(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ROW(bind), ROW(score), ROW(route), ROW(route_layer), ROW(compact), ROW(compact_layer), ROW(append), ROW(append_rows),
                         ROW(decode_attn), ROW(decode_attn_layer), ROW(decode_attn_static), ROW(block_tables), ROW(compact_q4), ROW(append_q4),
                         ROW(read_q4), ROW(decode_attn_q4), ROW(compact_q8), ROW(append_q8), ROW(read_q8), ROW(decode_attn_q8), ROW(norm_rope), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
    for (int i = 0; i < NAMES; ++i)
        if (!(name[i] = PyUnicode_InternFromString(spelled[i]))) return nullptr;
    return PyModule_Create(&module);
}
