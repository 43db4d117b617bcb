// The host path of the calls that a serving loop makes every step (sd_speculate, sd_step, sd_append; the verifier's
// sd_rotate, sd_attend, sd_accept, sd_commit, the first two once a layer), from torch tensors to the C entry points.
//
// What bounds it: nothing but the host.  A draft for one request takes the GPU 6.9 us; converting
// the arguments in Python and through ctypes took 6 of the call's 8.8 us (each of up to 13 tensors
// costs four attribute lookups, each argument a converter), so a small batch waited for its launches.
// Here a tensor costs one type check and a few loads: 3.1 us for the call (most of it the launch), and
// 17.6 us (22.6 before) from an idle GPU through one such draft to its end.
//
// Only the usual case is taken here: CUDA tensors, contiguous, of the right type.  Anything else (a
// pinned host tensor, or an argument that is not one) goes to the Python function that `setup` was
// given, which returns the address or raises.
#include <Python.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ops/empty.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "suffixspec.h"

namespace {

constexpr int64_t SD_MAX_DRAFT = 64;

decltype(&sd_speculate) f_speculate;
decltype(&sd_step) f_step;
decltype(&sd_append) f_append;
PyObject* slow_ptr;                                              // binding._ptr(tensor, dtype, name)

struct Field {
    const char* name;
    c10::ScalarType type;
    const char* dtype;                                           // the attribute of torch that names it
    PyObject* key;                                               // interned name
    PyObject* py_dtype;
};

enum { N_DRAFT, TOKENS, PARENTS, POSITIONS, MASK, CHOSEN_TREE, CHOSEN_P, SCORE, STATUS, N_OUT };
enum { SLOTS = N_OUT, OFFSETS, NEW_TOKENS, BUDGET_CAP, APPENDED, RESET, N_FIELDS };

Field fields[N_FIELDS] = {
    {"n_draft", c10::kInt, "int32"}, {"tokens", c10::kInt, "int32"}, {"parents", c10::kInt, "int32"},
    {"positions", c10::kInt, "int32"}, {"mask", c10::kInt, "int32"}, {"chosen_tree", c10::kInt, "int32"},
    {"chosen_p", c10::kInt, "int32"}, {"score", c10::kDouble, "float64"}, {"status", c10::kInt, "int32"},
    {"slots", c10::kInt, "int32"}, {"offsets", c10::kLong, "int64"}, {"new_tokens", c10::kInt, "int32"},
    {"budget_cap", c10::kInt, "int32"}, {"tokens", c10::kInt, "int32"}, {"reset", c10::kByte, "uint8"},
};

// A Python exception is already set where this is thrown.
struct Raised {};

void* address(PyObject* t, int field) {
    if (t == Py_None) return nullptr;
    const Field& f = fields[field];
    if (THPVariable_Check(t)) {
        const at::Tensor& v = THPVariable_Unpack(t);
        if (v.scalar_type() == f.type && v.is_cuda() && v.is_contiguous()) return v.data_ptr();
    }
    PyObject* r = PyObject_CallFunctionObjArgs(slow_ptr, t, f.py_dtype, f.key, nullptr);
    if (!r) throw Raised();
    void* p = r == Py_None ? nullptr : PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    if (!p && PyErr_Occurred()) throw Raised();
    return p;
}

int32_t length(PyObject* t) {
    if (THPVariable_Check(t)) return (int32_t)THPVariable_Unpack(t).numel();
    PyObject* r = PyObject_CallMethod(t, "numel", nullptr);
    if (!r) throw Raised();
    const long long n = PyLong_AsLongLong(r);
    Py_DECREF(r);
    if (n == -1 && PyErr_Occurred()) throw Raised();
    return (int32_t)n;
}

long long integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return v;
}

double real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised();
    return v;
}

void outputs(PyObject* out, void** p) {
    for (int k = 0; k < N_OUT; ++k) {
        PyObject* t = PyObject_GetItem(out, fields[k].key);
        if (!t) throw Raised();
        try {
            p[k] = address(t, k);
        } catch (...) {
            Py_DECREF(t);
            throw;
        }
        Py_DECREF(t);                                            // `out` holds it on
    }
}

bool count_is(Py_ssize_t n, Py_ssize_t want, const char* name) {
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "%s: %zd arguments expected, got %zd", name, want, n);
    return false;
}

sd_store* store_of(PyObject* o) {
    if (o == Py_None) return nullptr;                            // a store that was freed
    void* s = PyLong_AsVoidPtr(o);
    if (!s && PyErr_Occurred()) throw Raised();
    return (sd_store*)s;
}

sd_spec_params params(PyObject* const* a) {
    sd_spec_params p = {};
    p.P = (int32_t)integer(a[0]); p.alpha = real(a[1]); p.max_spec = (int32_t)integer(a[2]);
    p.flags = (uint32_t)integer(a[3]); p.tau = real(a[4]);
    return p;
}

// speculate(store, slots, P, alpha, max_spec, flags, tau, budget_cap, out) -> status
PyObject* speculate(PyObject*, PyObject* const* a, Py_ssize_t na) {
    HANDLE_TH_ERRORS
    if (!count_is(na, 9, "speculate")) return nullptr;
    try {
        sd_store* s = store_of(a[0]);
        const int32_t n = length(a[1]);
        const auto* slots = (const int32_t*)address(a[1], SLOTS);
        const sd_spec_params prm = params(a + 2);
        const auto* cap = (const int32_t*)address(a[7], BUDGET_CAP);
        void* o[N_OUT];
        outputs(a[8], o);
        void* st = c10::cuda::getCurrentCUDAStream().stream();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = f_speculate(s, n, slots, &prm, cap, (int32_t*)o[N_DRAFT], (int32_t*)o[TOKENS], (int32_t*)o[PARENTS],
                         (int32_t*)o[POSITIONS], (uint32_t*)o[MASK], (int32_t*)o[CHOSEN_TREE], (int32_t*)o[CHOSEN_P],
                         (double*)o[SCORE], (int32_t*)o[STATUS], st);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
    } catch (const Raised&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// step(store, slots, offsets, new_tokens, P, alpha, max_spec, flags, tau, budget_cap, out) -> status
PyObject* step(PyObject*, PyObject* const* a, Py_ssize_t na) {
    HANDLE_TH_ERRORS
    if (!count_is(na, 11, "step")) return nullptr;
    try {
        sd_store* s = store_of(a[0]);
        const int32_t n = length(a[1]);
        const auto* slots = (const int32_t*)address(a[1], SLOTS);
        const auto* off = (const int64_t*)address(a[2], OFFSETS);
        const auto* tok = (const int32_t*)address(a[3], NEW_TOKENS);
        const sd_spec_params prm = params(a + 4);
        const auto* cap = (const int32_t*)address(a[9], BUDGET_CAP);
        void* o[N_OUT];
        outputs(a[10], o);
        void* st = c10::cuda::getCurrentCUDAStream().stream();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = f_step(s, n, slots, off, tok, &prm, cap, (int32_t*)o[N_DRAFT], (int32_t*)o[TOKENS], (int32_t*)o[PARENTS],
                    (int32_t*)o[POSITIONS], (uint32_t*)o[MASK], (int32_t*)o[CHOSEN_TREE], (int32_t*)o[CHOSEN_P],
                    (double*)o[SCORE], (int32_t*)o[STATUS], st);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
    } catch (const Raised&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// append(store, slots, offsets, tokens, reset) -> status
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t na) {
    HANDLE_TH_ERRORS
    if (!count_is(na, 5, "append")) return nullptr;
    try {
        sd_store* s = store_of(a[0]);
        const int32_t n = length(a[1]);
        const auto* slots = (const int32_t*)address(a[1], SLOTS);
        const auto* off = (const int64_t*)address(a[2], OFFSETS);
        const auto* tok = (const int32_t*)address(a[3], APPENDED);
        const auto* reset = (const uint8_t*)address(a[4], RESET);
        void* st = c10::cuda::getCurrentCUDAStream().stream();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = f_append(s, n, slots, off, tok, reset, st);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
    } catch (const Raised&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// setup(addresses of sd_speculate, sd_step, sd_append, the slow way to an address)
PyObject* setup(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 4, "setup")) return nullptr;
    void* f[3];
    for (int k = 0; k < 3; ++k) {
        f[k] = PyLong_AsVoidPtr(a[k]);
        if (!f[k]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "setup: no address");
            return nullptr;
        }
    }
    PyObject* torch = PyImport_ImportModule("torch");
    if (!torch) return nullptr;
    for (Field& d : fields) {                                    // (kept for the life of the process)
        if (!d.key && !(d.key = PyUnicode_InternFromString(d.name))) return nullptr;
        if (!d.py_dtype && !(d.py_dtype = PyObject_GetAttrString(torch, d.dtype))) return nullptr;
    }
    Py_DECREF(torch);
    f_speculate = (decltype(f_speculate))f[0]; f_step = (decltype(f_step))f[1]; f_append = (decltype(f_append))f[2];
    Py_INCREF(a[3]);
    Py_XSETREF(slow_ptr, a[3]);
    Py_RETURN_NONE;
}

// ---- the verifier's calls ---------------------------------------------------------------------
// Each returns the call's result (the output it was given, or one of its own making), or the entry point's status where that is an error, or None where a tensor is
// not what is usual (its type, shape, strides or device): the same call in Python then takes it, or says what is wrong with it.  (Outputs made here: a call of one small
// request is 2 us shorter than with them made in Python.)
decltype(&sd_rotate) f_rotate;
decltype(&sd_attend) f_attend;
decltype(&sd_attend_workspace) f_attend_workspace;
decltype(&sd_accept) f_accept;
decltype(&sd_commit) f_commit;

struct Unusual {};

int32_t type_of(c10::ScalarType t) {
    if (t != c10::kBFloat16 && t != c10::kHalf && t != c10::kFloat) throw Unusual();
    return t == c10::kBFloat16 ? SD_BF16 : t == c10::kHalf ? SD_FP16 : SD_FP32;
}

const at::Tensor& cuda_tensor(PyObject* o, int device, int64_t dim) {
    if (!THPVariable_Check(o)) throw Unusual();
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != device || t.dim() != dim) throw Unusual();
    return t;
}

// A contiguous array of `type`, or null for None.
template <class T>
T* array(PyObject* o, int device, c10::ScalarType type, std::initializer_list<int64_t> shape) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = cuda_tensor(o, device, (int64_t)shape.size());
    if (t.scalar_type() != type || !t.is_contiguous()) throw Unusual();
    int64_t d = 0;
    for (const int64_t s : shape)
        if (t.size(d++) != s) throw Unusual();
    return (T*)t.data_ptr();
}

// The output `o`, or a new one like `like` where it is None; a new reference in `result`.
PyObject* made(PyObject* o, const at::Tensor& like) {
    if (o != Py_None) { Py_INCREF(o); return o; }
    return THPVariable_Wrap(at::empty(like.sizes(), like.options()));
}
PyObject* made(at::IntArrayRef shape, c10::ScalarType type, const at::Tensor& like) { return THPVariable_Wrap(at::empty(shape, like.options().dtype(type))); }

// Given back where it is not handed out.
struct Held {
    PyObject* o;
    ~Held() { Py_XDECREF(o); }
    PyObject* release() { PyObject* r = o; o = nullptr; return r; }
};

// Rows of heads: [rows][heads][head_dim] with adjacent elements.
void* heads_of(PyObject* o, int device, c10::ScalarType type, int64_t rows, int64_t heads, int64_t dim, int64_t* stride) {
    const at::Tensor& t = cuda_tensor(o, device, 3);
    if (t.scalar_type() != type || t.size(0) != rows || t.size(1) != heads || t.size(2) != dim || t.stride(2) != 1) throw Unusual();
    stride[0] = t.stride(0); stride[1] = t.stride(1);
    return t.data_ptr();
}

sd_cache cache_of(PyObject* ko, PyObject* vo, int device, bool layers) {
    if (!THPVariable_Check(ko)) throw Unusual();
    const int64_t dim = THPVariable_Unpack(ko).dim();
    if (dim != 4 && !(layers && dim == 5)) throw Unusual();
    const at::Tensor &k = cuda_tensor(ko, device, dim), &v = cuda_tensor(vo, device, dim);
    if (k.scalar_type() != v.scalar_type() || k.sizes() != v.sizes() || k.stride(dim - 1) != 1 || v.stride(dim - 1) != 1) throw Unusual();
    sd_cache c = {};
    const int64_t at = dim - 4;
    for (int64_t d = 0; d < dim; ++d)
        if (k.size(d) > 0x7FFFFFFF) throw Unusual();
    c.d_k = k.data_ptr(); c.d_v = v.data_ptr(); c.dtype = type_of(k.scalar_type());
    c.n_layers = dim == 5 ? (int32_t)k.size(0) : 1;
    c.n_pages = (int32_t)k.size(at); c.page_size = (int32_t)k.size(at + 1); c.kv_heads = (int32_t)k.size(at + 2); c.head_dim = (int32_t)k.size(at + 3);
    for (int d = 0; d < 3; ++d) { c.k_stride[d + 1] = k.stride(at + d); c.v_stride[d + 1] = v.stride(at + d); }
    if (dim == 5) { c.k_stride[0] = k.stride(0); c.v_stride[0] = v.stride(0); }
    return c;
}

// n from `offsets`, the table's and the mask's shapes; `rows` from the row arrays.
sd_rows rows_of(int64_t rows, PyObject* table, PyObject* offsets, PyObject* cached, PyObject* mask, PyObject* status, int device) {
    sd_rows b = {};
    const at::Tensor& off = cuda_tensor(offsets, device, 1);
    const int64_t n = off.size(0) - 1;
    if (n < 0 || n > 0x7FFFFFFE || rows > 0x7FFFFFFF) throw Unusual();
    b.n = (int32_t)n; b.rows = (int32_t)rows;
    b.d_offsets = array<const int64_t>(offsets, device, c10::kLong, {n + 1});
    b.d_cached = array<const int32_t>(cached, device, c10::kInt, {n});
    const at::Tensor& tab = cuda_tensor(table, device, 2);
    if (tab.size(1) > 0x7FFFFFFF) throw Unusual();
    b.table_stride = (int32_t)tab.size(1);
    b.d_table = array<const int32_t>(table, device, c10::kInt, {n, tab.size(1)});
    b.max_draft = SD_MAX_DRAFT;
    if (mask != Py_None) {
        const at::Tensor& m = cuda_tensor(mask, device, 3);
        if (m.size(1) > SD_MAX_DRAFT) throw Unusual();
        b.max_draft = (int32_t)m.size(1);
        b.d_mask = array<const uint32_t>(mask, device, c10::kInt, {n, m.size(1), (m.size(1) + 31) / 32});
    }
    b.d_status = array<int32_t>(status, device, c10::kInt, {n});
    return b;
}

#define VERIFIER_CALL(...)                                       \
    HANDLE_TH_ERRORS                                             \
    try {                                                        \
        const auto current = c10::cuda::getCurrentCUDAStream();  \
        const int device = current.device_index();               \
        void* st = current.stream();                             \
        int rc;                                                  \
        PyObject* result = nullptr;                              \
        __VA_ARGS__                                              \
        if (rc == 0) return result;                              \
        Py_XDECREF(result);                                      \
        return PyLong_FromLong(rc);                              \
    } catch (const Unusual&) {                                   \
        Py_RETURN_NONE;                                          \
    } catch (const Raised&) {                                    \
        return nullptr;                                          \
    }                                                            \
    END_HANDLE_TH_ERRORS

// rotate(q, k, v, k_cache, v_cache, table, offsets, cached, freq, mask, positions, q_weight, k_weight, eps, interleaved, scale, out, status)
PyObject* rotate(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 18, "rotate")) return nullptr;
    VERIFIER_CALL({
        const sd_cache c = cache_of(a[3], a[4], device, false);
        const at::Tensor &q = cuda_tensor(a[0], device, 3), &freq = cuda_tensor(a[8], device, 1);
        const auto type = THPVariable_Unpack(a[3]).scalar_type();
        const int64_t R = q.size(0), D = c.head_dim;
        sd_rotate_params p = {};
        if (q.size(1) > 65536 || freq.size(0) > 64) throw Unusual();
        p.q_heads = (int32_t)q.size(1); p.rot_dim = 2 * (int32_t)freq.size(0);
        p.eps = (float)real(a[13]); p.interleaved = (int32_t)integer(a[14]); p.scale = (float)real(a[15]);
        const void* dq = heads_of(a[0], device, type, R, q.size(1), D, p.q_stride);
        const void* dk = heads_of(a[1], device, type, R, c.kv_heads, D, p.k_stride);
        const void* dv = heads_of(a[2], device, type, R, c.kv_heads, D, p.v_stride);
        Held h = {made(a[16], q)};
        void* out = heads_of(h.o, device, type, R, q.size(1), D, p.out_stride);
        const sd_rows b = rows_of(R, a[5], a[6], a[7], a[9], a[17], device);
        const auto* f = array<const double>(a[8], device, c10::kDouble, {freq.size(0)});
        const auto* pos = array<const int32_t>(a[10], device, c10::kInt, {R});
        const void* qw = array<const void>(a[11], device, type, {D});
        const void* kw = array<const void>(a[12], device, type, {D});
        rc = f_rotate(&c, &b, &p, dq, dk, dv, f, pos, qw, kw, out, st);
        if (rc == 0) result = h.release();
    })
}

// attend(q, k_cache, v_cache, table, offsets, cached, mask, scale, window, sinks, shared, out, lse, status)
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 14, "attend")) return nullptr;
    VERIFIER_CALL({
        const sd_cache c = cache_of(a[1], a[2], device, false);
        const at::Tensor& q = cuda_tensor(a[0], device, 3);
        const auto type = THPVariable_Unpack(a[1]).scalar_type();
        const int64_t R = q.size(0);
        sd_attend_params p = {};
        if (q.size(1) > 65536) throw Unusual();
        p.q_heads = (int32_t)q.size(1);
        p.scale = a[7] == Py_None ? 1.0f / std::sqrt((float)std::max(c.head_dim, 1)) : (float)real(a[7]);
        const long long way[3] = {integer(a[8]), integer(a[9]), integer(a[10])};
        for (const long long w : way)
            if (w < 0 || w > 0x7FFFFFFF) throw Unusual();
        p.window = (int32_t)way[0]; p.sinks = (int32_t)way[1]; p.shared = (int32_t)way[2];
        const void* dq = heads_of(a[0], device, type, R, q.size(1), c.head_dim, p.q_stride);
        Held h = {made(a[11], q)};
        void* out = heads_of(h.o, device, type, R, q.size(1), c.head_dim, p.out_stride);
        const sd_rows b = rows_of(R, a[3], a[4], a[5], a[6], a[13], device);
        auto* lse = array<float>(a[12], device, c10::kFloat, {R, q.size(1)});
        const int64_t bytes = f_attend_workspace(&c, &b, &p);
        if (bytes < 0) rc = (int)bytes;
        else {
            const at::Tensor w = at::empty({bytes}, q.options().dtype(c10::kByte));
            rc = f_attend(&c, &b, &p, dq, out, lse, w.data_ptr(), bytes, st);
        }
        if (rc == 0) result = h.release();
    })
}

// accept(logits, offsets, tokens, parents, out, status)
PyObject* accept(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 6, "accept")) return nullptr;
    VERIFIER_CALL({
        const at::Tensor &x = cuda_tensor(a[0], device, 2), &tok = cuda_tensor(a[2], device, 2);
        const int64_t R = x.size(0), n = tok.size(0), M = tok.size(1);
        if ((x.size(1) > 1 && x.stride(1) != 1) || x.size(1) > 0x7FFFFFFF || R > 0x7FFFFFFF || n > 0x7FFFFFFE || M > SD_MAX_DRAFT) throw Unusual();
        const auto* off = array<const int64_t>(a[1], device, c10::kLong, {n + 1});
        const auto* tokens = array<const int32_t>(a[2], device, c10::kInt, {n, M});
        const auto* parents = array<const int32_t>(a[3], device, c10::kInt, {n, M});
        static PyObject* const keys[4] = {PyUnicode_InternFromString("targets"), PyUnicode_InternFromString("path"), PyUnicode_InternFromString("offsets"),
                                          PyUnicode_InternFromString("tokens")};
        Held h = {a[4] == Py_None ? PyDict_New() : (Py_INCREF(a[4]), a[4])};
        Held o[4] = {};
        for (int k = 0; k < 4; ++k) {
            if (a[4] == Py_None) {
                o[k].o = k == 0 || k == 3 ? made({R}, c10::kInt, x) : k == 1 ? made({n, M + 1}, c10::kInt, x) : made({n + 1}, c10::kLong, x);
                if (!h.o || !o[k].o || PyDict_SetItem(h.o, keys[k], o[k].o)) throw Raised();
            } else if (!(o[k].o = PyObject_GetItem(h.o, keys[k]))) throw Raised();
        }
        auto* targets = array<int32_t>(o[0].o, device, c10::kInt, {R});
        auto* path = array<int32_t>(o[1].o, device, c10::kInt, {n, M + 1});
        auto* new_offsets = array<int64_t>(o[2].o, device, c10::kLong, {n + 1});
        auto* new_tokens = array<int32_t>(o[3].o, device, c10::kInt, {R});
        auto* status = array<int32_t>(a[5], device, c10::kInt, {n});
        rc = f_accept((int32_t)n, (int32_t)R, (int32_t)M, (int32_t)x.size(1), type_of(x.scalar_type()), R > 1 ? x.stride(0) : x.size(1), x.data_ptr(), off,
                      tokens, parents, targets, path, new_offsets, new_tokens, status, st);
        if (rc == 0) result = h.release();
    })
}

// commit(k_cache, v_cache, table, cached, path, new_cached, status)
PyObject* commit(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 7, "commit")) return nullptr;
    VERIFIER_CALL({
        const sd_cache c = cache_of(a[0], a[1], device, true);
        const at::Tensor &path = cuda_tensor(a[4], device, 2), &tab = cuda_tensor(a[2], device, 2);
        const int64_t n = path.size(0), M1 = path.size(1);
        if (M1 < 1 || M1 > SD_MAX_DRAFT + 1 || n > 0x7FFFFFFE || tab.size(1) > 0x7FFFFFFF) throw Unusual();
        sd_rows b = {};
        b.n = (int32_t)n; b.max_draft = (int32_t)M1 - 1; b.table_stride = (int32_t)tab.size(1);
        b.d_table = array<const int32_t>(a[2], device, c10::kInt, {n, tab.size(1)});
        b.d_cached = array<const int32_t>(a[3], device, c10::kInt, {n});
        const auto* d_path = array<const int32_t>(a[4], device, c10::kInt, {n, M1});
        Held h = {made(a[5], cuda_tensor(a[3], device, 1))};
        auto* out = array<int32_t>(h.o, device, c10::kInt, {n});
        b.d_status = array<int32_t>(a[6], device, c10::kInt, {n});
        rc = f_commit(&c, &b, d_path, out, st);
        if (rc == 0) result = h.release();
    })
}

// setup_verifier(addresses of sd_rotate, sd_attend, sd_attend_workspace, sd_accept, sd_commit)
PyObject* setup_verifier(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 5, "setup_verifier")) return nullptr;
    void* f[5];
    for (int k = 0; k < 5; ++k) {
        f[k] = PyLong_AsVoidPtr(a[k]);
        if (!f[k]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "setup_verifier: no address");
            return nullptr;
        }
    }
    f_rotate = (decltype(f_rotate))f[0]; f_attend = (decltype(f_attend))f[1]; f_attend_workspace = (decltype(f_attend_workspace))f[2];
    f_accept = (decltype(f_accept))f[3]; f_commit = (decltype(f_commit))f[4];
    Py_RETURN_NONE;
}

#define METHOD(F) {#F, (PyCFunction)(void (*)(void))F, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(speculate), METHOD(step), METHOD(append), METHOD(setup),
                         METHOD(rotate), METHOD(attend), METHOD(accept), METHOD(commit), METHOD(setup_verifier), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_call", "The per-step calls, arguments converted natively.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__call() { return PyModule_Create(&module_def); }
