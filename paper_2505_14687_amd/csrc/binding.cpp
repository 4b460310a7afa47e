// The binding's calls in native code: an ordinary call (device tensors of a supported type, plain integers, the
// current or a given stream) is checked, its result allocated and the library entered without Python in between.  Of
// about 14 us a call took the host in Python, 8 went into attribute reads, comparisons and argument conversion.
//
// Every function returns what the call returns, or an int (the library's status where that is not GRAT_OK),
// or None: not an ordinary call, nothing has been done.  The caller then goes the long way in Python, which is where
// everything that is refused is refused, with its message.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/GradMode.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/device_lazy_init.h>

#include "grat.h"
#include "grat_sequence.h"
#include "grat_window.h"

namespace {

struct Library {   // entry points of libgrat.so, as the loader has found them
    decltype(&grat_block_list_shape) list_shape;
    decltype(&grat_build_block_lists) build_lists;
    decltype(&grat_attention_fwd) attention;
    decltype(&grat_attention_global_fwd) attention_global;
    decltype(&grat_attention_packed_fwd) attention_packed;
    decltype(&grat_dense_attention_fwd) dense;
} g_lib;

// set_library(addresses): in the order above
PyObject* set_library(PyObject*, PyObject* args) {
    unsigned long long a[6];
    if (!PyArg_ParseTuple(args, "KKKKKK", a, a + 1, a + 2, a + 3, a + 4, a + 5)) return nullptr;
    g_lib = {(decltype(g_lib.list_shape))a[0],       (decltype(g_lib.build_lists))a[1],
             (decltype(g_lib.attention))a[2],        (decltype(g_lib.attention_global))a[3],
             (decltype(g_lib.attention_packed))a[4], (decltype(g_lib.dense))a[5]};
    Py_RETURN_NONE;
}

struct SequenceLibrary {   // ... and those of grat_sequence.h
    decltype(&grat_rotary) rotary;
    decltype(&grat_rotary_append) append;
    decltype(&grat_block_means) means;
    decltype(&grat_block_scores_work) scores_work;
    decltype(&grat_block_scores) scores;
    decltype(&grat_select_blocks) select;
    decltype(&grat_selected_attention_work) attention_work;
    decltype(&grat_selected_attention_fwd) attention_fwd;
    decltype(&grat_selected_attention_bwd) attention_bwd;
} g_seq;

// set_sequence_library(addresses): in the order above
PyObject* set_sequence_library(PyObject*, PyObject* args) {
    unsigned long long a[9];
    if (!PyArg_ParseTuple(args, "KKKKKKKKK", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6, a + 7, a + 8)) return nullptr;
    g_seq = {(decltype(g_seq.rotary))a[0],         (decltype(g_seq.append))a[1],        (decltype(g_seq.means))a[2],
             (decltype(g_seq.scores_work))a[3],    (decltype(g_seq.scores))a[4],        (decltype(g_seq.select))a[5],
             (decltype(g_seq.attention_work))a[6], (decltype(g_seq.attention_fwd))a[7], (decltype(g_seq.attention_bwd))a[8]};
    Py_RETURN_NONE;
}

struct WindowLibrary {   // ... and those of grat_window.h
    decltype(&grat_window_attention_work) attention_work;
    decltype(&grat_window_attention_fwd) attention_fwd;
    decltype(&grat_window_attention_bwd) attention_bwd;
    decltype(&grat_cache_append) append;
    decltype(&grat_cache_read) read;
    decltype(&grat_cache_attention_work) cache_work;
    decltype(&grat_cache_attention_fwd) cache_attention;
} g_win;

// set_window_library(addresses): in the order above
PyObject* set_window_library(PyObject*, PyObject* args) {
    unsigned long long a[7];
    if (!PyArg_ParseTuple(args, "KKKKKKK", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6)) return nullptr;
    g_win = {(decltype(g_win.attention_work))a[0], (decltype(g_win.attention_fwd))a[1], (decltype(g_win.attention_bwd))a[2],
             (decltype(g_win.append))a[3],         (decltype(g_win.read))a[4],          (decltype(g_win.cache_work))a[5],
             (decltype(g_win.cache_attention))a[6]};
    Py_RETURN_NONE;
}

struct Unusual {};   // thrown where a call is not an ordinary one

void need(bool ok) {
    if (!ok) throw Unusual{};
}

// A plain dense tensor: no subclass, no wrapper of a transform, no lazy negation or conjugation.
const at::Tensor& tensor_of(PyObject* o) {
    need(THPVariable_CheckExact(o));
    const at::Tensor& t = THPVariable_Unpack(o);
    need(t.defined() && t.layout() == at::kStrided && t.has_storage());
    using K = c10::DispatchKey;
    const c10::DispatchKeySet keys = t.key_set();
    for (const K k : {K::Python, K::PythonTLSSnapshot, K::FuncTorchBatched, K::FuncTorchGradWrapper, K::Functionalize,
                      K::Negative, K::Conjugate, K::ZeroTensor})
        need(!keys.has(k));
    return t;
}

int64_t int_of(PyObject* o) {
    need(PyLong_CheckExact(o));
    int overflow = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
    need(overflow == 0 && v >= INT32_MIN && v <= INT32_MAX);
    return v;
}

int32_t bool_of(PyObject* o) {   // bool() as Python has it, of the kinds that cannot run code of their own
    need(PyBool_Check(o) || PyLong_CheckExact(o));
    return PyObject_IsTrue(o) ? 1 : 0;
}

float scale_of(PyObject* o) {
    need(PyFloat_CheckExact(o) || PyLong_CheckExact(o));
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Unusual{};
    }
    return (float)v;
}

struct Extents {   // of a grid, a group or a radius
    int32_t n = 0, v[3];
    explicit Extents(PyObject* o) {
        const bool list = PyList_CheckExact(o);
        need(list || PyTuple_Check(o));
        n = (int32_t)(list ? PyList_GET_SIZE(o) : PyTuple_GET_SIZE(o));
        need(n >= 1 && n <= 3);
        for (int i = 0; i < n; ++i) v[i] = (int32_t)int_of(list ? PyList_GET_ITEM(o, i) : PyTuple_GET_ITEM(o, i));
    }
};

unsigned long long attribute(PyObject* o, const char* name) {   // a whole number
    PyObject* p = PyObject_GetAttrString(o, name);
    const bool ok = p && PyLong_Check(p);
    const unsigned long long v = ok ? PyLong_AsUnsignedLongLong(p) : 0;
    Py_XDECREF(p);
    if (!ok || PyErr_Occurred()) {
        PyErr_Clear();
        throw Unusual{};
    }
    return v;
}

// The device is set up as it is ahead of every tensor that Python makes there, and nothing is done in a forked child.  The device is the current one, which
// the library works on, and the stream one of it.
hipStream_t stream_of(PyObject* o, const at::Tensor* t) {
    need(!torch::utils::is_device_in_bad_fork(at::kCUDA));
    torch::utils::device_lazy_init(at::kCUDA);
    const c10::hip::HIPStream current = c10::hip::getCurrentHIPStream();
    need(!t || t->device().index() == current.device_index());
    if (o == Py_None) return current.stream();
    need(attribute(o, "device_index") == (unsigned long long)current.device_index());
    return (hipStream_t)(uintptr_t)attribute(o, "cuda_stream");
}

grat_dtype dtype_of(const at::Tensor& t) {
    switch (t.scalar_type()) {
        case at::kBFloat16: return GRAT_BF16;
        case at::kHalf: return GRAT_F16;
        case at::kFloat: return GRAT_F32;
        default: throw Unusual{};
    }
}

void check_like(const at::Tensor& q, const at::Tensor& t) {
    need(t.sizes() == q.sizes() && t.strides() == q.strides() && t.scalar_type() == q.scalar_type() && t.device() == q.device());
}

struct Lists {
    const at::Tensor &count, &index;
    Lists(PyObject* c, PyObject* i, const Extents& grid, const Extents& group, const at::Tensor& q)
        : count(tensor_of(c)), index(tensor_of(i)) {
        need(grid.n == group.n);
        int64_t groups = 1;
        for (int k = 0; k < grid.n; ++k) {
            need(grid.v[k] >= 1 && group.v[k] >= 1 && groups < INT32_MAX);
            groups *= ((int64_t)grid.v[k] + group.v[k] - 1) / group.v[k];
        }
        for (const at::Tensor* t : {&count, &index})
            need(t->scalar_type() == at::kInt && t->is_contiguous() && t->device() == q.device());
        need(count.dim() == 1 && count.numel() == groups);
        need(index.dim() == 2 && index.size(0) == groups && index.size(1) >= 1 && index.size(1) <= INT32_MAX);
    }
    const int32_t* c() const { return (const int32_t*)count.data_ptr(); }
    const int32_t* i() const { return (const int32_t*)index.data_ptr(); }
    int32_t max_kv() const { return (int32_t)index.size(1); }
};

void check_sequence(int64_t rows, const Extents& grid, int64_t n_global) {
    __int128 n = 1;
    for (int k = 0; k < grid.n; ++k) n *= grid.v[k];
    need(n_global >= 0 && (__int128)rows == n + n_global);
}

template <typename F>
grat_status without_gil(F&& f) {
    PyThreadState* s = PyEval_SaveThread();
    const grat_status st = f();
    PyEval_RestoreThread(s);
    return st;
}

PyObject* result(grat_status st, PyObject* given, const at::Tensor& o) {
    if (st != GRAT_OK) return PyLong_FromLong((long)st);
    if (given != Py_None) {
        Py_INCREF(given);
        return given;
    }
    return THPVariable_Wrap(o);
}

// Runs f(), which returns a new reference; None where the call is not an ordinary one (or something went wrong before
// the library was entered: the long way then meets the same and reports it).
template <typename F>
PyObject* ordinary(Py_ssize_t have, Py_ssize_t want, F&& f) {
    if (have != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        need(!at::impl::torch_function_mode_enabled() && !c10::impl::TorchDispatchModeTLS::any_modes_set());
        return f();
    } catch (...) {
        if (PyErr_Occurred()) PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// attention(Q, K, V, scale, n_global or None, global_first, grid, group, kv_count, kv_index, out, stream)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return ordinary(n, 12, [&]() -> PyObject* {
        const at::Tensor &q = tensor_of(a[0]), &k = tensor_of(a[1]), &v = tensor_of(a[2]);
        need(q.dim() == 4 && q.is_cuda() && q.stride(3) == 1);
        check_like(q, k);
        check_like(q, v);
        const grat_dtype dt = dtype_of(q);
        const float scale = scale_of(a[3]);
        const bool joint = a[4] != Py_None;
        const int64_t n_global = joint ? int_of(a[4]) : 0;
        const int32_t first = joint ? bool_of(a[5]) : 1;
        const Extents grid(a[6]), group(a[7]);
        const Lists lists(a[8], a[9], grid, group, q);
        check_sequence(q.size(2), grid, n_global);
        need(q.size(0) <= INT32_MAX && q.size(1) <= INT32_MAX && q.size(3) <= INT32_MAX);
        const hipStream_t stream = stream_of(a[11], &q);
        const at::Tensor o = a[10] == Py_None ? at::empty_like(q) : tensor_of(a[10]);
        check_like(q, o);
        void *qp = q.data_ptr(), *kp = k.data_ptr(), *vp = v.data_ptr(), *op = o.data_ptr();
        const int32_t *cp = lists.c(), *ip = lists.i();
        const int32_t B = (int32_t)q.size(0), H = (int32_t)q.size(1), d = (int32_t)q.size(3);
        const int64_t sb = q.stride(0), sh = q.stride(1), sn = q.stride(2);
        return result(without_gil([&] {
            return joint ? g_lib.attention_global(qp, kp, vp, op, dt, B, H, d, sb, sh, sn, scale, (int32_t)n_global, first, grid.n, grid.v,
                                                  group.v, cp, ip, lists.max_kv(), stream)
                         : g_lib.attention(qp, kp, vp, op, dt, B, H, d, sb, sh, sn, scale, grid.n, grid.v, group.v, cp, ip,
                                           lists.max_kv(), stream);
        }), a[10], o);
    });
}

// packed(QKV, scale, n_global, global_first, grid, group, kv_count, kv_index, out, stream)
PyObject* packed(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return ordinary(n, 10, [&]() -> PyObject* {
        const at::Tensor& x = tensor_of(a[0]);
        need(x.dim() == 5 && x.size(2) == 3 && x.is_contiguous() && x.is_cuda());
        const grat_dtype dt = dtype_of(x);
        const float scale = scale_of(a[1]);
        const int64_t n_global = int_of(a[2]);
        const int32_t first = bool_of(a[3]);
        const Extents grid(a[4]), group(a[5]);
        const Lists lists(a[6], a[7], grid, group, x);
        check_sequence(x.size(1), grid, n_global);
        need(x.size(0) <= INT32_MAX && x.size(3) <= INT32_MAX && x.size(4) <= INT32_MAX);
        const hipStream_t stream = stream_of(a[9], &x);
        const std::array<int64_t, 4> shape = {x.size(0), x.size(1), x.size(3), x.size(4)};
        const at::Tensor o = a[8] == Py_None ? at::empty(shape, x.options()) : tensor_of(a[8]);
        need(o.sizes() == at::IntArrayRef(shape) && o.scalar_type() == x.scalar_type() && o.is_contiguous() && o.device() == x.device());
        void *xp = x.data_ptr(), *op = o.data_ptr();
        const int32_t *cp = lists.c(), *ip = lists.i();
        return result(without_gil([&] {
            return g_lib.attention_packed(xp, op, dt, (int32_t)shape[0], (int32_t)shape[2], (int32_t)shape[3], scale, (int32_t)n_global,
                                          first, grid.n, grid.v, group.v, cp, ip, lists.max_kv(), stream);
        }), a[8], o);
    });
}

// dense(Q, K, V, scale, out, stream)
PyObject* dense(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return ordinary(n, 6, [&]() -> PyObject* {
        const at::Tensor &q = tensor_of(a[0]), &k = tensor_of(a[1]), &v = tensor_of(a[2]);
        need(q.dim() == 4 && q.is_cuda() && q.stride(3) == 1);
        check_like(q, k);
        check_like(q, v);
        const grat_dtype dt = dtype_of(q);
        const float scale = scale_of(a[3]);
        need(q.size(0) <= INT32_MAX && q.size(1) <= INT32_MAX && q.size(3) <= INT32_MAX);
        const hipStream_t stream = stream_of(a[5], &q);
        const at::Tensor o = a[4] == Py_None ? at::empty_like(q) : tensor_of(a[4]);
        check_like(q, o);
        void *qp = q.data_ptr(), *kp = k.data_ptr(), *vp = v.data_ptr(), *op = o.data_ptr();
        return result(without_gil([&] {
            return g_lib.dense(qp, kp, vp, op, dt, (int32_t)q.size(0), (int32_t)q.size(1), q.size(2), (int32_t)q.size(3), q.stride(0),
                               q.stride(1), q.stride(2), scale, stream);
        }), a[4], o);
    });
}

// block_lists(grid, group, pattern id, radius or None, stream): (kv_count, kv_index) on the current device
PyObject* block_lists(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return ordinary(n, 5, [&]() -> PyObject* {
        const Extents grid(a[0]), group(a[1]);
        need(grid.n == group.n);
        const int64_t id = int_of(a[2]);
        need(id >= GRAT_BLOCK && id <= GRAT_DENSE);
        const grat_pattern pattern = (grat_pattern)id;
        int32_t radius[3];
        const bool has_radius = a[3] != Py_None;
        if (has_radius) {
            const Extents r(a[3]);
            need(r.n == grid.n);
            for (int k = 0; k < r.n; ++k) radius[k] = r.v[k];
        }
        const int32_t* rp = has_radius ? radius : nullptr;
        int32_t groups = 0, max_kv = 0;
        need(g_lib.list_shape(grid.n, grid.v, group.v, pattern, rp, &groups, &max_kv) == GRAT_OK && max_kv >= 1);
        const hipStream_t stream = stream_of(a[4], nullptr);
        const at::TensorOptions opt = at::TensorOptions().dtype(at::kInt).device(at::kCUDA);
        const at::Tensor count = at::empty({groups}, opt), index = at::empty({groups, max_kv}, opt);
        int32_t *cp = (int32_t*)count.data_ptr(), *ip = (int32_t*)index.data_ptr();
        const grat_status st = without_gil([&] { return g_lib.build_lists(grid.n, grid.v, group.v, pattern, rp, cp, ip, max_kv, stream); });
        if (st != GRAT_OK) return PyLong_FromLong((long)st);
        PyObject *c = THPVariable_Wrap(count), *i = THPVariable_Wrap(index);
        PyObject* pair = c && i ? PyTuple_Pack(2, c, i) : nullptr;
        Py_XDECREF(c);
        Py_XDECREF(i);
        return pair;
    });
}

// ---- token sequences (grat_sequence.h) ---------------------------------------------------------
// Calls on the current device and its current stream only: what is allocated then belongs to the stream it is used on.

// The current stream of the tensors' device, which has to be the current one.
hipStream_t current_stream(const at::Tensor& t, PyObject* given) {
    need(given == Py_None && t.is_cuda());
    return stream_of(given, &t);
}

// Nothing is recorded by autograd: a tensor that asks for a gradient is not an ordinary one (and is refused).
void no_gradient(const at::Tensor& t) { need(!(t.requires_grad() && c10::GradMode::is_enabled()) && !t._fw_grad(0).defined()); }

// A [B, H, N, d] tensor like the others.
const at::Tensor& rows_of(PyObject* o, const at::Tensor* like = nullptr) {
    const at::Tensor& t = tensor_of(o);
    need(t.dim() == 4 && t.stride(3) == 1 && t.is_cuda());
    if (like) need(t.scalar_type() == like->scalar_type() && t.device() == like->device());
    for (int i = 0; i < 4; ++i) need(t.size(i) >= 1 && t.size(i) <= INT32_MAX);
    no_gradient(t);
    return t;
}
void same_shape(const at::Tensor& a, const at::Tensor& b) { need(a.sizes() == b.sizes()); }
// (The stride of an axis of one element counts for nothing and may be any number.)
grat_tensor tensor4(const at::Tensor& t) {
    return {t.data_ptr(), t.size(0) > 1 ? t.stride(0) : 0, t.size(1) > 1 ? t.stride(1) : 0, t.size(2) > 1 ? t.stride(2) : t.size(3)};
}

// A contiguous tensor of one type and shape; null where None is given and allowed.
void* flat(PyObject* o, at::ScalarType type, at::IntArrayRef shape, const at::Tensor& like, bool optional = false) {
    if (optional && o == Py_None) return nullptr;
    const at::Tensor& t = tensor_of(o);
    no_gradient(t);
    need(t.scalar_type() == type && t.sizes() == shape && t.is_contiguous() && t.device() == like.device());
    return t.data_ptr();
}
int32_t positive(PyObject* o) {
    const int64_t v = int_of(o);
    need(v >= 1);
    return (int32_t)v;
}
int32_t groups_of(int64_t n, int64_t size) { return (int32_t)((n + size - 1) / size); }

at::Tensor scratch(int64_t bytes, const at::Tensor& like) { return at::empty({bytes}, like.options().dtype(at::kByte)); }

// New reference to a tuple of new references (taken over).
PyObject* tuple_of(std::initializer_list<PyObject*> items) {
    PyObject* t = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    bool ok = t != nullptr;
    for (PyObject* o : items) {
        ok = ok && o;
        if (t && o) PyTuple_SET_ITEM(t, i, o);
        else Py_XDECREF(o);
        ++i;
    }
    if (!ok) Py_CLEAR(t);
    return t;
}
// A tensor of the caller's has been written to: autograd then notices where it had saved it.  (Inference tensors have no version.)
void written(const at::Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
PyObject* given_or(PyObject* given, const at::Tensor& t) {
    if (given == Py_None) return THPVariable_Wrap(t);
    written(t);
    Py_INCREF(given);
    return given;
}
PyObject* sequence_result(grat_status st, PyObject* given, const at::Tensor& t) {
    return st != GRAT_OK ? PyLong_FromLong((long)st) : given_or(given, t);
}

struct Gradients {   // dQ, dK, dV: new ones, or a tuple of the caller's
    PyObject* given[3] = {Py_None, Py_None, Py_None};
    at::Tensor t[3];
    Gradients(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, PyObject* out) {
        if (out != Py_None) {
            need(PyTuple_CheckExact(out) && PyTuple_GET_SIZE(out) == 3);
            for (int i = 0; i < 3; ++i) need((given[i] = PyTuple_GET_ITEM(out, i)) != Py_None);
        }
        const at::Tensor* like[3] = {&q, &k, &v};
        for (int i = 0; i < 3; ++i) {
            t[i] = given[i] == Py_None ? at::empty_like(*like[i]) : rows_of(given[i], &q);
            same_shape(t[i], *like[i]);
        }
    }
    PyObject* result(grat_status st) const {
        if (st != GRAT_OK) return PyLong_FromLong((long)st);
        return tuple_of({given_or(given[0], t[0]), given_or(given[1], t[1]), given_or(given[2], t[2])});
    }
};

struct RotaryCall {
    grat_rotary_args args{};
    // table, positions, start, layout (0 half, 1 interleaved), axis_pairs, inverse
    RotaryCall(const at::Tensor& q, int64_t kv_heads, PyObject* table, PyObject* positions, PyObject* start, int64_t layout, PyObject* pairs,
               int32_t inverse) {
        const at::Tensor& t = tensor_of(table);
        need(t.dim() == 3 && t.size(2) == 2 && t.size(0) >= 1 && t.size(0) <= INT32_MAX && 2 * t.size(1) <= q.size(3) && t.size(1) >= 1);
        need(t.scalar_type() == at::kFloat && t.is_contiguous() && t.device() == q.device());
        no_gradient(t);
        args.dtype = dtype_of(q);
        args.batch = (int32_t)q.size(0);
        args.q_heads = (int32_t)q.size(1);
        args.kv_heads = (int32_t)kv_heads;
        args.head_dim = (int32_t)q.size(3);
        args.n_tokens = (int32_t)q.size(2);
        args.rot = (int32_t)(2 * t.size(1));
        args.interleaved = (int32_t)layout;
        args.inverse = inverse;
        args.axes = 1;
        args.axis_pairs[0] = (int32_t)t.size(1);
        if (pairs != Py_None) {
            const Extents e(pairs);
            args.axes = e.n;
            int64_t sum = 0;
            for (int i = 0; i < e.n; ++i) {
                need(e.v[i] >= 1);
                sum += args.axis_pairs[i] = e.v[i];
            }
            need(sum == t.size(1));
        }
        args.d_table = (const float*)t.data_ptr();
        args.n_pos = (int32_t)t.size(0);
        need(positions == Py_None || start == Py_None);
        if (positions != Py_None) {
            const at::Tensor& p = tensor_of(positions);
            need(p.dim() == 3 && (p.size(0) == 1 || p.size(0) == q.size(0)) && p.size(1) == q.size(2) && p.size(2) == args.axes);
            need(p.scalar_type() == at::kInt && p.is_contiguous() && p.device() == q.device());
            args.d_positions = (const int32_t*)p.data_ptr();
            args.positions_stride_b = p.size(0) > 1 ? q.size(2) * args.axes : 0;
        } else {
            need(args.axes == 1);
        }
        args.d_start = (const int32_t*)flat(start, at::kInt, {q.size(0)}, q, true);
    }
};

int64_t layout_of(PyObject* o) {
    const int64_t v = int_of(o);
    need(v == 0 || v == 1);
    return v;
}

// rotary(Q, K or None, table, positions, start, layout, axis_pairs, inverse, out or None, stream): (Q_out, K_out or None)
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return ordinary(n, 10, [&]() -> PyObject* {
        const at::Tensor& q = rows_of(a[0]);
        const bool with_k = a[1] != Py_None;
        const at::Tensor& k = with_k ? rows_of(a[1], &q) : q;
        need(k.size(0) == q.size(0) && k.size(2) == q.size(2) && k.size(3) == q.size(3));
        const RotaryCall call(q, with_k ? k.size(1) : 0, a[2], a[3], a[4], layout_of(a[5]), a[6], bool_of(a[7]));
        const hipStream_t stream = current_stream(q, a[9]);
        PyObject *gq = Py_None, *gk = Py_None;
        if (a[8] != Py_None) {
            need(PyTuple_CheckExact(a[8]) && PyTuple_GET_SIZE(a[8]) == 2);
            gq = PyTuple_GET_ITEM(a[8], 0);
            gk = PyTuple_GET_ITEM(a[8], 1);
            need(gq != Py_None && (gk != Py_None) == with_k);
        }
        const at::Tensor qo = gq == Py_None ? at::empty_like(q) : rows_of(gq, &q);
        const at::Tensor ko = !with_k ? qo : gk == Py_None ? at::empty_like(k) : rows_of(gk, &q);
        same_shape(q, qo);
        if (with_k) same_shape(k, ko);
        const grat_tensor t[4] = {tensor4(q), tensor4(qo), tensor4(k), tensor4(ko)};
        const grat_status st = without_gil([&] { return g_seq.rotary(&call.args, t, t + 1, with_k ? t + 2 : nullptr, with_k ? t + 3 : nullptr, stream); });
        if (st != GRAT_OK) return PyLong_FromLong((long)st);
        if (with_k) return tuple_of({given_or(gq, qo), given_or(gk, ko)});
        Py_INCREF(Py_None);
        return tuple_of({given_or(gq, qo), Py_None});
    });
}

// append(Q, K, V, table, K_cache, V_cache, start, layout, out, stream): Q_out
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return ordinary(n, 10, [&]() -> PyObject* {
        const at::Tensor &q = rows_of(a[0]), &k = rows_of(a[1], &q), &v = rows_of(a[2], &q), &kc = rows_of(a[4], &q), &vc = rows_of(a[5], &q);
        need(k.size(0) == q.size(0) && k.size(2) == q.size(2) && k.size(3) == q.size(3));
        same_shape(k, v);
        need(kc.size(0) == q.size(0) && kc.size(1) == k.size(1) && kc.size(3) == q.size(3));
        same_shape(kc, vc);
        need(a[6] != Py_None);
        const RotaryCall call(q, k.size(1), a[3], Py_None, a[6], layout_of(a[7]), Py_None, 0);
        const hipStream_t stream = current_stream(q, a[9]);
        const at::Tensor qo = a[8] == Py_None ? at::empty_like(q) : rows_of(a[8], &q);
        same_shape(q, qo);
        const grat_tensor t[6] = {tensor4(q), tensor4(qo), tensor4(k), tensor4(v), tensor4(kc), tensor4(vc)};
        const int32_t rows = (int32_t)kc.size(2);
        const grat_status st = without_gil([&] { return g_seq.append(&call.args, t, t + 1, t + 2, t + 3, t + 4, t + 5, rows, stream); });
        if (st == GRAT_OK) {
            written(kc);
            written(vc);
        }
        return sequence_result(st, a[8], qo);
    });
}

// means(K, block, k_len, new, out, stream)
PyObject* means(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return ordinary(n, 6, [&]() -> PyObject* {
        const at::Tensor& k = rows_of(a[0]);
        const int32_t block = positive(a[1]);
        const int64_t fresh = int_of(a[3]);
        need(fresh >= 0 && (fresh == 0 || a[4] != Py_None));
        const int64_t B = k.size(0), H = k.size(1), M = k.size(2), d = k.size(3), blocks = groups_of(M, block);
        const grat_sequence s{dtype_of(k), (int32_t)B, (int32_t)H, (int32_t)H, (int32_t)d, 1, (int32_t)M, 1, block, 0,
                              (const int32_t*)flat(a[2], at::kInt, {B}, k, true), nullptr};
        const hipStream_t stream = current_stream(k, a[5]);
        const at::Tensor out = a[4] == Py_None ? at::empty({B, H, blocks, d}, k.options().dtype(at::kFloat)) : tensor_of(a[4]);
        need(out.scalar_type() == at::kFloat && out.sizes() == at::IntArrayRef({B, H, blocks, d}) && out.is_contiguous() && out.device() == k.device());
        no_gradient(out);
        const grat_tensor t = tensor4(k);
        float* const o = (float*)out.data_ptr();
        return sequence_result(without_gil([&] { return g_seq.means(&s, &t, (int32_t)fresh, o, stream); }), a[4], out);
    });
}

// scores(Q, means, scale, q_group, block, n_k, causal, k_len, q_pos, out, stream)
PyObject* scores(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return ordinary(n, 11, [&]() -> PyObject* {
        const at::Tensor &q = rows_of(a[0]), &m = tensor_of(a[1]);
        const float scale = scale_of(a[2]);
        const int32_t q_group = positive(a[3]), block = positive(a[4]), n_k = positive(a[5]);
        need(m.dim() == 4);
        const int64_t B = q.size(0), Hkv = m.size(1), blocks = groups_of(n_k, block), groups = groups_of(q.size(2), q_group);
        need(Hkv >= 1 && q.size(1) % Hkv == 0);
        const float* const mp = (const float*)flat(a[1], at::kFloat, {B, Hkv, blocks, q.size(3)}, q);
        const grat_sequence s{dtype_of(q), (int32_t)B, (int32_t)q.size(1), (int32_t)Hkv, (int32_t)q.size(3), (int32_t)q.size(2), n_k, q_group, block,
                              bool_of(a[6]), (const int32_t*)flat(a[7], at::kInt, {B}, q, true), (const int32_t*)flat(a[8], at::kInt, {B}, q, true)};
        const hipStream_t stream = current_stream(q, a[10]);
        const int64_t bytes = g_seq.scores_work(&s);
        const at::Tensor work = bytes ? scratch(bytes, q) : at::Tensor();
        const at::Tensor out = a[9] == Py_None ? at::empty({B, Hkv, groups, blocks}, q.options().dtype(at::kFloat)) : tensor_of(a[9]);
        need(out.scalar_type() == at::kFloat && out.sizes() == at::IntArrayRef({B, Hkv, groups, blocks}) && out.is_contiguous() && out.device() == q.device());
        no_gradient(out);
        const grat_tensor t = tensor4(q);
        float* const o = (float*)out.data_ptr();
        void* const w = bytes ? work.data_ptr() : nullptr;
        return sequence_result(without_gil([&] { return g_seq.scores(&s, &t, mp, scale, o, w, stream); }), a[9], out);
    });
}

// select(scores, top, first, local, n_q, n_k, q_group, block, causal, k_len, q_pos, stream): (count, index)
PyObject* select(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return ordinary(n, 12, [&]() -> PyObject* {
        const at::Tensor& x = tensor_of(a[0]);
        need(x.dim() == 4 && x.is_cuda());
        const int32_t top = positive(a[1]), first = (int32_t)int_of(a[2]), local = (int32_t)int_of(a[3]);
        const int32_t n_q = positive(a[4]), n_k = positive(a[5]), q_group = positive(a[6]), block = positive(a[7]);
        const int64_t B = x.size(0), H = x.size(1), groups = groups_of(n_q, q_group);
        need(B >= 1 && H >= 1 && B <= INT32_MAX && H <= INT32_MAX);
        const float* const xp = (const float*)flat(a[0], at::kFloat, {B, H, groups, (int64_t)groups_of(n_k, block)}, x);
        const grat_sequence s{GRAT_BF16, (int32_t)B, (int32_t)H, (int32_t)H, 0, n_q, n_k, q_group, block, bool_of(a[8]),
                              (const int32_t*)flat(a[9], at::kInt, {B}, x, true), (const int32_t*)flat(a[10], at::kInt, {B}, x, true)};
        const hipStream_t stream = current_stream(x, a[11]);
        const at::TensorOptions opt = x.options().dtype(at::kInt);
        const at::Tensor count = at::empty({B, H, groups}, opt), index = at::empty({B, H, groups, top}, opt);
        int32_t *cp = (int32_t*)count.data_ptr(), *ip = (int32_t*)index.data_ptr();
        const grat_status st = without_gil([&] { return g_seq.select(&s, xp, top, first, local, cp, ip, stream); });
        if (st != GRAT_OK) return PyLong_FromLong((long)st);
        return tuple_of({THPVariable_Wrap(count), THPVariable_Wrap(index)});
    });
}

struct SelectedCall {   // Q, K, V, scale, count, index, q_group, block, causal, k_len, q_pos
    const at::Tensor &q, &k, &v;
    float scale;
    grat_sequence s{};
    const int32_t *count, *index;
    int32_t top;
    explicit SelectedCall(PyObject* const* a) : q(rows_of(a[0])), k(rows_of(a[1], &q)), v(rows_of(a[2], &q)), scale(scale_of(a[3])) {
        const int32_t q_group = positive(a[6]), block = positive(a[7]);
        const int64_t B = q.size(0), Hkv = k.size(1), groups = groups_of(q.size(2), q_group);
        need(k.size(0) == B && k.size(3) == q.size(3) && q.size(1) % Hkv == 0);
        same_shape(k, v);
        const at::Tensor& i = tensor_of(a[5]);
        need(i.dim() == 4 && i.size(3) >= 1 && i.size(3) <= INT32_MAX);
        top = (int32_t)i.size(3);
        count = (const int32_t*)flat(a[4], at::kInt, {B, Hkv, groups}, q);
        index = (const int32_t*)flat(a[5], at::kInt, {B, Hkv, groups, top}, q);
        s = grat_sequence{dtype_of(q), (int32_t)B, (int32_t)q.size(1), (int32_t)Hkv, (int32_t)q.size(3), (int32_t)q.size(2), (int32_t)k.size(2),
                          q_group, block, bool_of(a[8]), (const int32_t*)flat(a[9], at::kInt, {B}, q, true),
                          (const int32_t*)flat(a[10], at::kInt, {B}, q, true)};
    }
};

// selected_fwd(Q, K, V, scale, count, index, q_group, block, causal, k_len, q_pos, return_lse, out, stream): O or (O, lse)
PyObject* selected_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return ordinary(n, 14, [&]() -> PyObject* {
        const SelectedCall c(a);
        const bool with_lse = bool_of(a[11]);
        const hipStream_t stream = current_stream(c.q, a[13]);
        const int64_t bytes = g_seq.attention_work(&c.s, c.top, 0);
        const at::Tensor work = bytes ? scratch(bytes, c.q) : at::Tensor();
        const at::Tensor o = a[12] == Py_None ? at::empty_like(c.q) : rows_of(a[12], &c.q);
        same_shape(c.q, o);
        const at::Tensor lse = with_lse ? at::empty({c.q.size(0), c.q.size(1), c.q.size(2)}, c.q.options().dtype(at::kFloat)) : at::Tensor();
        const grat_tensor t[4] = {tensor4(c.q), tensor4(c.k), tensor4(c.v), tensor4(o)};
        float* const lp = with_lse ? (float*)lse.data_ptr() : nullptr;
        void* const w = bytes ? work.data_ptr() : nullptr;
        const grat_status st = without_gil([&] {
            return g_seq.attention_fwd(&c.s, t, t + 1, t + 2, t + 3, lp, c.scale, c.count, c.index, c.top, w, stream);
        });
        if (st != GRAT_OK || !with_lse) return sequence_result(st, a[12], o);
        return tuple_of({given_or(a[12], o), THPVariable_Wrap(lse)});
    });
}

// selected_bwd(Q, K, V, scale, count, index, q_group, block, causal, k_len, q_pos, dO, O, lse, out or None, stream): (dQ, dK, dV)
PyObject* selected_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return ordinary(n, 16, [&]() -> PyObject* {
        const SelectedCall c(a);
        const at::Tensor &g = rows_of(a[11], &c.q), &o = rows_of(a[12], &c.q);
        same_shape(c.q, g);
        same_shape(c.q, o);
        const float* const lse = (const float*)flat(a[13], at::kFloat, {c.q.size(0), c.q.size(1), c.q.size(2)}, c.q);
        const hipStream_t stream = current_stream(c.q, a[15]);
        Gradients d(c.q, c.k, c.v, a[14]);
        const at::Tensor work = scratch(g_seq.attention_work(&c.s, c.top, 1), c.q);
        const grat_tensor t[8] = {tensor4(g), tensor4(c.q), tensor4(c.k), tensor4(c.v), tensor4(o), tensor4(d.t[0]), tensor4(d.t[1]), tensor4(d.t[2])};
        void* const w = work.data_ptr();
        return d.result(without_gil([&] {
            return g_seq.attention_bwd(&c.s, t, t + 1, t + 2, t + 3, t + 4, lse, t + 5, t + 6, t + 7, c.scale, c.count, c.index, c.top, w, stream);
        }));
    });
}

// ---- attention within a window and over caches (grat_window.h) -----------------------------------------------------

struct Limits {   // window (None: no limit) and sinks
    int32_t window, sinks;
    Limits(PyObject* w, PyObject* f) : window(w == Py_None ? 0 : positive(w)), sinks((int32_t)int_of(f)) { need(sinks >= 0); }
};

struct WindowCall {   // Q, K, V, scale, window, sinks, causal, k_len, q_pos
    const at::Tensor &q, &k, &v;
    float scale;
    Limits limits;
    grat_sequence s{};
    explicit WindowCall(PyObject* const* a)
        : q(rows_of(a[0])), k(rows_of(a[1], &q)), v(rows_of(a[2], &q)), scale(scale_of(a[3])), limits(a[4], a[5]) {
        const int64_t B = q.size(0), Hkv = k.size(1);
        need(k.size(0) == B && k.size(3) == q.size(3) && q.size(1) % Hkv == 0);
        same_shape(k, v);
        s = grat_sequence{dtype_of(q), (int32_t)B, (int32_t)q.size(1), (int32_t)Hkv, (int32_t)q.size(3), (int32_t)q.size(2), (int32_t)k.size(2),
                          0, 0, bool_of(a[6]), (const int32_t*)flat(a[7], at::kInt, {B}, q, true), (const int32_t*)flat(a[8], at::kInt, {B}, q, true)};
    }
};

// window_fwd(Q, K, V, scale, window, sinks, causal, k_len, q_pos, return_lse, out, stream): O or (O, lse)
PyObject* window_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return ordinary(n, 12, [&]() -> PyObject* {
        const WindowCall c(a);
        const bool with_lse = bool_of(a[9]);
        const hipStream_t stream = current_stream(c.q, a[11]);
        const int64_t bytes = g_win.attention_work(&c.s, c.limits.window, c.limits.sinks, 0);
        const at::Tensor work = bytes ? scratch(bytes, c.q) : at::Tensor();
        const at::Tensor o = a[10] == Py_None ? at::empty_like(c.q) : rows_of(a[10], &c.q);
        same_shape(c.q, o);
        const at::Tensor lse = with_lse ? at::empty({c.q.size(0), c.q.size(1), c.q.size(2)}, c.q.options().dtype(at::kFloat)) : at::Tensor();
        const grat_tensor t[4] = {tensor4(c.q), tensor4(c.k), tensor4(c.v), tensor4(o)};
        float* const lp = with_lse ? (float*)lse.data_ptr() : nullptr;
        void* const w = bytes ? work.data_ptr() : nullptr;
        const grat_status st = without_gil([&] {
            return g_win.attention_fwd(&c.s, t, t + 1, t + 2, t + 3, lp, c.scale, c.limits.window, c.limits.sinks, w, stream);
        });
        if (st != GRAT_OK || !with_lse) return sequence_result(st, a[10], o);
        return tuple_of({given_or(a[10], o), THPVariable_Wrap(lse)});
    });
}

// window_bwd(Q, K, V, scale, window, sinks, causal, k_len, q_pos, dO, O, lse, out or None, stream): (dQ, dK, dV)
PyObject* window_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return ordinary(n, 14, [&]() -> PyObject* {
        const WindowCall c(a);
        const at::Tensor &g = rows_of(a[9], &c.q), &o = rows_of(a[10], &c.q);
        same_shape(c.q, g);
        same_shape(c.q, o);
        const float* const lse = (const float*)flat(a[11], at::kFloat, {c.q.size(0), c.q.size(1), c.q.size(2)}, c.q);
        const hipStream_t stream = current_stream(c.q, a[13]);
        Gradients d(c.q, c.k, c.v, a[12]);
        const at::Tensor work = scratch(g_win.attention_work(&c.s, c.limits.window, c.limits.sinks, 1), c.q);
        const grat_tensor t[8] = {tensor4(g), tensor4(c.q), tensor4(c.k), tensor4(c.v), tensor4(o), tensor4(d.t[0]), tensor4(d.t[1]), tensor4(d.t[2])};
        void* const w = work.data_ptr();
        return d.result(without_gil([&] {
            return g_win.attention_bwd(&c.s, t, t + 1, t + 2, t + 3, t + 4, lse, t + 5, t + 6, t + 7, c.scale, c.limits.window, c.limits.sinks, w, stream);
        }));
    });
}

// A cache of the dtype of `like`, or of 8 bits beside its rows' scales.
struct Cache {
    const at::Tensor &t, *scale;
    grat_tensor scales{};
    Cache(PyObject* cache, PyObject* s, const at::Tensor* like) : t(tensor_of(cache)), scale(s == Py_None ? nullptr : &tensor_of(s)) {
        need(t.dim() == 4 && t.stride(3) == 1 && t.is_cuda());
        for (int i = 0; i < 4; ++i) need(t.size(i) >= 1 && t.size(i) <= INT32_MAX);
        if (like) need(t.device() == like->device());
        no_gradient(t);
        if (!scale) {
            need(like && t.scalar_type() == like->scalar_type());
            return;
        }
        need(t.scalar_type() == at::kFloat8_e4m3fn && scale->scalar_type() == at::kFloat && scale->dim() == 3 && scale->device() == t.device());
        for (int i = 0; i < 3; ++i) need(scale->size(i) == t.size(i));
        no_gradient(*scale);
        scales = {scale->data_ptr(), t.size(0) > 1 ? scale->stride(0) : 0, t.size(1) > 1 ? scale->stride(1) : 0, t.size(2) > 1 ? scale->stride(2) : 1};
    }
    const grat_tensor* s() const { return scale ? &scales : nullptr; }
};

// cache_append(Q or None, K, V, table or None, K_cache, V_cache, start, K_scale, V_scale, positions, layout, axis_pairs, out, stream): Q_out (True where there is no Q)
PyObject* cache_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return ordinary(n, 14, [&]() -> PyObject* {
        const bool with_q = a[0] != Py_None;
        const at::Tensor &k = rows_of(a[1]), &v = rows_of(a[2], &k), &q = with_q ? rows_of(a[0], &k) : k;
        need(q.size(0) == k.size(0) && q.size(2) == k.size(2) && q.size(3) == k.size(3));
        same_shape(k, v);
        need((a[7] == Py_None) == (a[8] == Py_None) && a[3] != Py_None && a[6] != Py_None && (with_q || a[12] == Py_None));
        const Cache kc(a[4], a[7], &k), vc(a[5], a[8], &k);
        need(kc.t.size(0) == k.size(0) && kc.t.size(1) == k.size(1) && kc.t.size(3) == k.size(3));
        same_shape(kc.t, vc.t);
        RotaryCall call(q, k.size(1), a[3], a[9], Py_None, layout_of(a[10]), a[11], 0);
        call.args.d_start = (const int32_t*)flat(a[6], at::kInt, {k.size(0)}, k);
        const hipStream_t stream = current_stream(k, a[13]);
        const at::Tensor qo = !with_q ? k : a[12] == Py_None ? at::empty_like(q) : rows_of(a[12], &k);
        same_shape(q, qo);
        const grat_tensor t[6] = {tensor4(q), tensor4(qo), tensor4(k), tensor4(v), tensor4(kc.t), tensor4(vc.t)};
        const int32_t rows = (int32_t)kc.t.size(2);
        const grat_status st = without_gil([&] {
            return g_win.append(&call.args, with_q ? t : nullptr, with_q ? t + 1 : nullptr, t + 2, t + 3, t + 4, t + 5, kc.s(), vc.s(), rows, stream);
        });
        if (st != GRAT_OK) return PyLong_FromLong((long)st);
        for (const Cache* c : {&kc, &vc}) {
            written(c->t);
            if (c->scale) written(*c->scale);
        }
        if (with_q) return given_or(a[12], qo);
        Py_RETURN_TRUE;
    });
}

// cache_read(cache, scale, dtype id, k_len, out, stream)
PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return ordinary(n, 6, [&]() -> PyObject* {
        need(a[1] != Py_None);
        const Cache c(a[0], a[1], nullptr);
        const int64_t id = int_of(a[2]);
        need(id >= GRAT_BF16 && id <= GRAT_F16);
        const at::ScalarType type = id == GRAT_BF16 ? at::kBFloat16 : id == GRAT_F16 ? at::kHalf : at::kFloat;
        const int32_t* const len = (const int32_t*)flat(a[3], at::kInt, {c.t.size(0)}, c.t, true);
        const hipStream_t stream = current_stream(c.t, a[5]);
        const at::Tensor o = a[4] == Py_None ? at::empty(c.t.sizes(), c.t.options().dtype(type)) : rows_of(a[4]);
        need(o.scalar_type() == type && o.device() == c.t.device());
        same_shape(c.t, o);
        const grat_tensor t[2] = {tensor4(c.t), tensor4(o)};
        return sequence_result(without_gil([&] {
            return g_win.read((grat_dtype)id, (int32_t)c.t.size(0), (int32_t)c.t.size(1), (int32_t)c.t.size(2), (int32_t)c.t.size(3), t, c.s(), len, t + 1, stream);
        }), a[4], o);
    });
}

// cache_attention(Q, K_cache, V_cache, scale, k_len, K_scale, V_scale, parent, window, sinks, return_lse, out, stream): O or (O, lse)
PyObject* cache_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return ordinary(n, 13, [&]() -> PyObject* {
        const at::Tensor& q = rows_of(a[0]);
        need((a[5] == Py_None) == (a[6] == Py_None));
        const Cache k(a[1], a[5], &q), v(a[2], a[6], &q);
        const float scale = scale_of(a[3]);
        const int64_t B = q.size(0), N = q.size(2), Hkv = k.t.size(1);
        need(k.t.size(0) == B && k.t.size(3) == q.size(3) && q.size(1) % Hkv == 0);
        same_shape(k.t, v.t);
        const Limits limits(a[8], a[9]);
        const int32_t* parent = nullptr;
        int64_t parent_stride = 0;
        if (a[7] != Py_None) {
            const at::Tensor& p = tensor_of(a[7]);
            need(p.scalar_type() == at::kInt && p.is_contiguous() && p.device() == q.device());
            need((p.dim() == 1 && p.size(0) == N) || (p.dim() == 2 && (p.size(0) == 1 || p.size(0) == B) && p.size(1) == N));
            parent = (const int32_t*)p.data_ptr();
            parent_stride = p.dim() == 2 && p.size(0) > 1 ? N : 0;
        }
        const grat_sequence s{dtype_of(q), (int32_t)B, (int32_t)q.size(1), (int32_t)Hkv, (int32_t)q.size(3), (int32_t)N, (int32_t)k.t.size(2),
                              0, 0, 1, (const int32_t*)flat(a[4], at::kInt, {B}, q, true), nullptr};
        const bool with_lse = bool_of(a[10]);
        const hipStream_t stream = current_stream(q, a[12]);
        const int64_t bytes = g_win.cache_work(&s, limits.window, limits.sinks, k.scale ? 1 : 0);
        const at::Tensor work = bytes ? scratch(bytes, q) : at::Tensor();
        const at::Tensor o = a[11] == Py_None ? at::empty_like(q) : rows_of(a[11], &q);
        same_shape(q, o);
        const at::Tensor lse = with_lse ? at::empty({B, q.size(1), N}, q.options().dtype(at::kFloat)) : at::Tensor();
        const grat_tensor t[4] = {tensor4(q), tensor4(k.t), tensor4(v.t), tensor4(o)};
        float* const lp = with_lse ? (float*)lse.data_ptr() : nullptr;
        void* const w = bytes ? work.data_ptr() : nullptr;
        const grat_status st = without_gil([&] {
            return g_win.cache_attention(&s, t, t + 1, t + 2, k.s(), v.s(), t + 3, lp, scale, limits.window, limits.sinks, parent, parent_stride, w, stream);
        });
        if (st != GRAT_OK || !with_lse) return sequence_result(st, a[11], o);
        return tuple_of({given_or(a[11], o), THPVariable_Wrap(lse)});
    });
}

PyMethodDef kMethods[] = {
    {"set_library", set_library, METH_VARARGS, nullptr},
    {"attention", (PyCFunction)(void (*)())attention, METH_FASTCALL, nullptr},
    {"packed", (PyCFunction)(void (*)())packed, METH_FASTCALL, nullptr},
    {"dense", (PyCFunction)(void (*)())dense, METH_FASTCALL, nullptr},
    {"block_lists", (PyCFunction)(void (*)())block_lists, METH_FASTCALL, nullptr},
    {"set_sequence_library", set_sequence_library, METH_VARARGS, nullptr},
    {"rotary", (PyCFunction)(void (*)())rotary, METH_FASTCALL, nullptr},
    {"append", (PyCFunction)(void (*)())append, METH_FASTCALL, nullptr},
    {"means", (PyCFunction)(void (*)())means, METH_FASTCALL, nullptr},
    {"scores", (PyCFunction)(void (*)())scores, METH_FASTCALL, nullptr},
    {"select", (PyCFunction)(void (*)())select, METH_FASTCALL, nullptr},
    {"selected_fwd", (PyCFunction)(void (*)())selected_fwd, METH_FASTCALL, nullptr},
    {"selected_bwd", (PyCFunction)(void (*)())selected_bwd, METH_FASTCALL, nullptr},
    {"set_window_library", set_window_library, METH_VARARGS, nullptr},
    {"window_fwd", (PyCFunction)(void (*)())window_fwd, METH_FASTCALL, nullptr},
    {"window_bwd", (PyCFunction)(void (*)())window_bwd, METH_FASTCALL, nullptr},
    {"cache_append", (PyCFunction)(void (*)())cache_append, METH_FASTCALL, nullptr},
    {"cache_read", (PyCFunction)(void (*)())cache_read, METH_FASTCALL, nullptr},
    {"cache_attention", (PyCFunction)(void (*)())cache_attention, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&kModule); }
