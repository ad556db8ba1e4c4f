// The short way from Python to the entry points of include/spin.h: a CPython extension that reads the tensors' pointers, allocates
// the results and calls the library, for well-formed arguments.  A call of the ctypes binding spends 1 to 2.7 us on looking at its
// arguments and up to 2.5 on allocating in Python, as long as its kernels run on the smallest inputs: a 64^3 layer of three parties
// (two sharings, a product, a truncation) took 22 us back to back, of which its kernels are 12.
//
// Every function returns the result, or None for whatever it does not take (other types, shapes that disagree, an `out` that is too short, subclasses, modes that
// look at calls, workspaces beyond what needs no look at the device's memory, no memory left): spin.py then goes the way that
// says what is wrong, or does it.  A status of the library other than SPIN_OK comes back as an int.  Nothing is kept between calls but the
// addresses of the library's functions.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <array>
#include <vector>

#include "../../include/spin.h"

namespace {

// The calls that exist for 64- and 32-bit words.
template <class T> struct ByWord;
template <> struct ByWord<uint64_t> {
    static constexpr at::ScalarType type = at::kLong;
    static constexpr int bits = 64;
    decltype(&spin_cache_append) append;
    decltype(&spin_cache_copy) copy;
    decltype(&spin_cache_compact) compact;
    decltype(&spin_cache_scores) scores;
    decltype(&spin_cache_values) values;
    decltype(&spin_cache_values_workspace_bytes) values_bytes;
    decltype(&spin_relbias_trunc) bias;
    decltype(&spin_relbias_grad) grad;
    decltype(&spin_linattn_scores) linattn_scores;
    decltype(&spin_linattn_states) linattn_states;
    decltype(&spin_linattn_states_workspace_bytes) linattn_states_bytes;
    decltype(&spin_linattn_outputs) linattn_outputs;
    decltype(&spin_linattn_step) linattn_step;
    decltype(&spin_layernorm) norm;
    decltype(&spin_layernorm_grad) norm_grad;
    decltype(&spin_layernorm_grad_workspace_bytes) norm_grad_bytes;
};
template <> struct ByWord<uint32_t> {
    static constexpr at::ScalarType type = at::kInt;
    static constexpr int bits = 32;
    decltype(&spin32_cache_append) append;
    decltype(&spin32_cache_copy) copy;
    decltype(&spin32_cache_compact) compact;
    decltype(&spin32_cache_scores) scores;
    decltype(&spin32_cache_values) values;
    decltype(&spin32_cache_values_workspace_bytes) values_bytes;
    decltype(&spin32_relbias_trunc) bias;
    decltype(&spin32_relbias_grad) grad;
    decltype(&spin32_linattn_scores) linattn_scores;
    decltype(&spin32_linattn_states) linattn_states;
    decltype(&spin32_linattn_states_workspace_bytes) linattn_states_bytes;
    decltype(&spin32_linattn_outputs) linattn_outputs;
    decltype(&spin32_linattn_step) linattn_step;
    decltype(&spin32_layernorm) norm;
    decltype(&spin32_layernorm_grad) norm_grad;
    decltype(&spin32_layernorm_grad_workspace_bytes) norm_grad_bytes;
};
struct Library {
    decltype(&spin_share) share, bshare;
    decltype(&spin_open) open, bopen;
    decltype(&spin_beaver_mul) beaver_mul, beaver_and;
    decltype(&spin_trunc) trunc;
    decltype(&spin_beaver_matmul) matmul, matmul_nt;
    decltype(&spin_beaver_matmul_preferred_workspace_bytes) matmul_preferred;
    decltype(&spin_beaver_matmul_grouped) grouped;
    decltype(&spin_beaver_matmul_grouped_workspace_bytes) grouped_bytes;
    decltype(&spin_completed_square_trunc) completed_square;
    ByWord<uint64_t> wide;
    ByWord<uint32_t> narrow;
} lib;
template <class T> inline const ByWord<T> &by_word()
{
    if constexpr (sizeof(T) == 8) return lib.wide;
    else return lib.narrow;
}
constexpr int kEntries = sizeof(Library) / sizeof(void *);
size_t unasked_bytes;                                    // workspaces up to this size are taken without a look at the device's memory

// ---- arguments ------------------------------------------------------------------------------------------------
// A contiguous int64 CUDA tensor with memory of its own; null for anything else.
inline const at::Tensor *ring_tensor(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.has_storage() || !t.is_cuda() || t.scalar_type() != at::kLong || !t.is_contiguous()) return nullptr;
    return &t;
}
inline uint64_t *words(const at::Tensor &t) { return (uint64_t *)t.mutable_data_ptr(); }

// Plain ints only; 64-bit ones wrap as they do in ctypes.
inline bool word(PyObject *o, uint64_t &v)
{
    if (!PyLong_CheckExact(o)) return false;
    v = PyLong_AsUnsignedLongLongMask(o);
    return true;
}
inline bool integer(PyObject *o, int least, int most, int &v)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    const long n = PyLong_AsLongAndOverflow(o, &overflow);
    if (overflow || n < least || n > most) return false;
    v = (int)n;
    return true;
}
inline bool parties(int64_t n) { return n >= 1 && n <= SPIN_MAX_PARTIES; }

PyObject *none() { Py_RETURN_NONE; }

// The interpreter's lock is given up for a library call, and taken again however that ends: guarded() answers exceptions with it.
struct Unlocked {
    PyThreadState *state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};
// The call on torch's current stream (which is asked for before: that may throw).
template <class F> inline spin_status unlocked(F &&call)
{
    const spin_stream stream = (spin_stream)c10::hip::getCurrentHIPStream(c10::hip::current_device()).stream();
    const Unlocked scope;
    return call(stream);
}
// The result, or the status as an int.
template <class F> inline PyObject *run(const at::Tensor &result, F &&call)
{
    const spin_status st = unlocked(call);
    return st == SPIN_OK ? THPVariable_Wrap(result) : PyLong_FromLong(st);
}

// What a function's body throws (torch's allocator, above all) is left to the long way.
template <class F> inline PyObject *guarded(F &&body)
{
    if (at::impl::torch_function_mode_enabled()) return none();
    try {
        return body();
    } catch (...) {
        PyErr_Clear();
        return none();
    }
}

// ---- calls ----------------------------------------------------------------------------------------------------
// (x, n, seed, stream_id, out)
PyObject *sharing(PyObject *const *a, Py_ssize_t count, decltype(lib.share) fn)
{
    return guarded([&]() -> PyObject * {
        const at::Tensor *x = count == 5 ? ring_tensor(a[0]) : nullptr, *out = nullptr;
        int n;
        uint64_t seed, stream_id;
        if (!x || !integer(a[1], 1, SPIN_MAX_PARTIES, n) || !word(a[2], seed) || !word(a[3], stream_id)) return none();
        if (a[4] != Py_None && (!(out = ring_tensor(a[4])) || out->numel() < n * x->numel())) return none();
        at::Tensor fresh;
        if (!out) {
            c10::SmallVector<int64_t, 8> shape{n};
            shape.append(x->sizes().begin(), x->sizes().end());
            fresh = at::empty(shape, x->options());
            out = &fresh;
        }
        const uint64_t *from = words(*x);
        uint64_t *to = words(*out);
        const size_t each = (size_t)x->numel();
        return run(*out, [&](spin_stream s) { return fn(from, each, n, seed, stream_id, to, s); });
    });
}

// (shares, mask, out)
PyObject *opening(PyObject *const *a, Py_ssize_t count, decltype(lib.open) fn)
{
    return guarded([&]() -> PyObject * {
        const at::Tensor *shares = count == 3 ? ring_tensor(a[0]) : nullptr, *mask = nullptr, *out = nullptr;
        if (!shares || shares->dim() < 1 || !parties(shares->size(0))) return none();
        if (a[1] != Py_None && (!(mask = ring_tensor(a[1])) || mask->sizes() != shares->sizes())) return none();
        // the library reads the number of elements off `out`
        if (a[2] != Py_None && (!(out = ring_tensor(a[2])) || out->numel() != shares->numel() / shares->size(0))) return none();
        at::Tensor fresh;
        if (!out) {
            fresh = at::empty(shares->sizes().slice(1), shares->options());
            out = &fresh;
        }
        const uint64_t *from = words(*shares), *masks = mask ? words(*mask) : nullptr;
        uint64_t *to = words(*out);
        const size_t each = (size_t)out->numel();
        const int n = (int)shares->size(0);
        return run(*out, [&](spin_stream s) { return fn(from, masks, each, n, to, s); });
    });
}

// the first `inputs` of a are tensors of one shape, the next but `extra` is out
template <int INPUTS, class F> inline PyObject *elementwise(PyObject *const *a, PyObject *out_arg, F &&call)
{
    const at::Tensor *t[INPUTS], *out = nullptr;
    for (int i = 0; i < INPUTS; ++i) {
        t[i] = ring_tensor(a[i]);
        if (!t[i] || t[i]->sizes() != t[0]->sizes()) return none();
    }
    if (t[0]->dim() < 1 || !parties(t[0]->size(0))) return none();
    if (out_arg != Py_None && (!(out = ring_tensor(out_arg)) || out->numel() < t[0]->numel())) return none();
    at::Tensor fresh;
    if (!out) {
        fresh = at::empty(t[0]->sizes(), t[0]->options());
        out = &fresh;
    }
    const uint64_t *v[INPUTS];
    for (int i = 0; i < INPUTS; ++i) v[i] = words(*t[i]);
    uint64_t *to = words(*out);
    const int n = (int)t[0]->size(0);
    const size_t each = (size_t)(t[0]->numel() / n);
    return run(*out, [&](spin_stream s) { return call(n, each, v, to, s); });
}

// (x, y, a, b, c, out)
PyObject *multiplying(PyObject *const *a, Py_ssize_t count, decltype(lib.beaver_mul) fn)
{
    return guarded([&]() -> PyObject * {
        if (count != 6) return none();
        return elementwise<5>(a, a[5], [&](int n, size_t each, const uint64_t *const *v, uint64_t *out, spin_stream s) {
            return fn(n, each, v[0], v[1], v[2], v[3], v[4], out, s);
        });
    });
}

// (x, r, r_top, r_msb, f, out)
PyObject *truncating(PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        int f;
        if (count != 6 || !integer(a[4], 1, 61, f)) return none();
        return elementwise<4>(a, a[5], [&](int n, size_t each, const uint64_t *const *v, uint64_t *out, spin_stream s) {
            return lib.trunc(n, each, f, v[0], v[1], v[2], v[3], out, s);
        });
    });
}

struct Product {
    const at::Tensor *X, *Y, *A, *B, *C, *out;
    at::Tensor fresh;
    int n, batch, M, N, K;
};
// X, Y, A, B, C (null or of another shape than they should have: false) and out or None; allocates out.
inline bool product(PyObject *const *a, PyObject *out, bool transposed, Product &p)
{
    if (!(p.X = ring_tensor(a[0])) || !(p.Y = ring_tensor(a[1])) || !(p.A = ring_tensor(a[2])) || !(p.B = ring_tensor(a[3])) ||
        !(p.C = ring_tensor(a[4])) || p.X->dim() != 4 || p.Y->dim() != 4)
        return false;
    const int64_t n = p.X->size(0), batch = p.X->size(1), M = p.X->size(2), K = p.X->size(3), N = p.Y->size(transposed ? 2 : 3);
    if (!parties(n) || std::max({batch, M, N, K}) > 0x7fffffff) return false;
    const std::array<int64_t, 4> y{n, batch, transposed ? N : K, transposed ? K : N}, z{n, batch, M, N};
    if (p.Y->sizes() != at::IntArrayRef(y) || p.A->sizes() != p.X->sizes() || p.B->sizes() != p.Y->sizes() || p.C->sizes() != at::IntArrayRef(z))
        return false;
    p.out = nullptr;
    if (out != Py_None && (!(p.out = ring_tensor(out)) || p.out->numel() < p.C->numel())) return false;
    if (!p.out) {
        p.fresh = at::empty(p.C->sizes(), p.C->options());
        p.out = &p.fresh;
    }
    p.n = (int)n, p.batch = (int)batch, p.M = (int)M, p.N = (int)N, p.K = (int)K;
    return true;
}
// workspace: a contiguous CUDA tensor
inline const at::Tensor *workspace_tensor(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.defined() && t.has_storage() && t.is_cuda() && t.is_contiguous() ? &t : nullptr;
}

// (X, Y, A, B, C, path, out, workspace, y_transposed)
PyObject *matmul(PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        int path;
        Product p;
        if (count != 9 || !integer(a[5], 0, 1, path) || !PyBool_Check(a[8])) return none();
        const bool transposed = a[8] == Py_True;
        if (!product(a, a[6], transposed, p)) return none();
        const at::Tensor *ws = nullptr;
        at::Tensor fresh;
        if (a[7] != Py_None) {
            if (!(ws = workspace_tensor(a[7]))) return none();
        } else {
            const size_t size = lib.matmul_preferred(p.n, p.batch, p.M, p.N, p.K, path);
            if (size == 0 || size > unasked_bytes) return none();
            fresh = at::empty({(int64_t)size}, p.X->options().dtype(at::kByte));
            ws = &fresh;
        }
        auto fn = transposed ? lib.matmul_nt : lib.matmul;
        const uint64_t *X = words(*p.X), *Y = words(*p.Y), *A = words(*p.A), *B = words(*p.B), *C = words(*p.C);
        uint64_t *Z = words(*p.out);
        void *space = ws->mutable_data_ptr();
        const size_t bytes = (size_t)ws->numel() * ws->element_size();
        return run(*p.out, [&](spin_stream s) { return fn(p.n, p.batch, p.M, p.N, p.K, X, Y, A, B, C, Z, path, space, bytes, s); });
    });
}

// (groups, path, workspace): a list of dicts
PyObject *grouped(PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        int path;
        if (count != 3 || !PyList_CheckExact(a[0]) || !integer(a[1], 0, 1, path)) return none();
        const Py_ssize_t groups = PyList_GET_SIZE(a[0]);
        if (groups < 1 || groups > SPIN_MAX_GROUPS) return none();
        static PyObject *keys[7];
        if (!keys[0]) {
            const char *names[7] = {"X", "Y", "A", "B", "C", "out", "y_transposed"};
            for (int i = 6; i >= 0; --i) keys[i] = PyUnicode_InternFromString(names[i]);
        }
        std::vector<Product> p((size_t)groups);
        std::vector<spin_matmul_group> desc((size_t)groups);
        for (Py_ssize_t i = 0; i < groups; ++i) {
            PyObject *g = PyList_GET_ITEM(a[0], i), *v[7];
            if (!PyDict_CheckExact(g)) return none();
            for (int k = 0; k < 7; ++k) {
                v[k] = PyDict_GetItemWithError(g, keys[k]);
                if (!v[k] && (k < 5 || PyErr_Occurred())) return PyErr_Clear(), none();
            }
            if (v[6] && !PyBool_Check(v[6])) return none();
            const bool transposed = v[6] == Py_True;
            if (!product(v, v[5] ? v[5] : Py_None, transposed, p[i]) || p[i].n != p[0].n) return none();
            desc[i] = spin_matmul_group{p[i].batch, p[i].M, p[i].N, p[i].K, words(*p[i].X), words(*p[i].Y), words(*p[i].A), words(*p[i].B),
                                        words(*p[i].C), words(p[i].fresh.defined() ? p[i].fresh : *p[i].out), transposed ? 1 : 0};
        }
        const size_t need = lib.grouped_bytes(p[0].n, (int)groups, desc.data(), path);
        if (need == 0) return none();
        const at::Tensor *ws = nullptr;
        at::Tensor fresh;
        if (a[2] != Py_None) {
            if (!(ws = workspace_tensor(a[2]))) return none();
        } else {
            fresh = at::empty({(int64_t)need}, p[0].X->options().dtype(at::kByte));
            ws = &fresh;
        }
        void *space = ws->mutable_data_ptr();
        const size_t bytes = (size_t)ws->numel() * ws->element_size();
        THPObjectPtr list(PyList_New(groups));
        if (!list) return PyErr_Clear(), none();
        for (Py_ssize_t i = 0; i < groups; ++i) {
            PyObject *out = PyDict_GetItemWithError(PyList_GET_ITEM(a[0], i), keys[5]);
            PyObject *z = p[i].fresh.defined() ? THPVariable_Wrap(p[i].fresh) : Py_NewRef(out);
            if (!z) return PyErr_Clear(), none();
            PyList_SET_ITEM(list.get(), i, z);
        }
        const spin_status st = unlocked([&](spin_stream s) { return lib.grouped(p[0].n, (int)groups, desc.data(), path, space, bytes, s); });
        return st == SPIN_OK ? list.release() : PyLong_FromLong(st);
    });
}

// (x, t3, t2, lin, t0, triples, tuples, f, out): triples and tuples two sequences of three tensors
PyObject *completed_square(PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        uint64_t c[4];
        int f[2];
        if (count != 9 || !PyTuple_CheckExact(a[7]) || PyTuple_GET_SIZE(a[7]) != 2) return none();
        for (int i = 0; i < 4; ++i)
            if (!word(a[1 + i], c[i])) return none();
        for (int i = 0; i < 2; ++i)
            if (!integer(PyTuple_GET_ITEM(a[7], i), 1, 61, f[i])) return none();
        PyObject *t[13] = {a[0]};
        int filled = 1;
        for (int k = 0; k < 2; ++k) {
            PyObject *two = a[5 + k];
            if (!PyList_CheckExact(two) && !PyTuple_CheckExact(two)) return none();
            if (PySequence_Fast_GET_SIZE(two) != 2) return none();
            for (int i = 0; i < 2; ++i) {
                PyObject *three = PySequence_Fast_GET_ITEM(two, i);
                if (!PyTuple_CheckExact(three) || PyTuple_GET_SIZE(three) != 3) return none();
                for (int j = 0; j < 3; ++j) t[filled++] = PyTuple_GET_ITEM(three, j);
            }
        }
        return elementwise<13>(t, a[8], [&](int n, size_t each, const uint64_t *const *v, uint64_t *out, spin_stream s) {
            return lib.completed_square(n, each, v[0], c[0], c[1], c[2], c[3], v + 1, v + 7, f, out, s);
        });
    });
}

// ---- a paged cache, attention over it, relative position bias: (word bits, the arguments of the calls in spin.py) -------------
using Shape = at::IntArrayRef;
template <class T> inline const at::Tensor *word_tensor(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.has_storage() || !t.is_cuda() || t.scalar_type() != ByWord<T>::type || !t.is_contiguous()) return nullptr;
    return &t;
}
template <class T> inline const at::Tensor *word_tensor(PyObject *o, Shape shape)
{
    const at::Tensor *t = word_tensor<T>(o);
    return t && t->sizes() == shape ? t : nullptr;
}
// A device list of int32_t (as the 32-bit words are); absent lists stay null.
inline bool list_of(PyObject *o, Shape shape, const int32_t *&to)
{
    to = nullptr;
    if (o == Py_None) return true;
    const at::Tensor *t = word_tensor<uint32_t>(o, shape);
    if (t) to = (const int32_t *)t->const_data_ptr();
    return t != nullptr;
}
template <class T> inline T *data(const at::Tensor *t) { return (T *)t->mutable_data_ptr(); }
inline bool sequence(PyObject *o, Py_ssize_t count) { return (PyTuple_CheckExact(o) || PyList_CheckExact(o)) && PySequence_Fast_GET_SIZE(o) == count; }
inline bool fits(std::initializer_list<int64_t> sizes)
{
    for (int64_t v : sizes)
        if (v < 1 || v > 0x7fffffff) return false;
    return true;
}
// The cache of K and V (one of them may be null) and, where it is looked at, its table of `batch` sequences.
template <class T> inline bool cache_of(const at::Tensor *K, const at::Tensor *V, PyObject *table, int64_t batch, spin_cache &c)
{
    const at::Tensor *pool = K ? K : V;
    if (!pool || pool->dim() != 5 || (K && V && K->sizes() != V->sizes())) return false;
    const Shape s = pool->sizes();
    if (!fits({s[1], s[2], s[3], s[4]}) || !parties(s[0] - 1)) return false;
    c = spin_cache{(int)s[0] - 1, (int)s[1], (int)s[2], (int)s[3], (int)s[4], K ? data<T>(K) : nullptr, V ? data<T>(V) : nullptr, (int)batch, 0, nullptr};
    if (!table) return true;
    const at::Tensor *t = word_tensor<uint32_t>(table);
    if (!t || t->dim() != 2 || t->size(0) != batch || !fits({batch, t->size(1)})) return false;
    c.table_pages = (int)t->size(1);
    c.table = (const int32_t *)t->const_data_ptr();
    return true;
}
template <class T> inline bool pools_of(PyObject *o, const at::Tensor *&K, const at::Tensor *&V)
{
    return sequence(o, 2) && (K = word_tensor<T>(PySequence_Fast_GET_ITEM(o, 0))) && (V = word_tensor<T>(PySequence_Fast_GET_ITEM(o, 1)));
}
template <class T> inline bool tuple_of(PyObject *o, int f, Shape shape, const T *(&r)[3])
{
    for (int k = 0; k < 3; ++k) r[k] = nullptr;
    if (f == 0) return true;
    if (!sequence(o, 3)) return false;
    for (int k = 0; k < 3; ++k) {
        const at::Tensor *t = word_tensor<T>(PySequence_Fast_GET_ITEM(o, k), shape);
        if (!t) return false;
        r[k] = data<T>(t);
    }
    return true;
}
inline bool bucketing(PyObject *o, int64_t buckets, spin_relbias &v)
{
    const at::Tensor *t = word_tensor<uint32_t>(o);
    if (!t || t->dim() != 1 || t->numel() % 2 == 0 || !fits({buckets, t->numel()})) return false;
    v = spin_relbias{(int)buckets, (int)(t->numel() / 2), (const int32_t *)t->const_data_ptr(), nullptr};
    return true;
}
template <class T> inline bool bias_of(PyObject *table, PyObject *bucket_of, int64_t n, int64_t heads, spin_relbias &v)
{
    const at::Tensor *t = word_tensor<T>(table);
    if (!t || t->dim() != 3 || t->size(0) != n || t->size(1) != heads || !bucketing(bucket_of, t->size(2), v)) return false;
    v.table = data<T>(t);
    return true;
}
// `out` or a fresh tensor of that shape.
template <class T> struct Result {
    const at::Tensor *t = nullptr;
    at::Tensor fresh;
    bool take(PyObject *out, Shape shape, const at::Tensor &like)
    {
        int64_t words = 1;
        for (int64_t v : shape) words *= v;
        if (out != Py_None) return (t = word_tensor<T>(out)) && t->numel() >= words;
        fresh = at::empty(shape, like.options());
        t = &fresh;
        return true;
    }
};
inline PyObject *answer(spin_status st, PyObject *result) { return st == SPIN_OK ? Py_NewRef(result) : PyLong_FromLong(st); }

template <class T> PyObject *cache_append(PyObject *const *a)      // pools, table, start, x, b, count
{
    const at::Tensor *K, *V, *Kx, *Vx, *Kb, *Vb;
    spin_cache c;
    const int32_t *start, *count;
    if (!pools_of<T>(a[0], K, V) || !pools_of<T>(a[3], Kx, Vx) || !pools_of<T>(a[4], Kb, Vb) || Kx->dim() != 5) return none();
    const Shape s = Kx->sizes();
    if (Vx->sizes() != s || Kb->sizes() != s || Vb->sizes() != s || !fits({s[1], s[3]}) || !cache_of<T>(K, V, a[1], s[1], c)) return none();
    if (c.n != s[0] || c.heads != s[2] || c.dim != s[4] || !list_of(a[2], s.slice(1, 1), start) || !start || !list_of(a[5], s.slice(1, 1), count)) return none();
    const int rows = (int)s[3];
    const T *p[4] = {data<T>(Kx), data<T>(Kb), data<T>(Vx), data<T>(Vb)};
    return answer(unlocked([&](spin_stream q) { return by_word<T>().append(&c, rows, start, count, p[0], p[1], p[2], p[3], q); }), a[0]);
}
template <class T> PyObject *cache_copy(PyObject *const *a)        // pools, src, dst
{
    const at::Tensor *K, *V, *src = word_tensor<uint32_t>(a[1]);
    spin_cache c;
    const int32_t *from, *to;
    if (!src || src->dim() != 1 || !fits({src->numel()}) || !pools_of<T>(a[0], K, V) || !cache_of<T>(K, V, nullptr, 0, c)) return none();
    if (!list_of(a[1], src->sizes(), from) || !list_of(a[2], src->sizes(), to) || !to) return none();
    const int pairs = (int)src->numel();
    return answer(unlocked([&](spin_stream q) { return by_word<T>().copy(&c, pairs, from, to, q); }), a[0]);
}
template <class T> PyObject *cache_compact(PyObject *const *a)     // pools, table, context, kept, kept_count
{
    const at::Tensor *K, *V, *kept = word_tensor<uint32_t>(a[3]);
    spin_cache c;
    const int32_t *context, *list, *count;
    if (!kept || kept->dim() != 2 || !fits({kept->size(0), kept->size(1)}) || !pools_of<T>(a[0], K, V) || !cache_of<T>(K, V, a[1], kept->size(0), c)) return none();
    const Shape b = kept->sizes().slice(0, 1);
    if (!list_of(a[2], b, context) || !context || !list_of(a[3], kept->sizes(), list) || !list_of(a[4], b, count) || !count) return none();
    const int nodes = (int)kept->size(1);
    return answer(unlocked([&](spin_stream q) { return by_word<T>().compact(&c, nodes, context, list, count, q); }), a[0]);
}
// What scores and values share: x, A (of `last` words a row), C, tuple, tree.
template <class T> struct Attention {
    spin_cache c;
    const at::Tensor *x, *A, *C;
    const T *r[3];
    const uint64_t *tree = nullptr;
    const int32_t *context;
    int f;
    Shape rows;
    bool take(PyObject *pool, bool keys, PyObject *table, PyObject *ctx, PyObject *px, PyObject *pA, PyObject *pC, PyObject *pf, PyObject *tup, PyObject *ptree)
    {
        x = word_tensor<T>(px), C = word_tensor<T>(pC);
        if (!x || !C || x->dim() != 5 || C->dim() != 5 || !(A = word_tensor<T>(pA, x->sizes())) || !integer(pf, 0, ByWord<T>::bits - 3, f)) return false;
        rows = x->sizes().slice(0, 4);
        const at::Tensor *p = word_tensor<T>(pool);
        if (C->sizes().slice(0, 4) != rows || !fits({rows[1], rows[2], rows[3], x->size(4), C->size(4)}) ||
            !cache_of<T>(keys ? p : nullptr, keys ? nullptr : p, table, rows[1], c))
            return false;
        if (c.n != rows[0] || c.dim != (keys ? x : C)->size(4) || !list_of(ctx, rows.slice(1, 1), context) || !context || !tuple_of<T>(tup, f, C->sizes(), r)) return false;
        if (ptree == Py_None) return true;
        const int64_t shape[2] = {rows[1], rows[3]};
        const at::Tensor *t = word_tensor<uint64_t>(ptree, Shape(shape, 2));
        if (t) tree = data<uint64_t>(t);
        return t != nullptr;
    }
};
template <class T> PyObject *cache_scores(PyObject *const *a)      // K, table, context, Q, A, C, f, tuple, tree, masked, bias, depth, out
{
    Attention<T> v;
    Result<T> out;
    spin_relbias bias;
    const int32_t *depth = nullptr;
    uint64_t masked;
    if (!v.take(a[0], true, a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8]) || !word(a[9], masked)) return none();
    const bool biased = a[10] != Py_None;
    const int64_t nodes[2] = {v.rows[1], v.rows[3]};
    if (biased && (!sequence(a[10], 2) || !bias_of<T>(PySequence_Fast_GET_ITEM(a[10], 0), PySequence_Fast_GET_ITEM(a[10], 1), v.rows[0], v.rows[2], bias) ||
                   !list_of(a[11], Shape(nodes, 2), depth)))
        return none();
    if (!out.take(a[12], v.C->sizes(), *v.C)) return none();
    const T *Q = data<T>(v.x), *A = data<T>(v.A), *C = data<T>(v.C);
    T *to = data<T>(out.t);
    return run(*out.t, [&](spin_stream q) {
        return by_word<T>().scores(&v.c, (int)v.rows[2], (int)v.rows[3], (int)v.C->size(4), v.f, v.context, v.tree, Q, A, C, v.r[0], v.r[1], v.r[2], (T)masked,
                                   biased ? &bias : nullptr, depth, to, q);
    });
}
template <class T> PyObject *cache_values(PyObject *const *a)      // V, table, context, P, A, C, f, tuple, tree, out, workspace
{
    Attention<T> v;
    Result<T> out;
    if (!v.take(a[0], false, a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8]) || !out.take(a[9], v.C->sizes(), *v.C)) return none();
    const int heads = (int)v.rows[2], nodes = (int)v.rows[3], columns = (int)v.x->size(4);
    const at::Tensor *ws = nullptr;
    at::Tensor fresh;
    if (a[10] != Py_None) {
        if (!(ws = workspace_tensor(a[10]))) return none();
    } else {
        const size_t size = by_word<T>().values_bytes(&v.c, heads, nodes, columns);
        if (size == 0 || size > unasked_bytes) return none();
        fresh = at::empty({(int64_t)size}, v.x->options().dtype(at::kByte));
        ws = &fresh;
    }
    const T *P = data<T>(v.x), *A = data<T>(v.A), *C = data<T>(v.C);
    T *to = data<T>(out.t);
    void *space = ws->mutable_data_ptr();
    const size_t bytes = (size_t)ws->numel() * ws->element_size();
    return run(*out.t, [&](spin_stream q) {
        return by_word<T>().values(&v.c, heads, nodes, columns, v.f, v.context, v.tree, P, A, C, v.r[0], v.r[1], v.r[2], to, space, bytes, q);
    });
}
template <class T> struct Pairs {                          // x [n, batch, heads, Q, K], first, causal, lengths
    const at::Tensor *x;
    int d[5], first;
    const int32_t *lengths;
    bool take(PyObject *px, PyObject *pfirst, PyObject *causal, PyObject *plengths)
    {
        x = word_tensor<T>(px);
        if (!x || x->dim() != 5 || !PyBool_Check(causal) || !integer(pfirst, -0x7fffffff, 0x7fffffff, first)) return false;
        const Shape s = x->sizes();
        if (!parties(s[0]) || !fits({s[1], s[2], s[3], s[4]}) || !list_of(plengths, s.slice(1, 1), lengths)) return false;
        for (int k = 0; k < 5; ++k) d[k] = (int)s[k];
        return true;
    }
};
template <class T> PyObject *relbias_trunc(PyObject *const *a)     // x, bias, bucket_of, f, tuple, first, causal, lengths, masked, out
{
    Pairs<T> p;
    Result<T> out;
    spin_relbias bias;
    const T *r[3];
    int f;
    uint64_t masked;
    if (!p.take(a[0], a[5], a[6], a[7]) || !integer(a[3], 0, ByWord<T>::bits - 3, f) || !word(a[8], masked) || !bias_of<T>(a[1], a[2], p.d[0], p.d[2], bias) ||
        !tuple_of<T>(a[4], f, p.x->sizes(), r) || !out.take(a[9], p.x->sizes(), *p.x))
        return none();
    const T *x = data<T>(p.x);
    T *to = data<T>(out.t);
    const int causal = a[6] == Py_True;
    return run(*out.t, [&](spin_stream q) {
        return by_word<T>().bias(p.d[0], p.d[1], p.d[2], p.d[3], p.d[4], p.first, causal, p.lengths, f, x, r[0], r[1], r[2], (T)masked, &bias, to, q);
    });
}
template <class T> PyObject *relbias_grad(PyObject *const *a)      // dS, bucket_of, buckets, first, causal, lengths, out
{
    Pairs<T> p;
    Result<T> out;
    spin_relbias bias;
    int buckets;
    if (!p.take(a[0], a[3], a[4], a[5]) || !integer(a[2], 1, 0x7fffffff, buckets) || !bucketing(a[1], buckets, bias)) return none();
    const int64_t shape[3] = {p.d[0], p.d[2], buckets};
    if (!out.take(a[6], Shape(shape, 3), *p.x)) return none();
    const T *dS = data<T>(p.x);
    T *to = data<T>(out.t);
    const int causal = a[4] == Py_True;
    return run(*out.t, [&](spin_stream q) { return by_word<T>().grad(p.d[0], p.d[1], p.d[2], p.d[3], p.d[4], p.first, causal, p.lengths, dS, &bias, to, q); });
}
// ---- linear attention with a decay, layer norm: (word bits, the arguments of the calls in spin.py) ------------------------------
// Operands of one call: shapes and that all are on the current device, whose stream the kernels run on.
template <class T> struct Operands {
    const int device = c10::hip::current_device();
    const at::Tensor *ring(PyObject *o, Shape shape) const
    {
        const at::Tensor *t = word_tensor<T>(o, shape);
        return t && t->get_device() == device ? t : nullptr;
    }
    bool word(PyObject *o, Shape shape, const T *&p) const
    {
        const at::Tensor *t = ring(o, shape);
        if (t) p = data<T>(t);
        return t != nullptr;
    }
    bool masked(PyObject *o, Shape shape, spin_masked &m) const
    {
        const T *x, *a;
        if (!sequence(o, 2) || !word(PySequence_Fast_GET_ITEM(o, 0), shape, x) || !word(PySequence_Fast_GET_ITEM(o, 1), shape, a)) return false;
        m = spin_masked{x, a};
        return true;
    }
    bool tuple(PyObject *o, Shape shape, spin_tuple &m) const
    {
        const T *r[3];
        if (!sequence(o, 3)) return false;
        for (int k = 0; k < 3; ++k)
            if (!word(PySequence_Fast_GET_ITEM(o, k), shape, r[k])) return false;
        m = spin_tuple{r[0], r[1], r[2]};
        return true;
    }
    // heads, their decay, and the lengths (or which sequences are active)
    bool heads(Shape x, int64_t tokens, int64_t chunk, PyObject *f, PyObject *decay, PyObject *g, PyObject *lengths, spin_linattn &s) const
    {
        const int most = ByWord<T>::bits - 3;
        if (!parties(x[0]) || !fits({x[1], x[2], tokens, chunk}) || !integer(f, 1, most, s.f) || !integer(g, 0, most, s.g)) return false;
        s.n = (int)x[0], s.batch = (int)x[1], s.heads = (int)x[2], s.tokens = (int)tokens, s.chunk = (int)chunk;
        s.decay = nullptr;
        if (decay != Py_None) {
            const int64_t shape[2] = {x[2], chunk + 1};
            const T *w;
            if (!word(decay, Shape(shape, 2), w)) return false;
            s.decay = w;
        }
        if (!list_of(lengths, x.slice(1, 1), s.lengths)) return false;
        return !s.lengths || THPVariable_Unpack(lengths).get_device() == device;
    }
    // `out` (which may be longer) or a fresh tensor
    bool result(PyObject *out, Shape shape, const at::Tensor &like, Result<T> &r) const { return r.take(out, shape, like) && r.t->get_device() == device; }
};
template <class T> inline const at::Tensor *first_of(PyObject *pair, int64_t dims)
{
    const at::Tensor *t = sequence(pair, 2) ? word_tensor<T>(PySequence_Fast_GET_ITEM(pair, 0)) : nullptr;
    return t && t->dim() == dims ? t : nullptr;
}
inline PyObject *item(PyObject *o, Py_ssize_t k) { return o == Py_None ? Py_None : PySequence_Fast_GET_ITEM(o, k); }
// Several results, or the status.
template <class F> inline PyObject *run_all(std::initializer_list<const at::Tensor *> results, F &&call)
{
    THPObjectPtr all(PyTuple_New((Py_ssize_t)results.size()));
    if (!all) return PyErr_Clear(), none();
    Py_ssize_t k = 0;
    for (const at::Tensor *t : results) {
        PyObject *o = t ? THPVariable_Wrap(*t) : none();
        if (!o) return PyErr_Clear(), none();
        PyTuple_SET_ITEM(all.get(), k++, o);
    }
    const spin_status st = unlocked(call);
    return st == SPIN_OK ? all.release() : PyLong_FromLong(st);
}
struct Workspace {
    at::Tensor fresh;
    const at::Tensor *t = nullptr;
    bool take(PyObject *o, size_t need, const at::Tensor &like)
    {
        if (o != Py_None) return (t = workspace_tensor(o)) && t->get_device() == like.get_device();
        if (need == 0 || need > unasked_bytes) return false;
        fresh = at::empty({(int64_t)need}, like.options().dtype(at::kByte));
        t = &fresh;
        return true;
    }
    void *space() const { return t->mutable_data_ptr(); }
    size_t bytes() const { return (size_t)t->numel() * t->element_size(); }
};

template <class T> PyObject *linattn_scores(PyObject *const *a)    // x, y, C, tuple, f, decay, g, lengths, out
{
    const Operands<T> ops;
    const at::Tensor *x = first_of<T>(a[0], 5), *C = word_tensor<T>(a[2]);
    if (!x || !C || C->dim() != 6 || C->size(5) < 1) return none();
    const Shape s = x->sizes();
    const int64_t chunk = C->size(5), pairs[6] = {s[0], s[1], s[2], (s[3] + chunk - 1) / chunk, chunk, chunk};
    spin_linattn d;
    spin_masked mx, my;
    spin_tuple t;
    const T *c;
    Result<T> out;
    if (!ops.heads(s, s[3], chunk, a[4], a[5], a[6], a[7], d) || !fits({s[4]}) || !ops.masked(a[0], s, mx) || !ops.masked(a[1], s, my) ||
        !ops.word(a[2], Shape(pairs, 6), c) || !ops.tuple(a[3], Shape(pairs, 6), t) || !ops.result(a[8], Shape(pairs, 6), *C, out))
        return none();
    T *to = data<T>(out.t);
    return run(*out.t, [&](spin_stream q) { return by_word<T>().linattn_scores(&d, (int)s[4], &mx, &my, c, &t, to, q); });
}
template <class T> PyObject *linattn_states(PyObject *const *a)    // x, y, C, tuple, f, chunk, decay, g, lengths, first, reverse, out, workspace
{
    const Operands<T> ops;
    const at::Tensor *x = first_of<T>(a[0], 5), *y = first_of<T>(a[1], 5), *C = word_tensor<T>(a[2]);
    int chunk;
    if (!x || !y || !C || !integer(a[5], 1, 0x7fffff, chunk) || !PyBool_Check(a[10]) || (a[11] != Py_None && !sequence(a[11], 2))) return none();
    const Shape s = x->sizes();
    const int64_t rows = s[4], columns = y->size(4), state[5] = {s[0], s[1], s[2], rows, columns};
    const int64_t every[6] = {s[0], s[1], s[2], (s[3] + chunk - 1) / chunk, rows, columns}, values[5] = {s[0], s[1], s[2], s[3], columns};
    spin_linattn d;
    spin_masked mx, my;
    spin_tuple t;
    const T *c, *first = nullptr;
    Result<T> states, last;
    Workspace ws;
    if (!ops.heads(s, s[3], chunk, a[4], a[6], a[7], a[8], d) || !fits({rows, columns}) || !ops.masked(a[0], s, mx) || !ops.masked(a[1], Shape(values, 5), my) ||
        !ops.word(a[2], Shape(every, 6), c) || !ops.tuple(a[3], Shape(every, 6), t) || (a[9] != Py_None && !ops.word(a[9], Shape(state, 5), first)) ||
        !ops.result(item(a[11], 0), Shape(every, 6), *C, states) || !ops.result(item(a[11], 1), Shape(state, 5), *C, last) ||
        !ws.take(a[12], by_word<T>().linattn_states_bytes(&d, (int)rows, (int)columns), *C))
        return none();
    T *to = data<T>(states.t), *end = data<T>(last.t);
    const int reverse = a[10] == Py_True;
    return run_all({states.t, last.t}, [&](spin_stream q) {
        return by_word<T>().linattn_states(&d, (int)rows, (int)columns, reverse, &mx, &my, c, &t, first, to, end, ws.space(), ws.bytes(), q);
    });
}
template <class T> PyObject *linattn_outputs(PyObject *const *a)   // P, y, x, S, C, tuple, f, decay, g, lengths, reverse, transposed, out
{
    const Operands<T> ops;
    const at::Tensor *P = first_of<T>(a[0], 6), *x = first_of<T>(a[2], 5), *C = word_tensor<T>(a[4]);
    if (!P || !x || !C || C->dim() != 5 || P->size(5) < 1 || !PyBool_Check(a[10]) || !PyBool_Check(a[11])) return none();
    const Shape s = x->sizes();
    const bool reverse = a[10] == Py_True, transposed = a[11] == Py_True;
    const int64_t rows = s[4], columns = C->size(4), chunk = P->size(5), chunks = (s[3] + chunk - 1) / chunk;
    const int64_t values[5] = {s[0], s[1], s[2], s[3], columns}, pairs[6] = {s[0], s[1], s[2], chunks, chunk, chunk};
    const int64_t state[6] = {s[0], s[1], s[2], chunks, transposed ? columns : rows, transposed ? rows : columns};
    spin_linattn d;
    spin_masked mp, my, mx, ms;
    spin_tuple t;
    const T *c;
    Result<T> out;
    if (!ops.heads(s, s[3], chunk, a[6], a[7], a[8], a[9], d) || !fits({rows, columns}) || !ops.masked(a[0], Shape(pairs, 6), mp) ||
        !ops.masked(a[1], Shape(values, 5), my) || !ops.masked(a[2], s, mx) || !ops.masked(a[3], Shape(state, 6), ms) || !ops.word(a[4], Shape(values, 5), c) ||
        !ops.tuple(a[5], Shape(values, 5), t) || !ops.result(a[12], Shape(values, 5), *C, out))
        return none();
    T *to = data<T>(out.t);
    return run(*out.t, [&](spin_stream q) {
        return by_word<T>().linattn_outputs(&d, (int)rows, (int)columns, reverse, transposed, &mp, &my, &mx, &ms, c, &t, to, q);
    });
}
template <class T> PyObject *linattn_step(PyObject *const *a)      // S, q, k, v, mask, C, tuples, f, decay, g, active, out
{
    const Operands<T> ops;
    const at::Tensor *S = word_tensor<T>(a[0]);
    if (!S || S->dim() != 5 || !sequence(a[5], 2) || !sequence(a[6], 2) || (a[11] != Py_None && !sequence(a[11], 2))) return none();
    const Shape s = S->sizes();
    const int64_t keys[4] = {s[0], s[1], s[2], s[3]}, values[4] = {s[0], s[1], s[2], s[4]};
    spin_linattn d;
    spin_masked q, k, v;
    spin_tuple tS, tO;
    const T *state, *mask, *CS, *CO;
    Result<T> result, after;
    if (!ops.heads(s, 1, 1, a[7], a[8], a[9], a[10], d) || !fits({s[3], s[4]}) || !ops.word(a[0], s, state) || !ops.masked(a[1], Shape(keys, 4), q) ||
        !ops.masked(a[2], Shape(keys, 4), k) || !ops.masked(a[3], Shape(values, 4), v) || !ops.word(a[4], s, mask) ||
        !ops.word(PySequence_Fast_GET_ITEM(a[5], 0), s, CS) || !ops.word(PySequence_Fast_GET_ITEM(a[5], 1), Shape(values, 4), CO) ||
        !ops.tuple(PySequence_Fast_GET_ITEM(a[6], 0), s, tS) || !ops.tuple(PySequence_Fast_GET_ITEM(a[6], 1), Shape(values, 4), tO) ||
        !ops.result(item(a[11], 0), Shape(values, 4), *S, result) || !ops.result(item(a[11], 1), s, *S, after))
        return none();
    T *to = data<T>(result.t), *next = data<T>(after.t);
    return run_all({result.t, after.t}, [&](spin_stream stream) {
        return by_word<T>().linattn_step(&d, (int)s[3], (int)s[4], state, &q, &k, &v, mask, CS, &tS, CO, &tO, next, to, stream);
    });
}
// [n, rows, dim], f, shift
template <class T> inline bool norm_of(const at::Tensor *x, PyObject *f, PyObject *shift, spin_norm &s)
{
    const int most = ByWord<T>::bits - 3;
    if (!x || x->dim() != 3 || !parties(x->size(0)) || !fits({x->size(1), x->size(2)}) || !integer(f, 1, most - 1, s.f) || !integer(shift, 1, most, s.shift)) return false;
    s.n = (int)x->size(0), s.rows = (int)x->size(1), s.dim = (int)x->size(2);
    return true;
}
template <class T> PyObject *layernorm(PyObject *const *a)         // x, gamma, beta, masks, C, tuples, row_words, f, shift, line, eps, out
{
    const Operands<T> ops;
    const at::Tensor *x = word_tensor<T>(a[0]), *w = word_tensor<T>(a[6]);
    spin_norm d;
    uint64_t offset, slope, eps;
    if (!norm_of<T>(x, a[7], a[8], d) || !w || w->dim() != 3 || !fits({w->size(1)}) || w->size(1) % 15 != 0 || !sequence(a[3], 2) || !sequence(a[4], 2) || !sequence(a[5], 2) ||
        !sequence(a[9], 2) || !word(PySequence_Fast_GET_ITEM(a[9], 0), offset) || !word(PySequence_Fast_GET_ITEM(a[9], 1), slope) || !word(a[10], eps) ||
        (a[11] != Py_None && !sequence(a[11], 3)))
        return none();
    const Shape s = x->sizes();
    const int64_t columns[2] = {s[0], s[2]}, words[3] = {s[0], w->size(1), s[1]}, rows[2] = {s[0], s[1]};
    spin_masked gamma;
    spin_tuple t[2];
    const T *value, *beta, *mask[2], *C[2], *row_words;
    Result<T> out, xhat, rstd;
    // xhat and rstd may be left out
    const bool keeps_xhat = a[11] == Py_None || PySequence_Fast_GET_ITEM(a[11], 1) != Py_None, keeps_rstd = a[11] == Py_None || PySequence_Fast_GET_ITEM(a[11], 2) != Py_None;
    if (!ops.word(a[0], s, value) || !ops.masked(a[1], Shape(columns, 2), gamma) || !ops.word(a[2], Shape(columns, 2), beta) || !ops.word(a[6], Shape(words, 3), row_words))
        return none();
    for (int k = 0; k < 2; ++k)
        if (!ops.word(PySequence_Fast_GET_ITEM(a[3], k), s, mask[k]) || !ops.word(PySequence_Fast_GET_ITEM(a[4], k), s, C[k]) ||
            !ops.tuple(PySequence_Fast_GET_ITEM(a[5], k), s, t[k]))
            return none();
    if (!ops.result(item(a[11], 0), s, *x, out) || (keeps_xhat && !ops.result(item(a[11], 1), s, *x, xhat)) ||
        (keeps_rstd && !ops.result(item(a[11], 2), Shape(rows, 2), *x, rstd)))
        return none();
    T *to = data<T>(out.t), *to_xhat = keeps_xhat ? data<T>(xhat.t) : nullptr, *to_rstd = keeps_rstd ? data<T>(rstd.t) : nullptr;
    const int iterations = (int)(w->size(1) / 15) - 1;
    return run_all({out.t, xhat.t, rstd.t}, [&](spin_stream q) {
        return by_word<T>().norm(&d, iterations, (T)offset, (T)slope, (T)eps, value, &gamma, beta, mask[0], mask[1], C[0], &t[0], C[1], &t[1], row_words, to, to_xhat, to_rstd,
                                 q);
    });
}
template <class T> PyObject *layernorm_grad(PyObject *const *a)    // dy, xhat, rstd, gamma, masks, C, tuples, row_words, column_words, f, shift, out, workspace
{
    const Operands<T> ops;
    const at::Tensor *dy = word_tensor<T>(a[0]);
    spin_norm d;
    if (!norm_of<T>(dy, a[9], a[10], d) || !sequence(a[4], 3) || !sequence(a[5], 2) || !sequence(a[6], 2) || (a[11] != Py_None && !sequence(a[11], 3))) return none();
    const Shape s = dy->sizes();
    const int64_t columns[2] = {s[0], s[2]}, row[2] = {s[0], s[1]}, words[3] = {s[0], 22, s[1]}, four[3] = {s[0], 4, s[2]};
    spin_masked gamma;
    spin_tuple t[2];
    const T *value, *xhat, *rstd, *mask[3], *C[2], *row_words, *column_words;
    Result<T> dx, dgamma, dbeta;
    Workspace ws;
    if (!ops.word(a[0], s, value) || !ops.word(a[1], s, xhat) || !ops.word(a[2], Shape(row, 2), rstd) || !ops.masked(a[3], Shape(columns, 2), gamma) ||
        !ops.word(a[7], Shape(words, 3), row_words) || !ops.word(a[8], Shape(four, 3), column_words))
        return none();
    for (int k = 0; k < 3; ++k)
        if (!ops.word(PySequence_Fast_GET_ITEM(a[4], k), s, mask[k])) return none();
    for (int k = 0; k < 2; ++k)
        if (!ops.word(PySequence_Fast_GET_ITEM(a[5], k), s, C[k]) || !ops.tuple(PySequence_Fast_GET_ITEM(a[6], k), s, t[k])) return none();
    if (!ops.result(item(a[11], 0), s, *dy, dx) || !ops.result(item(a[11], 1), Shape(columns, 2), *dy, dgamma) ||
        !ops.result(item(a[11], 2), Shape(columns, 2), *dy, dbeta) || !ws.take(a[12], by_word<T>().norm_grad_bytes(&d), *dy))
        return none();
    const spin_masked m_dy{value, mask[0]}, m_xhat{xhat, mask[1]};
    T *to = data<T>(dx.t), *to_gamma = data<T>(dgamma.t), *to_beta = data<T>(dbeta.t);
    return run_all({dx.t, dgamma.t, dbeta.t}, [&](spin_stream q) {
        return by_word<T>().norm_grad(&d, &m_dy, &m_xhat, rstd, &gamma, mask[2], C[0], &t[0], C[1], &t[1], row_words, column_words, to, to_gamma, to_beta, ws.space(), ws.bytes(), q);
    });
}
// The first argument says which words; `count` follow.
inline PyObject *either(PyObject *const *a, Py_ssize_t got, Py_ssize_t count, PyObject *(*wide)(PyObject *const *), PyObject *(*narrow)(PyObject *const *))
{
    return guarded([&]() -> PyObject * {
        int bits;
        if (got != count + 1 || !integer(a[0], 32, 64, bits) || (bits != 32 && bits != 64)) return none();
        return bits == 64 ? wide(a + 1) : narrow(a + 1);
    });
}

// ---- module ---------------------------------------------------------------------------------------------------
// bind(addresses of the library's functions in the order of Library, bytes that need no look at the device's memory)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    if (count != 2 || !PyTuple_CheckExact(a[0]) || PyTuple_GET_SIZE(a[0]) != kEntries) {
        PyErr_SetString(PyExc_TypeError, "bind takes the library's addresses and a size");
        return nullptr;
    }
    void *entries[kEntries];
    for (int i = 0; i < kEntries; ++i) entries[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(a[0], i));
    unasked_bytes = PyLong_AsSize_t(a[1]);
    if (PyErr_Occurred()) return nullptr;
    memcpy(&lib, entries, sizeof lib);
    return none();
}

#define FAST(name, call) \
    {name, (PyCFunction)(void *)+[](PyObject *, PyObject *const *a, Py_ssize_t count) -> PyObject * { return call; }, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", (PyCFunction)(void *)bind, METH_FASTCALL, nullptr},
                         FAST("share", sharing(a, count, lib.share)),
                         FAST("bshare", sharing(a, count, lib.bshare)),
                         FAST("open", opening(a, count, lib.open)),
                         FAST("bopen", opening(a, count, lib.bopen)),
                         FAST("beaver_mul", multiplying(a, count, lib.beaver_mul)),
                         FAST("beaver_and", multiplying(a, count, lib.beaver_and)),
                         FAST("trunc", truncating(a, count)),
                         FAST("matmul", matmul(a, count)),
                         FAST("grouped", grouped(a, count)),
                         FAST("completed_square", completed_square(a, count)),
                         FAST("cache_append", either(a, count, 6, cache_append<uint64_t>, cache_append<uint32_t>)),
                         FAST("cache_copy", either(a, count, 3, cache_copy<uint64_t>, cache_copy<uint32_t>)),
                         FAST("cache_compact", either(a, count, 5, cache_compact<uint64_t>, cache_compact<uint32_t>)),
                         FAST("cache_scores", either(a, count, 13, cache_scores<uint64_t>, cache_scores<uint32_t>)),
                         FAST("cache_values", either(a, count, 11, cache_values<uint64_t>, cache_values<uint32_t>)),
                         FAST("relbias_trunc", either(a, count, 10, relbias_trunc<uint64_t>, relbias_trunc<uint32_t>)),
                         FAST("relbias_grad", either(a, count, 7, relbias_grad<uint64_t>, relbias_grad<uint32_t>)),
                         FAST("linattn_scores", either(a, count, 9, linattn_scores<uint64_t>, linattn_scores<uint32_t>)),
                         FAST("linattn_states", either(a, count, 13, linattn_states<uint64_t>, linattn_states<uint32_t>)),
                         FAST("linattn_outputs", either(a, count, 13, linattn_outputs<uint64_t>, linattn_outputs<uint32_t>)),
                         FAST("linattn_step", either(a, count, 12, linattn_step<uint64_t>, linattn_step<uint32_t>)),
                         FAST("layernorm", either(a, count, 12, layernorm<uint64_t>, layernorm<uint32_t>)),
                         FAST("layernorm_grad", either(a, count, 13, layernorm_grad<uint64_t>, layernorm_grad<uint32_t>)),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
