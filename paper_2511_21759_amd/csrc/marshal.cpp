// Marshalling of the calls of 8-bit pages: looks at the tensors, packs the C structures and makes the call, in one step from Python (a call of
// a few rows takes the GPU 3 to 7 us, and the same checks made in Python 10 to 17).  What it does not take - anything but tensors of the
// described kind on the current device - it leaves to the binding's own path by returning None; that path also says what is wrong.
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ops/empty.h>

#include "../../include/odb.h"

namespace {

using at::Tensor;

typedef int (*store_entry)(const odb_quant_rows *, const odb_quant_pages *, void *);
typedef int (*read_entry)(const odb_quant_pages *, const int32_t *, int, int, void *, void *, long long, long long, void *);
typedef int (*attention_entry)(const odb_attention *, const odb_quant_pages *, void *);
typedef long long (*workspace_entry)(const odb_attention *, const odb_quant_pages *);

// arguments by number: a tensor, or none where that is allowed
struct Args {
    PyObject *const *a;
    int device;
    bool good = true;
    const Tensor *tensor(int i) {
        if (!THPVariable_Check(a[i])) { good = false; return nullptr; }
        return &THPVariable_Unpack(a[i]);
    }
    const Tensor *maybe(int i) { return a[i] == Py_None ? nullptr : tensor(i); }
    long long number(int i) {
        const long long x = PyLong_AsLongLong(a[i]);
        if (x == -1 && PyErr_Occurred()) { PyErr_Clear(); good = false; }
        return x;
    }
    int small(int i) {
        const long long x = number(i);
        if (x < INT_MIN || x > INT_MAX) good = false;
        return (int)x;
    }
    double real(int i) {
        const double x = PyFloat_AsDouble(a[i]);
        if (x == -1.0 && PyErr_Occurred()) { PyErr_Clear(); good = false; }
        return x;
    }
    bool truth(int i) {
        const int x = PyObject_IsTrue(a[i]);
        if (x < 0) { PyErr_Clear(); good = false; }
        return x == 1;
    }
    const int32_t *ints(const Tensor *t, int64_t n, int64_t m = -1) {
        if (!t) return nullptr;
        if (t->scalar_type() != at::kInt || t->get_device() != device || !t->is_contiguous() || t->dim() != (m < 0 ? 1 : 2) || t->size(0) != n || (m >= 0 && t->size(1) != m))
            good = false;
        return good ? (const int32_t *)t->const_data_ptr() : nullptr;
    }
    // rows [rows, heads, dim] whose heads follow each other: the stride from row to row
    long long rows(const Tensor *t, at::ScalarType type, int64_t n, int64_t heads, int64_t dim) {
        if (!t || t->dim() != 3 || t->size(0) != n || t->size(1) != heads || t->size(2) != dim || t->scalar_type() != type || t->get_device() != device ||
            t->stride(2) != 1 || (t->stride(1) != dim && heads != 1)) {
            good = false;
            return 0;
        }
        return n > 1 ? t->stride(0) : std::max<int64_t>(t->stride(0), heads * dim);
    }
};

int code_of(at::ScalarType t) { return t == at::kHalf ? ODB_F16 : t == at::kBFloat16 ? ODB_BF16 : t == at::kFloat ? ODB_F32 : -1; }

// four tensors from argument i on
bool pages_of(Args &x, int i, int dtype, odb_quant_pages &p) {
    const Tensor *k = x.tensor(i), *v = x.tensor(i + 1), *ks = x.tensor(i + 2), *vs = x.tensor(i + 3);
    if (!x.good || k->dim() != 4 || ks->dim() != 3 || k->sizes() != v->sizes() || k->strides() != v->strides() || k->scalar_type() != v->scalar_type() ||
        ks->sizes() != vs->sizes() || ks->strides() != vs->strides() || ks->scalar_type() != at::kFloat || vs->scalar_type() != at::kFloat)
        return false;
    const int codes = k->scalar_type() == at::kChar ? ODB_INT8 : k->scalar_type() == at::kFloat8_e4m3fn ? ODB_E4M3 : -1;
    const int64_t groups = ks->size(2);
    if (codes < 0 || k->stride(3) != 1 || ks->size(0) != k->size(0) || ks->size(1) != k->size(1) || groups < 1 || k->size(2) % groups || (ks->stride(2) != 1 && groups != 1))
        return false;
    for (const Tensor *t : {k, v, ks, vs})
        if (t->get_device() != x.device) return false;
    for (int j = 0; j < 4; j++)
        if (k->size(j) > INT_MAX) return false;
    p = odb_quant_pages{k->data_ptr(), v->data_ptr(), (float *)ks->data_ptr(), (float *)vs->data_ptr(), (int)k->size(0), (int)k->size(2), (int)k->size(1), (int)k->size(3),
                        codes, (int)(k->size(2) / groups), dtype, k->stride(0), k->stride(1), k->stride(2), ks->stride(0), ks->stride(1)};
    return true;
}

Tensor empty_like(const Tensor &q, at::IntArrayRef shape, at::ScalarType type) { return at::empty(shape, q.options().dtype(type).requires_grad(false)); }

// Other threads of Python run while memory is found and the call is made, which may wait for room in a queue.  (Tensors that are arguments stay: the
// caller holds them.)
struct Unlocked {
    PyThreadState *state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};

// the results, or the entry's error code
template <class F>
PyObject *finish(int rc, F results) { return rc ? PyLong_FromLong(rc) : results(); }

// (entry, stream, device, q, k, v, pools x 4, table, positions, tables, kv_len, cu_rows, first_pos, q_gain, k_gain, eps, interleaved, bfloat16, out, odd)
PyObject *store(PyObject *, PyObject *const *a, Py_ssize_t n) try {
    if (n != 23) Py_RETURN_NONE;
    Args x{a, 0};
    const long long entry = x.number(0), stream = x.number(1);
    x.device = x.small(2);
    const Tensor *q = x.tensor(3), *k = x.tensor(4), *v = x.tensor(5), *table = x.tensor(10), *positions = x.tensor(11), *tables = x.tensor(12), *kv_len = x.tensor(13);
    const Tensor *cu = x.maybe(14), *first = x.maybe(15), *qg = x.maybe(16), *kg = x.maybe(17), *out = x.maybe(21), *odd = x.maybe(22);
    const at::ScalarType type = x.truth(20) ? at::kBFloat16 : at::kHalf;
    odb_quant_pages p;
    if (!x.good || !pages_of(x, 6, code_of(type), p) || q->dim() != 3 || tables->dim() != 2 || table->dim() != 3) Py_RETURN_NONE;
    const int64_t rows = q->size(0), heads = q->size(1), dim = q->size(2), reqs = tables->size(0), columns = tables->size(1);
    const at::ScalarType given = q->scalar_type();
    if (code_of(given) < 0 || dim != p.head_dim || rows < 1 || rows > INT_MAX || heads > INT_MAX || reqs > INT_MAX || columns > INT_MAX || (!cu && rows != reqs)) Py_RETURN_NONE;
    if (table->scalar_type() != at::kFloat || table->size(2) != 2 || table->get_device() != x.device || !table->is_contiguous() || table->size(0) > INT_MAX || table->size(1) > 1 << 20) Py_RETURN_NONE;
    for (const Tensor *t : {qg, kg})
        if (t && (t->scalar_type() != at::kFloat || t->dim() != 1 || t->size(0) != dim || t->get_device() != x.device || !t->is_contiguous())) Py_RETURN_NONE;
    odb_quant_rows r{};
    r.q_row = x.rows(q, given, rows, heads, dim);
    r.k_row = x.rows(k, given, rows, p.n_kv_heads, dim);
    r.v_row = x.rows(v, given, rows, p.n_kv_heads, dim);
    r.eps = (float)x.real(18);
    r.interleaved = x.truth(19);
    r.positions = x.ints(positions, rows);
    r.cu_rows = x.ints(cu, reqs + 1);
    r.first_pos = x.ints(first, reqs);
    r.kv_len = x.ints(kv_len, reqs);
    r.tables = x.ints(tables, reqs, columns);
    r.odd = (int32_t *)x.ints(odd, 1);
    if (out) r.q_out_row = x.rows(out, type, rows, heads, dim);
    if (!x.good) Py_RETURN_NONE;
    r.q = q->data_ptr(); r.k = k->data_ptr(); r.v = v->data_ptr();
    r.in_dtype = code_of(given); r.rows = (int)rows; r.n_heads = (int)heads;
    r.q_gain = qg ? (const float *)qg->data_ptr() : nullptr; r.k_gain = kg ? (const float *)kg->data_ptr() : nullptr;
    r.table = (const float *)table->data_ptr(); r.n_pos = (int)table->size(0); r.rot_dim = 2 * (int)table->size(1);
    r.columns = (int)columns; r.n = (int)reqs;
    Tensor made;
    int rc;
    {
        Unlocked other_threads;
        if (!out) {
            made = empty_like(*q, {rows, heads, dim}, type);
            r.q_out_row = heads * dim;
            out = &made;
        }
        r.q_out = out->data_ptr();
        rc = ((store_entry)entry)(&r, &p, (void *)stream);
    }
    return finish(rc, [&] {
        if (made.defined()) return THPVariable_Wrap(made);
        Py_INCREF(a[21]);
        return a[21];
    });
} catch (const std::exception &) {                                     // (no memory, say: the other path meets it again and names it)
    Py_RETURN_NONE;
}

// (entry, stream, device, pools x 4, slots, dtype: 0, 1 or 2)
PyObject *read(PyObject *, PyObject *const *a, Py_ssize_t n) try {
    if (n != 9) Py_RETURN_NONE;
    Args x{a, 0};
    const long long entry = x.number(0), stream = x.number(1);
    x.device = x.small(2);
    const Tensor *slots = x.tensor(7);
    const int dtype = x.small(8);
    odb_quant_pages p;
    if (!x.good || !pages_of(x, 3, ODB_F16, p) || dtype < 0 || dtype > 2) Py_RETURN_NONE;
    const int64_t rows = slots->numel();
    const int32_t *at = x.ints(slots, rows);
    if (!x.good || rows < 1 || rows > INT_MAX) Py_RETURN_NONE;
    const at::ScalarType type = dtype == ODB_F16 ? at::kHalf : dtype == ODB_BF16 ? at::kBFloat16 : at::kFloat;
    const int64_t row = (int64_t)p.n_kv_heads * p.head_dim;
    Tensor k, v;
    int rc;
    {
        Unlocked other_threads;
        k = empty_like(*slots, {rows, p.n_kv_heads, p.head_dim}, type);
        v = empty_like(*slots, {rows, p.n_kv_heads, p.head_dim}, type);
        rc = ((read_entry)entry)(&p, at, (int)rows, dtype, k.data_ptr(), v.data_ptr(), row, row, (void *)stream);
    }
    return finish(rc, [&]() -> PyObject * {
        PyObject *pair = PyTuple_New(2);
        if (!pair) return nullptr;
        PyTuple_SET_ITEM(pair, 0, THPVariable_Wrap(k));
        PyTuple_SET_ITEM(pair, 1, THPVariable_Wrap(v));
        return pair;
    });
} catch (const std::exception &) {
    Py_RETURN_NONE;
}

// (entry, workspace's entry, stream, device, q, pools x 4, tables, kv_len, cu_rows, first_pos, scale, causal, window, sinks, max_rows, max_len, out, workspace)
PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n) try {
    if (n != 21) Py_RETURN_NONE;
    Args x{a, 0};
    const long long entry = x.number(0), space = x.number(1), stream = x.number(2);
    x.device = x.small(3);
    const Tensor *q = x.tensor(4), *tables = x.tensor(9), *kv_len = x.tensor(10), *cu = x.maybe(11), *first = x.maybe(12), *out = x.maybe(19), *work = x.maybe(20);
    if (!x.good) Py_RETURN_NONE;
    const at::ScalarType type = q->scalar_type();
    odb_quant_pages p;
    if ((type != at::kHalf && type != at::kBFloat16) || !pages_of(x, 5, code_of(type), p) || q->dim() != 3 || tables->dim() != 2) Py_RETURN_NONE;
    const int64_t rows = q->size(0), heads = q->size(1), dim = q->size(2), reqs = tables->size(0), columns = tables->size(1);
    if (dim != p.head_dim || rows < 1 || rows > INT_MAX || heads > INT_MAX || reqs > INT_MAX || columns > INT_MAX || (!cu && rows != reqs)) Py_RETURN_NONE;
    odb_attention r{};
    r.q_row = x.rows(q, type, rows, heads, dim);
    r.out_row = out ? x.rows(out, type, rows, heads, dim) : heads * dim;
    r.cu_rows = x.ints(cu, reqs + 1);
    r.first_pos = x.ints(first, reqs);
    r.kv_len = x.ints(kv_len, reqs);
    r.tables = x.ints(tables, reqs, columns);
    r.scale = (float)x.real(13);
    r.causal = x.truth(14); r.window = x.small(15); r.sinks = x.small(16); r.max_rows = x.small(17); r.max_len = x.small(18);
    if (work && (work->scalar_type() != at::kByte || work->get_device() != x.device || !work->is_contiguous())) Py_RETURN_NONE;
    if (!x.good) Py_RETURN_NONE;
    r.columns = (int)columns; r.n = (int)reqs; r.rows = (int)rows; r.n_heads = (int)heads;
    r.q = q->data_ptr();
    const long long need = ((workspace_entry)space)(&r, &p);
    if (need < 0) return PyLong_FromLongLong(need);
    Tensor made, room;
    int rc;
    {
        Unlocked other_threads;
        if (!out) {
            made = empty_like(*q, {rows, heads, dim}, type);
            out = &made;
        }
        r.out = out->data_ptr();
        if (need > 0) {
            if (!work) {
                room = empty_like(*q, {need}, at::kByte);
                work = &room;
            }
            r.workspace = work->data_ptr();
            r.workspace_bytes = (size_t)work->numel();
        }
        rc = ((attention_entry)entry)(&r, &p, (void *)stream);
    }
    return finish(rc, [&] {
        if (made.defined()) return THPVariable_Wrap(made);
        Py_INCREF(a[19]);
        return a[19];
    });
} catch (const std::exception &) {
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"store", (PyCFunction)(void (*)(void))store, METH_FASTCALL, nullptr},
                         {"read", (PyCFunction)(void (*)(void))read, METH_FASTCALL, nullptr},
                         {"attention", (PyCFunction)(void (*)(void))attention, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
