// Host side of the binding: the levels of a call as the array of 64-bit words that mka_level[3], mka_level_grad[3] and
// mka_paged_level[3] are, the call's small outputs, and the calls of the library that short steps consist of.  Asked for one by one from Python, the
// pointers, shapes and strides of the six tensors of a call took longer than a short decode takes on the GPU (6.3 us; 0.2 us here); the
// rest of a call's arguments through ctypes took 1.7 us of a router's 4.6, and of a forward's 12.2 (a short prompt is over in 17) 7.7.
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <torch/csrc/autograd/python_variable.h>

#include <Python.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <tuple>
#include <type_traits>
#include <utility>
#include <vector>

#include "mka.h"

namespace {

constexpr char kLevelsWanted[] = "levels: tensors [batch, head, row, column] with dense columns, K and V alike; tables and row counts int32";
constexpr char kTypesWanted[] = "levels: bf16 or f32, all alike";
constexpr char kPoolsWanted[] = "paged levels: pools of bf16 (8-bit pools have entry points of their own)";
constexpr char kTensorWanted[] = "a tensor (or None where an argument may be left out) is expected";
constexpr char kCountWanted[] = "wrong number of arguments";
struct Bad { const char* what = kLevelsWanted; };    // what an assertion of the binding would have refused
struct PyErrSet {};                                  // the Python error is set

const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) throw Bad{kTensorWanted};
    return THPVariable_Unpack(o);
}

struct Held {                                        // a reference of our own
    PyObject* o;
    explicit Held(PyObject* x) : o(x) { if (!o) throw PyErrSet(); }
    ~Held() { Py_XDECREF(o); }
    Held(const Held&) = delete;
    Held& operator=(const Held&) = delete;
};
// Entries of a list or tuple, or of whatever else answers x[i] (then held as long as this is).
class Seq {
    PyObject* x_;
    const bool plain_;
    std::vector<PyObject*> held_;

  public:
    explicit Seq(PyObject* x) : x_(x), plain_(PyList_Check(x) || PyTuple_Check(x)) { Py_INCREF(x_); }
    ~Seq() {
        for (PyObject* h : held_) Py_DECREF(h);
        Py_DECREF(x_);
    }
    Seq(const Seq&) = delete;
    Seq& operator=(const Seq&) = delete;
    PyObject* at(Py_ssize_t i) {
        if (plain_ && i < PySequence_Fast_GET_SIZE(x_)) return PySequence_Fast_GET_ITEM(x_, i);
        const Held at(PyLong_FromSsize_t(i));
        PyObject* item = PyObject_GetItem(x_, at.o);
        if (!item) throw PyErrSet();
        held_.push_back(item);
        return item;
    }
    const at::Tensor* tensor_at(Py_ssize_t i) {               // nullptr for None
        PyObject* x = at(i);
        return x == Py_None ? nullptr : &tensor(x);
    }
};

int64_t address(const at::Tensor& t) { return static_cast<int64_t>(reinterpret_cast<intptr_t>(t.data_ptr())); }
int64_t integer(PyObject* o) {                       // int(o)
    int64_t v;
    if (PyLong_CheckExact(o)) {
        v = PyLong_AsLongLong(o);
    } else {
        const Held whole(PyNumber_Long(o));
        v = PyLong_AsLongLong(whole.o);
    }
    if (v == -1 && PyErr_Occurred()) throw PyErrSet();
    return v;
}
template <size_t N> PyObject* bytes(const int64_t (&w)[N]) { return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(w), sizeof(w)); }

// Four dimensions, the last one dense, and V laid out as K.
void check_layout(const at::Tensor& k, const at::Tensor& v) {
    if (k.dim() != 4 || k.stride(3) != 1 || v.strides() != k.strides()) throw Bad{};
}
void check_pair(const at::Tensor& k, const at::Tensor& v) {
    check_layout(k, v);
    if (v.sizes() != k.sizes()) throw Bad{};
}

// Rows that the library takes for bf16 or f32 (of `like`'s type, if given): any other type's would be read past their end.
void check_type(const at::Tensor& k, const at::Tensor& v, const at::Tensor* like = nullptr) {
    const auto type = (like ? *like : k).scalar_type();
    if ((type != at::kBFloat16 && type != at::kFloat) || k.scalar_type() != type || v.scalar_type() != type) throw Bad{kTypesWanted};
}

template <typename F>
PyObject* guarded(F f) {
    HANDLE_TH_ERRORS
    try {
        return f();
    } catch (const Bad& bad) {
        PyErr_SetString(PyExc_AssertionError, bad.what);
        return nullptr;
    } catch (const PyErrSet&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// Words of a level: k, v, n, stride_b, stride_h, stride_n; zeros where keys are None or have no rows.
void put_level(int64_t* o, const at::Tensor& k, const at::Tensor& v) {
    o[0] = address(k); o[1] = address(v); o[2] = k.size(2);
    for (int i = 0; i < 3; ++i) o[3 + i] = k.stride(i);
}
PyObject* levels(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 2) throw Bad{kCountWanted};
        Seq K(a[0]), V(a[1]);
        int64_t w[18] = {};
        const at::Tensor* first = nullptr;
        for (int l = 0; l < 3; ++l) {
            const at::Tensor* k = K.tensor_at(l);
            if (!k || k->size(2) == 0) continue;
            const at::Tensor* v = V.tensor_at(l);
            if (!v) throw Bad{};
            check_pair(*k, *v);
            check_type(*k, *v, first);
            first = k;
            put_level(w + 6 * l, *k, *v);
        }
        return bytes(w);
    });
}
PyObject* grads(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 3) throw Bad{kCountWanted};
        Seq K(a[0]), dK(a[1]), dV(a[2]);
        int64_t w[18] = {};
        for (int l = 0; l < 3; ++l) {
            const at::Tensor* k = K.tensor_at(l);
            if (!k || k->size(2) == 0) continue;
            const at::Tensor *dk = dK.tensor_at(l), *dv = dV.tensor_at(l);
            if (!dk || !dv) throw Bad{};
            check_layout(*dk, *dv);
            check_type(*dk, *dv, k);
            put_level(w + 6 * l, *dk, *dv);
        }
        return bytes(w);
    });
}

PyObject* paged_levels(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded([&]() -> PyObject* {
        if (n_args != 5) throw Bad{kCountWanted};
        Seq K(a[0]), V(a[1]), tabs(a[2]), rows(a[3]), n(a[4]);
        const bool counted = a[3] != Py_None;
        int64_t w[36] = {};
        for (int l = 0; l < 3; ++l) {
            int64_t* o = w + 12 * l;
            o[7] = 1;
            const at::Tensor* k = K.tensor_at(l);
            if (!k) continue;
            const int64_t most = integer(n.at(l));
            if (most == 0) continue;
            const at::Tensor *v = V.tensor_at(l), *tab = tabs.tensor_at(l), *r = counted ? rows.tensor_at(l) : nullptr;
            if (!v || !tab) throw Bad{};
            check_pair(*k, *v);
            if (k->scalar_type() != at::kBFloat16 || v->scalar_type() != at::kBFloat16) throw Bad{kPoolsWanted};
            // [B, pages]: one table per sequence; [B, H_kv, pages]: one per (sequence, KV head)
            if (tab->scalar_type() != at::kInt || (tab->dim() != 2 && tab->dim() != 3) || tab->stride(tab->dim() - 1) != 1) throw Bad{};
            if (r && (r->scalar_type() != at::kInt || !r->is_contiguous())) throw Bad{};
            o[0] = address(*k); o[1] = address(*v); o[2] = address(*tab); o[3] = r ? address(*r) : 0;
            o[4] = most; o[5] = tab->stride(0); o[6] = tab->dim() == 3 ? tab->stride(1) : 0; o[7] = k->size(2);
            for (int i = 0; i < 3; ++i) o[8 + i] = k->stride(i);
            o[11] = k->size(0);
        }
        return bytes(w);
    });
}

PyObject* paged_level(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 3) throw Bad{kCountWanted};
        const at::Tensor &k = tensor(a[0]), &v = tensor(a[1]), &tab = tensor(a[2]);
        check_layout(k, v);
        check_type(k, v);
        if (tab.scalar_type() != at::kInt || tab.dim() != 2 || tab.stride(1) != 1) throw Bad{};
        const int64_t w[12] = {address(k), address(v), address(tab), 0, tab.size(1) * k.size(2), tab.stride(0), 0, k.size(2),
                               k.stride(0), k.stride(1), k.stride(2), k.size(0)};
        return bytes(w);
    });
}

// ---- 8-bit paged levels and page tables
constexpr char kLevels8Wanted[] = "8-bit levels: pools [pages, H_kv, page rows, d] of float8_e4m3fn or int8, exponents uint8 [pages, H_kv, blocks] with dense "
                                  "blocks, K and V alike; tables and row counts int32, one row of a table per sequence; all on the device of the queries";
constexpr char kTablesWanted[] = "page tables: int32 refs [pages], table [sequences, width] with dense rows, rows [sequences], all on one device";
constexpr char kPlanesWanted[] = "planes: tensors [pages, ...] whose pages, or whose heads in a page, are dense, on the device of the tables";
void want(bool ok, const char* what) {
    if (!ok) throw Bad{what};
}
bool dense_from(const at::Tensor& t, int64_t dim) {          // dimensions dim, dim + 1, ... lie densely
    int64_t expected = 1;
    for (int64_t i = t.dim() - 1; i >= dim; --i) {
        if (t.size(i) != 1 && t.stride(i) != expected) return false;
        expected *= t.size(i);
    }
    return true;
}
// The 17 words of one mka_paged_level8.
void put_level8(int64_t* o, const at::Device& dev, int64_t B, int64_t H_kv, int64_t d, const at::Tensor& k, const at::Tensor& v, const at::Tensor& ek,
                const at::Tensor& ev, const at::Tensor& tab, const at::Tensor* rows, int64_t n) {
    const char* const what = kLevels8Wanted;
    for (const at::Tensor* t : {&k, &v, &ek, &ev, &tab}) want(t->device() == dev, what);
    const auto code = k.scalar_type();
    want((code == at::kFloat8_e4m3fn || code == at::kChar) && v.scalar_type() == code && k.dim() == 4 && k.stride(3) == 1, what);
    want(v.sizes() == k.sizes() && v.strides() == k.strides() && k.size(1) == H_kv && k.size(3) == d, what);
    want(ek.scalar_type() == at::kByte && ev.scalar_type() == at::kByte && ek.dim() == 3 && ev.sizes() == ek.sizes() && ev.strides() == ek.strides(), what);
    want(ek.size(0) == k.size(0) && ek.size(1) == H_kv && ek.size(2) > 0 && k.size(2) % ek.size(2) == 0 && (ek.stride(2) == 1 || ek.size(2) == 1), what);
    const int last = static_cast<int>(tab.dim()) - 1;
    want(tab.scalar_type() == at::kInt && (last == 1 || last == 2) && (tab.stride(last) == 1 || tab.size(last) == 1) && tab.size(0) == B, what);
    want((last == 1 || tab.size(1) == H_kv) && tab.size(last) * k.size(2) >= n, what);
    if (rows) want(rows->device() == dev && rows->scalar_type() == at::kInt && rows->is_contiguous() && rows->numel() == B, what);
    o[0] = address(k); o[1] = address(v); o[2] = address(ek); o[3] = address(ev); o[4] = address(tab); o[5] = rows ? address(*rows) : 0;
    o[6] = n; o[7] = B > 1 ? tab.stride(0) : std::max(tab.stride(0), tab.numel()); o[8] = last == 2 ? (H_kv > 1 ? tab.stride(1) : tab.size(2)) : 0;
    for (int i = 0; i < 3; ++i) o[9 + i] = k.stride(i);
    o[12] = ek.stride(0); o[13] = ek.stride(1); o[14] = k.size(0);
    const int32_t tail[4] = {static_cast<int32_t>(k.size(2)), static_cast<int32_t>(k.size(2) / ek.size(2)), code == at::kChar ? MKA_CODE_S8 : MKA_CODE_E4M3, 0};
    memcpy(o + 15, tail, sizeof(tail));
}
void put_levels8(int64_t (&w)[51], const at::Tensor& q, int64_t H_kv, int64_t d, PyObject* pools_k, PyObject* pools_v, PyObject* exps_k, PyObject* exps_v,
                 PyObject* tables, PyObject* row_counts, PyObject* most_rows) {
    static_assert(sizeof(w) == 3 * sizeof(mka_paged_level8), "17 words to a level");
    Seq K(pools_k), V(pools_v), EK(exps_k), EV(exps_v), tabs(tables), rows(row_counts), n(most_rows);
    memset(w, 0, sizeof(w));
    for (int l = 0; l < 3; ++l) {
        const at::Tensor* k = K.tensor_at(l);
        const int64_t most = k ? integer(n.at(l)) : 0;
        if (most == 0) continue;
        const at::Tensor *v = V.tensor_at(l), *ek = EK.tensor_at(l), *ev = EV.tensor_at(l), *tab = tabs.tensor_at(l);
        want(v && ek && ev && tab, kLevels8Wanted);
        put_level8(w + 17 * l, q.device(), q.size(0), H_kv, d, *k, *v, *ek, *ev, *tab, row_counts == Py_None ? nullptr : rows.tensor_at(l), most);
    }
}
void put_append8(int64_t (&w)[23], const at::Tensor& nk, const at::Tensor& nv, const at::Tensor& k, const at::Tensor& v, const at::Tensor& ek, const at::Tensor& ev,
                 const at::Tensor& tab) {
    check_pair(nk, nv);
    want(nv.device() == nk.device() && nv.scalar_type() == nk.scalar_type() && tab.dim() == 2, kLevels8Wanted);
    put_level(w, nk, nv);
    put_level8(w + 6, nk.device(), nk.size(0), nk.size(1), nk.size(3), k, v, ek, ev, tab, nullptr, tab.size(1) * k.size(2));
}
PyObject* paged_levels8(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded([&]() -> PyObject* {
        if (n_args != 9) throw Bad{kCountWanted};
        const at::Tensor& q = tensor(a[0]);
        want(q.dim() >= 3, kLevels8Wanted);
        int64_t w[51];
        put_levels8(w, q, integer(a[1]), q.size(q.dim() - 1), a[2], a[3], a[4], a[5], a[6], a[7], a[8]);
        return bytes(w);
    });
}
PyObject* append_levels8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 7) throw Bad{kCountWanted};
        int64_t w[23] = {};
        put_append8(w, tensor(a[0]), tensor(a[1]), tensor(a[2]), tensor(a[3]), tensor(a[4]), tensor(a[5]), tensor(a[6]));
        return bytes(w);
    });
}
mka_page_tables tables_of(const at::Tensor& refs, const at::Tensor& tab, const at::Tensor& rows, int64_t page_rows) {
    for (const at::Tensor* t : {&refs, &tab, &rows}) want(t->scalar_type() == at::kInt && t->device() == refs.device(), kTablesWanted);
    want(refs.dim() == 1 && refs.is_contiguous() && rows.dim() == 1 && rows.is_contiguous() && tab.dim() == 2 && tab.size(0) == rows.numel(), kTablesWanted);
    want(tab.stride(1) == 1 || tab.size(1) <= 1 || tab.size(0) == 0, kTablesWanted);
    want(tab.size(0) <= INT32_MAX && tab.size(1) <= INT32_MAX && page_rows > 0 && page_rows <= INT32_MAX, kTablesWanted);
    mka_page_tables t = {};
    t.refs = static_cast<int32_t*>(refs.data_ptr()); t.table = static_cast<int32_t*>(tab.data_ptr()); t.rows = static_cast<int32_t*>(rows.data_ptr());
    t.pages = refs.numel(); t.table_stride = tab.size(0) > 1 ? tab.stride(0) : tab.size(1);
    t.seqs = static_cast<int32_t>(tab.size(0)); t.width = static_cast<int32_t>(tab.size(1)); t.page_rows = static_cast<int32_t>(page_rows);
    return t;
}
std::vector<mka_page_plane> planes_of(PyObject* tensors, const at::Tensor& refs) {
    const Held in(PySequence_Fast(tensors, "a sequence of tensors is expected"));
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(in.o);
    std::vector<mka_page_plane> planes(static_cast<size_t>(n));
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::Tensor& t = tensor(PySequence_Fast_GET_ITEM(in.o, i));
        want(t.dim() >= 2 && t.device() == refs.device() && t.size(0) == refs.numel(), kPlanesWanted);
        const int64_t es = t.element_size();
        int64_t inner = es, heads = 1, stride_h = 0;
        const bool whole = dense_from(t, 1);
        for (int64_t k = whole ? 1 : 2; k < t.dim(); ++k) inner *= t.size(k);
        if (!whole) {
            want(dense_from(t, 2), kPlanesWanted);
            heads = t.size(1); stride_h = t.stride(1) * es;
        }
        want(inner <= INT32_MAX && heads <= INT32_MAX, kPlanesWanted);
        planes[i] = {t.data_ptr(), t.stride(0) * es, stride_h, static_cast<int32_t>(heads), static_cast<int32_t>(inner)};
    }
    return planes;
}
PyObject* page_tables(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 4) throw Bad{kCountWanted};
        const mka_page_tables t = tables_of(tensor(a[0]), tensor(a[1]), tensor(a[2]), integer(a[3]));
        return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&t), sizeof(t));
    });
}
PyObject* page_planes(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 2) throw Bad{kCountWanted};
        const std::vector<mka_page_plane> planes = planes_of(a[0], tensor(a[1]));
        return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(planes.data()), static_cast<Py_ssize_t>(planes.size() * sizeof(mka_page_plane)));
    });
}

PyObject* empties_like(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 1) throw Bad{kCountWanted};
        const Held in(PySequence_Fast(a[0], "a sequence of tensors is expected"));
        const Py_ssize_t size = PySequence_Fast_GET_SIZE(in.o);
        Held out(PyList_New(size));
        for (Py_ssize_t i = 0; i < size; ++i) {
            PyObject* x = PySequence_Fast_GET_ITEM(in.o, i);
            PyObject* o = x == Py_None ? Py_None : THPVariable_Wrap(at::empty_like(tensor(x)));
            if (x == Py_None) Py_INCREF(o);
            PyList_SET_ITEM(out.o, i, o);
        }
        Py_INCREF(out.o);
        return out.o;
    });
}

PyObject* empty_f32(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 3) throw Bad{kCountWanted};
        const at::Tensor& t = tensor(a[0]);
        const int64_t keep = integer(a[1]), extra = integer(a[2]);
        if (keep < 0 || keep > t.dim()) throw Bad{"as many dimensions as the tensor has, at most"};
        std::vector<int64_t> size(t.sizes().begin(), t.sizes().begin() + keep);
        if (extra) size.push_back(extra);
        return THPVariable_Wrap(at::empty(size, at::TensorOptions().device(t.device()).dtype(at::kFloat)));
    });
}

// A C argument from a Python object; what was taken out of the object lives as long as this.
template <typename P> struct Arg;
template <> struct Arg<int64_t> {
    int64_t v;
    explicit Arg(PyObject* o) : v(0) {                // an int or what answers __index__ as one (numpy's, a tensor's); no float
        const Held whole(PyNumber_Index(o));
        v = PyLong_AsLongLong(whole.o);
        if (v == -1 && PyErr_Occurred()) throw PyErrSet();
    }
};
template <> struct Arg<int32_t> {
    int32_t v;
    explicit Arg(PyObject* o) : v(static_cast<int32_t>(Arg<int64_t>(o).v)) {}
};
template <> struct Arg<size_t> {
    size_t v;
    explicit Arg(PyObject* o) : v(static_cast<size_t>(Arg<int64_t>(o).v)) {}
};
void* pointer(PyObject* o) {                         // an int, or None for null
    if (o == Py_None) return nullptr;
    if (!PyLong_Check(o)) throw Bad{"an address is expected: an int or None"};
    void* const v = PyLong_AsVoidPtr(o);
    if (!v && PyErr_Occurred()) throw PyErrSet();
    return v;
}
// A tensor's memory, or that of whatever else has a data_ptr(), as a storage has, or None; no int, as True in an output's place would be address 1.
template <typename T> struct Arg<T*> {
    T* v;
    explicit Arg(PyObject* o) : v(nullptr) {
        if (o == Py_None) return;
        if (THPVariable_Check(o)) {
            v = static_cast<T*>(tensor(o).data_ptr());
            return;
        }
        if (!PyObject_HasAttrString(o, "data_ptr")) throw Bad{kTensorWanted};
        const Held at(PyObject_CallMethod(o, "data_ptr", nullptr));
        v = static_cast<T*>(pointer(at.o));
    }
};
struct Address {                                     // of a function, or a stream's handle: an int, or what holds one as a c_void_p does
    void* v;
    explicit Address(PyObject* o) : v(nullptr) {
        if (o == Py_None || PyLong_Check(o) || !PyObject_HasAttrString(o, "value")) {
            v = pointer(o);
            return;
        }
        const Held at(PyObject_GetAttrString(o, "value"));
        v = pointer(at.o);
    }
};
template <typename T> struct Levels {                // three levels as `levels`, `grads` or `paged_levels` returned them
    const T* v;
    explicit Levels(PyObject* o) : v(nullptr) {
        if (!PyBytes_Check(o) || PyBytes_GET_SIZE(o) != static_cast<Py_ssize_t>(3 * sizeof(T))) throw Bad{};
        v = reinterpret_cast<const T*>(PyBytes_AS_STRING(o));
    }
};
template <> struct Arg<const mka_level*> : Levels<mka_level> { using Levels::Levels; };
template <> struct Arg<const mka_level_grad*> : Levels<mka_level_grad> { using Levels::Levels; };
template <> struct Arg<const mka_paged_level*> : Levels<mka_paged_level> { using Levels::Levels; };
PyObject* shape_class = nullptr;                     // the binding's mka_shape: other buffers of its size are no shapes
PyObject* shape_type(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 1 || !PyType_Check(a[0])) {
        PyErr_SetString(PyExc_TypeError, "a class is expected");
        return nullptr;
    }
    Py_INCREF(a[0]);
    Py_XDECREF(shape_class);
    shape_class = a[0];
    Py_RETURN_NONE;
}
template <> struct Arg<const mka_shape*> {
    mka_shape copy;
    const mka_shape* v;
    explicit Arg(PyObject* o) : v(&copy) {
        if (!shape_class || !PyObject_TypeCheck(o, reinterpret_cast<PyTypeObject*>(shape_class))) {
            PyErr_SetString(PyExc_TypeError, "an mka_shape is expected");
            throw PyErrSet();
        }
        Py_buffer view;
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw PyErrSet();
        const bool fits = view.len == static_cast<Py_ssize_t>(sizeof(mka_shape));
        if (fits) memcpy(&copy, view.buf, sizeof(mka_shape));
        PyBuffer_Release(&view);
        if (!fits) {
            PyErr_SetString(PyExc_TypeError, "an mka_shape is expected");
            throw PyErrSet();
        }
    }
    Arg(const Arg&) = delete;
};

// The library's function at address a[0] (of the type of the declaration named) with the other arguments, the last of which is the stream; its
// status.  Other threads run meanwhile.
template <typename R, typename... P, size_t... I>
PyObject* invoke(R (*)(P...), PyObject* const* a, std::index_sequence<I...>) {
    const auto f = reinterpret_cast<R (*)(P...)>(Address(a[0]).v);
    if (!f) throw Bad{"the address of a function is expected"};
    const std::tuple<std::conditional_t<I + 1 == sizeof...(P), Address, Arg<P>>...> args{a[1 + I]...};
    R status;
    Py_BEGIN_ALLOW_THREADS
    status = f(std::get<I>(args).v...);
    Py_END_ALLOW_THREADS
    return PyLong_FromLongLong(static_cast<long long>(status));
}
template <typename R, typename... P>
PyObject* call(R (*declared)(P...), PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != static_cast<Py_ssize_t>(1 + sizeof...(P))) throw Bad{kCountWanted};
        return invoke(declared, a, std::index_sequence_for<P...>());
    });
}
#define MKA_CALL(name) \
    PyObject* call_##name(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(static_cast<decltype(&mka_##name)>(nullptr), a, n); }
MKA_CALL(router)
MKA_CALL(fwd_with_scratch)
MKA_CALL(fwd_paged_with_scratch)
MKA_CALL(decode)
MKA_CALL(decode_paged)
MKA_CALL(bwd)
#undef MKA_CALL

// ---- the calls of the 8-bit cache and of the page tables: their checks, their structs and the call in one (a call's checks in Python took as long as its kernels)
constexpr char kHereWanted[] = "tensors on the current CUDA device are expected";
constexpr char kQueryWanted[] = "q and O: contiguous bf16 of the shape's sizes on the current device; LSE: contiguous f32, one for each row of q";
constexpr char kGateWanted[] = "gate: contiguous f32 [B, T, 3] on the device of the queries";
constexpr char kI32Wanted[] = "contiguous int32 tensors of the right size on the device of the others are expected";
template <typename F, typename... A>
PyObject* call_checked(PyObject* address, F, A... args) {
    const auto f = reinterpret_cast<F>(Address(address).v);
    if (!f) throw Bad{"the address of a function is expected"};
    mka_status status;
    Py_BEGIN_ALLOW_THREADS
    status = f(args...);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(static_cast<long>(status));
}
void here(const at::Tensor& t, PyObject* device) { want(t.is_cuda() && t.device().index() == integer(device), kHereWanted); }
const at::Tensor* optional(PyObject* o) { return o == Py_None ? nullptr : &tensor(o); }
int32_t* i32(const at::Tensor* t, const at::Tensor& like, int64_t numel) {
    if (!t) return nullptr;
    want(t->scalar_type() == at::kInt && t->is_contiguous() && t->device() == like.device() && t->numel() == numel, kI32Wanted);
    return static_cast<int32_t*>(t->data_ptr());
}
struct Workspace {
    void* v;
    size_t bytes;
    Workspace(const at::Tensor& t, const at::Tensor& like) : v(t.data_ptr()), bytes(static_cast<size_t>(t.numel()) * t.element_size()) {
        want(t.device() == like.device() && t.is_contiguous(), "ws: a contiguous tensor on the device of the others");
    }
};

// attend8(address, device, shape, H_kv, q, pools_k, pools_v, exps_k, exps_v, tables, rows or None, n, gate, O, LSE, ws, stream): mka_decode_paged8 or mka_fwd_paged8
PyObject* attend8(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded([&]() -> PyObject* {
        if (n_args != 17) throw Bad{kCountWanted};
        const Arg<const mka_shape*> shape(a[2]);
        const mka_shape& s = shape.copy;
        const int64_t H_kv = integer(a[3]);
        const at::Tensor &q = tensor(a[4]), &gate = tensor(a[12]), &O = tensor(a[13]), &LSE = tensor(a[14]);
        here(q, a[1]);
        const bool rows3 = q.dim() == 3 && s.T == 1 && q.size(0) == s.B && q.size(1) == s.H && q.size(2) == s.d;
        const bool rows4 = q.dim() == 4 && q.size(0) == s.B && q.size(1) == s.H && q.size(2) == s.T && q.size(3) == s.d;
        want((rows3 || rows4) && q.scalar_type() == at::kBFloat16 && q.is_contiguous(), kQueryWanted);
        want(O.scalar_type() == at::kBFloat16 && O.is_contiguous() && O.device() == q.device() && O.numel() == q.numel(), kQueryWanted);
        want(LSE.scalar_type() == at::kFloat && LSE.is_contiguous() && LSE.device() == q.device() && LSE.numel() == (int64_t)s.B * s.H * s.T, kQueryWanted);
        want(gate.scalar_type() == at::kFloat && gate.is_contiguous() && gate.device() == q.device() && gate.numel() == 3 * (int64_t)s.B * s.T, kGateWanted);
        int64_t w[51];
        put_levels8(w, q, H_kv, s.d, a[5], a[6], a[7], a[8], a[9], a[10], a[11]);
        const Workspace ws(tensor(a[15]), q);
        return call_checked(a[0], &mka_decode_paged8, &s, static_cast<int32_t>(H_kv), q.data_ptr(), reinterpret_cast<const mka_paged_level8*>(w),
                            static_cast<const float*>(gate.data_ptr()), O.data_ptr(), static_cast<float*>(LSE.data_ptr()), ws.v, ws.bytes, Address(a[16]).v);
    });
}
// append8(address, device, K, V, pool_k, pool_v, exp_k, exp_v, table, dst_offset, dst_offsets or None, stream): mka_append_kv_paged8
PyObject* append8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 12) throw Bad{kCountWanted};
        const at::Tensor& K = tensor(a[2]);
        here(K, a[1]);
        int64_t w[23] = {};
        put_append8(w, K, tensor(a[3]), tensor(a[4]), tensor(a[5]), tensor(a[6]), tensor(a[7]), tensor(a[8]));
        const auto dtype = K.scalar_type();
        want(dtype == at::kBFloat16 || dtype == at::kFloat, "rows of bf16 or f32 are expected");
        want(K.size(0) <= INT32_MAX && K.size(1) <= INT32_MAX, kLevels8Wanted);
        return call_checked(a[0], &mka_append_kv_paged8, static_cast<int32_t>(K.size(0)), static_cast<int32_t>(K.size(1)), K.size(2), static_cast<int32_t>(K.size(3)),
                            dtype == at::kBFloat16 ? int32_t{MKA_BF16} : int32_t{MKA_F32}, reinterpret_cast<const mka_level*>(w),
                            reinterpret_cast<const mka_paged_level8*>(w + 6), Arg<int64_t>(a[9]).v, static_cast<const int32_t*>(i32(optional(a[10]), K, K.size(0))),
                            Address(a[11]).v);
    });
}
// pages_resize(address, device, planes, refs, table, rows, new_rows, page_rows, missing or None, ws, stream)
PyObject* pages_resize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 11) throw Bad{kCountWanted};
        const at::Tensor &refs = tensor(a[3]), &rows = tensor(a[5]);
        here(refs, a[1]);
        const mka_page_tables t = tables_of(refs, tensor(a[4]), rows, integer(a[7]));
        const std::vector<mka_page_plane> planes = planes_of(a[2], refs);
        const Workspace ws(tensor(a[9]), refs);
        return call_checked(a[0], &mka_pages_resize, &t, planes.data(), static_cast<int32_t>(planes.size()), static_cast<const int32_t*>(i32(&tensor(a[6]), refs, rows.numel())),
                            i32(optional(a[8]), refs, 1), ws.v, ws.bytes, Address(a[10]).v);
    });
}
// pages_fork(address, device, refs, table, rows, parents, children, page_rows, stream)
PyObject* pages_fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 9) throw Bad{kCountWanted};
        const at::Tensor &refs = tensor(a[2]), &parents = tensor(a[5]);
        here(refs, a[1]);
        const mka_page_tables t = tables_of(refs, tensor(a[3]), tensor(a[4]), integer(a[7]));
        want(parents.numel() <= INT32_MAX, kI32Wanted);
        return call_checked(a[0], &mka_pages_fork, &t, static_cast<const int32_t*>(i32(&parents, refs, parents.numel())),
                            static_cast<const int32_t*>(i32(&tensor(a[6]), refs, parents.numel())), static_cast<int32_t>(parents.numel()), Address(a[8]).v);
    });
}
// pages_compact(address, device, planes, refs, table, rows, page_rows, refs_out, table_out, remap, live or None, ws, stream)
PyObject* pages_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 13) throw Bad{kCountWanted};
        const at::Tensor &refs = tensor(a[3]), &rows = tensor(a[5]);
        here(refs, a[1]);
        const mka_page_tables t = tables_of(refs, tensor(a[4]), rows, integer(a[6])), out = tables_of(refs, tensor(a[8]), rows, integer(a[6]));
        want(out.width == t.width, kTablesWanted);
        const std::vector<mka_page_plane> planes = planes_of(a[2], refs);
        const Workspace ws(tensor(a[11]), refs);
        return call_checked(a[0], &mka_pages_compact, &t, planes.data(), static_cast<int32_t>(planes.size()), i32(&tensor(a[7]), refs, refs.numel()), out.table, out.table_stride,
                            i32(&tensor(a[9]), refs, refs.numel()), i32(optional(a[10]), refs, 1), ws.v, ws.bytes, Address(a[12]).v);
    });
}

PyObject* empty_like(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 1) throw Bad{kCountWanted};
        return THPVariable_Wrap(at::empty_like(tensor(a[0])));
    });
}
PyObject* row_counts(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 1) throw Bad{kCountWanted};
        Seq K(a[0]);
        int64_t rows[3];
        for (int l = 0; l < 3; ++l) {
            const at::Tensor* k = K.tensor_at(l);
            rows[l] = k ? k->size(2) : 0;
        }
        return Py_BuildValue("LLL", static_cast<long long>(rows[0]), static_cast<long long>(rows[1]), static_cast<long long>(rows[2]));
    });
}

template <typename F> PyMethodDef method(const char* name, F f, const char* doc) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, doc};
}
PyMethodDef methods[] = {
    method("levels", levels, "levels(K, V) -> mka_level[3] as bytes; None or no rows: an absent level"),
    method("grads", grads, "grads(K, dK, dV) -> mka_level_grad[3] as bytes; a level absent from K is absent"),
    method("paged_levels", paged_levels, "paged_levels(pools_k, pools_v, tables, rows or None, n) -> mka_paged_level[3] as bytes"),
    method("paged_level", paged_level, "paged_level(pool_k, pool_v, table) -> one mka_paged_level over the table's width as bytes"),
    method("paged_levels8", paged_levels8, "paged_levels8(q, H_kv, pools_k, pools_v, exps_k, exps_v, tables, rows or None, n) -> mka_paged_level8[3] as bytes"),
    method("append_levels8", append_levels8, "append_levels8(K, V, pool_k, pool_v, exp_k, exp_v, table) -> a mka_level and a mka_paged_level8 as bytes"),
    method("page_tables", page_tables, "page_tables(refs, table, rows, page_rows) -> mka_page_tables as bytes"),
    method("page_planes", page_planes, "page_planes(tensors, refs) -> mka_page_plane[] as bytes"),
    method("empties_like", empties_like, "empties_like(tensors) -> list of empty_like, None for None"),
    method("empty_f32", empty_f32, "empty_f32(t, keep, extra) -> fp32 tensor of t's first `keep` dimensions, then `extra` if not 0"),
    method("shape_type", shape_type, "shape_type(cls): the class whose instances are shapes"),
    method("empty_like", empty_like, "empty_like(t)"),
    method("row_counts", row_counts, "row_counts(K) -> the rows of three levels, 0 for None"),
    method("call_router", call_router, "call_router(address, arguments of mka_router...) -> its status"),
    method("call_fwd", call_fwd_with_scratch, "the same for mka_fwd_with_scratch"),
    method("call_fwd_paged", call_fwd_paged_with_scratch, "the same for mka_fwd_paged_with_scratch"),
    method("call_decode", call_decode, "the same for mka_decode"),
    method("call_decode_paged", call_decode_paged, "the same for mka_decode_paged"),
    method("call_bwd", call_bwd, "the same for mka_bwd"),
    method("attend8", attend8, "checks and call of mka_decode_paged8 or mka_fwd_paged8"),
    method("append8", append8, "checks and call of mka_append_kv_paged8"),
    method("pages_resize", pages_resize, "checks and call of mka_pages_resize"),
    method("pages_fork", pages_fork, "checks and call of mka_pages_fork"),
    method("pages_compact", pages_compact, "checks and call of mka_pages_compact"),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host_args", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host_args() { return PyModule_Create(&module); }
