// Argument marshalling of the ctypes-free call path: fills an argument struct of radar.h from a dictionary of Python
// objects (the calls of the 4-bit cache: from positional arguments, further down) and calls the library.  A step makes a dozen calls of thirty arguments each, and where the draft model runs
// between them nothing hides their host time: filled field by field from Python a call took 25 us, of which the library
// and its launches are 5.  RADAR_BUILT_FOR names the torch and Python it is compiled against.  Nothing is kept between calls: every tensor is checked and its address taken each time.
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cstring>
#include <exception>
#include <vector>

#include "../../include/radar.h"

namespace {

enum Kind : int { kInt = 0, kInt64 = 1, kFloat = 2, kPointer = 3 };

struct Field {
    Py_ssize_t offset;
    int kind;
    int dtype;          // c10::ScalarType a tensor must have, -1: any
    bool required;
    bool address;       // a pointer field that may also be given as a plain address
};

struct Filler {
    PyObject_HEAD
    Py_ssize_t size;
    PyObject* index;                    // {name: position in fields}
    std::vector<Field>* fields;
    Py_ssize_t n_required;
};

constexpr Py_ssize_t kMaxStruct = 1024;

// Writes one argument; false with a Python error set.
bool fill(const Field& f, PyObject* name, PyObject* v, unsigned char* out) {
    unsigned char* to = out + f.offset;
    switch (f.kind) {
        case kInt: {
            const long x = PyLong_AsLong(v);
            if (x == -1 && PyErr_Occurred()) return false;
            if (x < INT_MIN || x > INT_MAX) { PyErr_Format(PyExc_OverflowError, "%U does not fit an int", name); return false; }
            const int y = static_cast<int>(x);
            std::memcpy(to, &y, sizeof y);
            return true;
        }
        case kInt64: {
            const long long x = PyLong_AsLongLong(v);
            if (x == -1 && PyErr_Occurred()) return false;
            std::memcpy(to, &x, sizeof x);
            return true;
        }
        case kFloat: {
            const double x = PyFloat_AsDouble(v);
            if (x == -1.0 && PyErr_Occurred()) return false;
            const float y = static_cast<float>(x);
            std::memcpy(to, &y, sizeof y);
            return true;
        }
        default: {
            void* p = nullptr;
            if (v == Py_None) {
            } else if (THPVariable_Check(v)) {
                try {
                    const at::Tensor& t = THPVariable_Unpack(v);
                    if (!t.is_cuda() || !t.is_contiguous()) { PyErr_Format(PyExc_ValueError, "%U: expected a contiguous CUDA tensor", name); return false; }
                    if (f.dtype >= 0 && static_cast<int>(t.scalar_type()) != f.dtype) {
                        PyErr_Format(PyExc_ValueError, "%U: expected dtype %s, got %s", name, c10::toString(static_cast<c10::ScalarType>(f.dtype)),
                                     c10::toString(t.scalar_type()));
                        return false;
                    }
                    p = t.data_ptr();
                } catch (const std::exception& e) {
                    PyErr_SetString(PyExc_RuntimeError, e.what());
                    return false;
                }
            } else if (f.address) {
                p = PyLong_AsVoidPtr(v);
                if (p == nullptr && PyErr_Occurred()) return false;
            } else {
                PyErr_Format(PyExc_TypeError, "%U: expected a tensor or None, got %s", name, Py_TYPE(v)->tp_name);
                return false;
            }
            std::memcpy(to, &p, sizeof p);
            return true;
        }
    }
}

// filler(function address, context handle, stream handle, {name: value}) -> status
PyObject* filler_call(PyObject* self_, PyObject* args, PyObject* kwargs) {
    Filler* self = reinterpret_cast<Filler*>(self_);
    if (kwargs != nullptr && PyDict_GET_SIZE(kwargs) != 0) { PyErr_SetString(PyExc_TypeError, "positional arguments only"); return nullptr; }
    PyObject *fn, *ctx, *stream, *dict;
    if (!PyArg_UnpackTuple(args, "call", 4, 4, &fn, &ctx, &stream, &dict)) return nullptr;
    if (!PyDict_Check(dict)) { PyErr_SetString(PyExc_TypeError, "expected a dictionary"); return nullptr; }
    void* const f = PyLong_AsVoidPtr(fn);
    if (f == nullptr) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null function"); return nullptr; }
    void* const c = PyLong_AsVoidPtr(ctx);
    if (c == nullptr && PyErr_Occurred()) return nullptr;
    void* const s = PyLong_AsVoidPtr(stream);
    if (s == nullptr && PyErr_Occurred()) return nullptr;
    alignas(16) unsigned char buf[kMaxStruct];
    std::memset(buf, 0, static_cast<size_t>(self->size));
    Py_ssize_t pos = 0, required = 0;
    PyObject *key, *value;
    while (PyDict_Next(dict, &pos, &key, &value)) {
        PyObject* at = PyDict_GetItemWithError(self->index, key);
        if (at == nullptr) {
            if (!PyErr_Occurred()) PyErr_Format(PyExc_TypeError, "unexpected keyword argument '%S'", key);
            return nullptr;
        }
        const Field& fld = (*self->fields)[static_cast<size_t>(PyLong_AsSsize_t(at))];
        if (!fill(fld, key, value, buf)) return nullptr;
        required += fld.required ? 1 : 0;
    }
    if (required != self->n_required) {
        PyObject *name, *at;
        for (pos = 0; PyDict_Next(self->index, &pos, &name, &at);)
            if ((*self->fields)[static_cast<size_t>(PyLong_AsSsize_t(at))].required && PyDict_GetItemWithError(dict, name) == nullptr) {
                PyErr_Format(PyExc_TypeError, "missing required keyword argument '%S'", name);
                return nullptr;
            }
    }
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = reinterpret_cast<int (*)(void*, const void*, void*)>(f)(c, buf, s);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// Filler(struct size, [(name, offset, kind, dtype, required, address), ...]); dtype: a tensor of the type, or None
PyObject* filler_new(PyTypeObject* type, PyObject* args, PyObject*) {
    Py_ssize_t size;
    PyObject* list;
    if (!PyArg_ParseTuple(args, "nO!", &size, &PyList_Type, &list)) return nullptr;
    if (size <= 0 || size > kMaxStruct) { PyErr_SetString(PyExc_ValueError, "struct size out of range"); return nullptr; }
    Filler* self = reinterpret_cast<Filler*>(type->tp_alloc(type, 0));
    if (self == nullptr) return nullptr;
    self->size = size;
    self->n_required = 0;
    self->index = PyDict_New();
    self->fields = new std::vector<Field>;
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list); ++i) {
        PyObject *name, *dtype;
        Py_ssize_t offset;
        int kind, required, address;
        if (!PyArg_ParseTuple(PyList_GET_ITEM(list, i), "O!niOpp", &PyUnicode_Type, &name, &offset, &kind, &dtype, &required, &address)) { Py_DECREF(self); return nullptr; }
        const Py_ssize_t bytes = kind == kInt || kind == kFloat ? 4 : 8;
        if (kind < kInt || kind > kPointer || offset < 0 || offset + bytes > size) { Py_DECREF(self); PyErr_SetString(PyExc_ValueError, "bad field"); return nullptr; }
        Field f{offset, kind, -1, required != 0, address != 0};
        if (dtype != Py_None) {
            if (!THPVariable_Check(dtype)) { Py_DECREF(self); PyErr_SetString(PyExc_TypeError, "dtype: a tensor of the type, or None"); return nullptr; }
            f.dtype = static_cast<int>(THPVariable_Unpack(dtype).scalar_type());
        }
        PyObject* at = PyLong_FromSsize_t(static_cast<Py_ssize_t>(self->fields->size()));
        self->fields->push_back(f);
        self->n_required += f.required ? 1 : 0;
        const int rc = at == nullptr ? -1 : PyDict_SetItem(self->index, name, at);
        Py_XDECREF(at);
        if (rc != 0) { Py_DECREF(self); return nullptr; }
    }
    return reinterpret_cast<PyObject*>(self);
}

void filler_dealloc(PyObject* self_) {
    Filler* self = reinterpret_cast<Filler*>(self_);
    Py_XDECREF(self->index);
    delete self->fields;
    PyTypeObject* type = Py_TYPE(self_);
    type->tp_free(self_);
    Py_DECREF(type);
}

// ---- the calls of the 4-bit cache -------------------------------------------------------------------------------------
// Their arguments follow from the tensors' shapes and strides, which costs Python more than the calls' kernels take (a single token's
// attention 17 us a call from Python, its kernels 6); so these are read, checked and filled in here.  Positional arguments:
// function address, context handle, stream handle, then as binding.py documents them.
struct Bad : std::exception {};                     // a Python error is set

[[noreturn]] void refuse(const char* text) { PyErr_SetString(PyExc_ValueError, text); throw Bad(); }
void need(bool ok, const char* text) { if (!ok) refuse(text); }

const at::Tensor* tensor(PyObject* v, const char* name, bool optional = false) {
    if (v == Py_None && optional) return nullptr;
    if (!THPVariable_Check(v)) { PyErr_Format(PyExc_TypeError, "%s: expected a tensor%s, got %s", name, optional ? " or None" : "", Py_TYPE(v)->tp_name); throw Bad(); }
    const at::Tensor& t = THPVariable_Unpack(v);
    if (!t.is_cuda()) { PyErr_Format(PyExc_ValueError, "%s: expected a CUDA tensor", name); throw Bad(); }
    return &t;
}
template <typename T = void>
T* packed(PyObject* v, const char* name, at::ScalarType dtype, bool optional = false, const at::Tensor** out = nullptr) {
    const at::Tensor* t = tensor(v, name, optional);
    if (out != nullptr) *out = t;
    if (t == nullptr) return nullptr;
    if (!t->is_contiguous()) { PyErr_Format(PyExc_ValueError, "%s: expected a contiguous CUDA tensor", name); throw Bad(); }
    if (t->scalar_type() != dtype) { PyErr_Format(PyExc_ValueError, "%s: expected dtype %s, got %s", name, c10::toString(dtype), c10::toString(t->scalar_type())); throw Bad(); }
    return static_cast<T*>(t->data_ptr());
}
long long whole(PyObject* v, long long lo, long long hi, const char* name) {
    const long long x = PyLong_AsLongLong(v);
    if (x == -1 && PyErr_Occurred()) throw Bad();
    if (x < lo || x > hi) { PyErr_Format(PyExc_OverflowError, "%s does not fit", name); throw Bad(); }
    return x;
}
int small(PyObject* v, const char* name) { return static_cast<int>(whole(v, INT_MIN, INT_MAX, name)); }
// rows [..., heads, d] whose leading dimensions may have any strides, the last two lie together
void* strided_rows(const at::Tensor& t, int64_t dims, const char* name) {
    if (t.dim() != dims || t.stride(-1) != 1 || (t.size(-2) != 1 && t.stride(-2) != t.size(-1))) {
        PyErr_Format(PyExc_ValueError, "%s: expected a CUDA tensor of %d dimensions whose last two are contiguous", name, static_cast<int>(dims));
        throw Bad();
    }
    return t.data_ptr();
}
// (tensors of one shape; the stride of a dimension of one element leads nowhere)
bool same_strides(const at::Tensor& x, const at::Tensor& y) {
    for (int64_t i = 0; i < x.dim(); ++i)
        if (x.size(i) > 1 && x.stride(i) != y.stride(i)) return false;
    return true;
}
int dtype_code(const at::Tensor& t) {
    if (t.scalar_type() == at::kFloat) return RADAR_F32;
    if (t.scalar_type() == at::kBFloat16) return RADAR_BF16;
    PyErr_Format(PyExc_ValueError, "unsupported dtype %s", c10::toString(t.scalar_type()));
    throw Bad();
}
// pages of a pool [n_pages, page bytes] or [n_layers, n_pages, page bytes]
struct Pool { void* p; int64_t n_pages, layer_bytes; };
Pool pool(PyObject* v, int64_t page_size, int64_t Hkv, int64_t d, int64_t n_layers) {
    const at::Tensor* t;
    void* p = packed(v, "pages", at::kByte, false, &t);
    const int64_t bytes = page_size > 0 && page_size % 16 == 0 ? Hkv * (page_size / 16) * 18 * d : -1;
    if ((t->dim() != 2 && t->dim() != 3) || t->size(-1) != bytes || (t->dim() == 3 ? t->size(0) : 1) != n_layers) {
        PyErr_Format(PyExc_ValueError, "pages: expected [%lld layers, n_pages, %lld] (without the first dimension for one layer)", static_cast<long long>(n_layers),
                     static_cast<long long>(bytes));
        throw Bad();
    }
    return {p, t->size(-2), t->size(-2) * bytes};
}

template <typename Fill>
PyObject* cache_call(PyObject* const* args, Py_ssize_t n, Py_ssize_t want, Fill fill_args) {
    if (n != want) { PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n); return nullptr; }
    try {
        void* const f = PyLong_AsVoidPtr(args[0]);
        void* const c = PyLong_AsVoidPtr(args[1]);
        void* const s = PyLong_AsVoidPtr(args[2]);
        if (PyErr_Occurred()) return nullptr;
        if (f == nullptr) { PyErr_SetString(PyExc_ValueError, "null function"); return nullptr; }
        auto a = fill_args(args + 3);
        int status;
        Py_BEGIN_ALLOW_THREADS
        status = reinterpret_cast<int (*)(void*, const void*, void*)>(f)(c, &a, s);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(status);
    } catch (const Bad&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// page_size, cache_len, new_len, extra, block_table, free_pages, free_count, slots, start, granted, cache_len_out, free_count_out, path_nodes, rows, src_row
PyObject* cache_extend(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return cache_call(args, n, 18, [](PyObject* const* v) {
        radar_cache_extend_args a = {};
        const at::Tensor *len, *nu, *table, *stack, *slots, *start, *granted, *path, *src, *len_out;
        a.page_size = small(v[0], "page_size");
        a.cache_len = packed<int32_t>(v[1], "cache_len", at::kInt, false, &len);
        a.new_len = packed<int32_t>(v[2], "new_len", at::kInt, false, &nu);
        a.extra = small(v[3], "extra");
        a.block_table = packed<int32_t>(v[4], "block_table", at::kInt, false, &table);
        a.free_pages = packed<int32_t>(v[5], "free_pages", at::kInt, false, &stack);
        a.free_count = packed<int32_t>(v[6], "free_count", at::kInt);
        a.slots = packed<int64_t>(v[7], "slots", at::kLong, false, &slots);
        a.start = packed<int32_t>(v[8], "start", at::kInt, false, &start);
        a.granted = packed<uint8_t>(v[9], "granted", at::kByte, false, &granted);
        a.cache_len_out = packed<int32_t>(v[10] == Py_None ? v[1] : v[10], "cache_len_out", at::kInt, false, &len_out);
        a.free_count_out = packed<int32_t>(v[11] == Py_None ? v[6] : v[11], "free_count_out", at::kInt);
        const int64_t B = len->numel();
        need(table->dim() == 2 && table->size(0) == B && nu->numel() == B && granted->numel() == B && start->numel() == B + 1 && len_out->numel() == B,
             "radar_cache_extend: cache_len, new_len, granted [B], block_table [B, max_pages] and start [B + 1] disagree about B");
        need(B <= INT_MAX && table->size(1) <= INT_MAX && stack->numel() <= INT_MAX, "radar_cache_extend: more than an int counts");
        a.B = static_cast<int>(B);
        a.max_pages = static_cast<int>(table->size(1));
        a.free_capacity = static_cast<int>(stack->numel());
        a.slot_capacity = slots->numel();
        a.path_nodes = packed<int32_t>(v[12], "path_nodes", at::kInt, true, &path);
        if (path != nullptr) {
            a.rows = small(v[13], "rows");
            a.src_row = packed<int32_t>(v[14], "src_row", at::kInt, true, &src);
            need(path->dim() == 2 && path->size(0) == B && path->size(1) <= INT_MAX && src != nullptr && src->numel() >= a.slot_capacity,
                 "radar_cache_extend: path_nodes [B, columns] needs src_row of at least the slots' size");
            a.path_stride = static_cast<int>(path->size(1));
        }
        return a;
    });
}

// K, V, slots, pages, page_size, src_row
PyObject* cache_store(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return cache_call(args, n, 9, [](PyObject* const* v) {
        radar_cache_store_args a = {};
        const at::Tensor &K = *tensor(v[0], "K"), &V = *tensor(v[1], "V"), *slots, *src;
        need((K.dim() == 3 || K.dim() == 4) && K.sizes() == V.sizes() && K.scalar_type() == V.scalar_type() && same_strides(K, V),
             "K and V must share shape, dtype and strides");
        const bool layers = K.dim() == 4;
        const int64_t rows = K.size(-3), Hkv = K.size(-2), d = K.size(-1);
        need(Hkv <= INT_MAX && d <= INT_MAX && K.size(0) <= INT_MAX, "K and V: too large");
        a.n_layers = layers ? static_cast<int>(K.size(0)) : 1;
        a.Hkv = static_cast<int>(Hkv);
        a.d = static_cast<int>(d);
        a.page_size = small(v[4], "page_size");
        a.dtype = dtype_code(K);
        a.K = strided_rows(K, K.dim(), "K");
        a.V = strided_rows(V, K.dim(), "V");
        a.slots = packed<int64_t>(v[2], "slots", at::kLong, false, &slots);
        a.src_row = packed<int32_t>(v[5], "src_row", at::kInt, true, &src);
        a.n_tokens = slots->numel();
        a.n_rows = rows;
        a.row_stride = rows > 1 ? K.stride(-3) : Hkv * d;
        a.row_layer_stride = a.n_layers > 1 ? K.stride(0) : 0;
        need((src == nullptr ? rows : src->numel()) >= a.n_tokens, "fewer rows (or entries of src_row) than slots");
        const Pool p = pool(v[3], a.page_size, Hkv, d, a.n_layers);
        a.pages = p.p; a.n_pages = p.n_pages; a.page_layer_stride = p.layer_bytes;
        return a;
    });
}

// pages, page_size, block_table, first, start, K, V
PyObject* cache_load(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return cache_call(args, n, 10, [](PyObject* const* v) {
        radar_cache_load_args a = {};
        const at::Tensor &K = *tensor(v[5], "K"), &V = *tensor(v[6], "V"), *table, *first, *start;
        need((K.dim() == 3 || K.dim() == 4) && K.sizes() == V.sizes() && K.scalar_type() == V.scalar_type(), "K and V must share shape and dtype");
        need(K.is_contiguous() && V.is_contiguous(), "K and V: expected contiguous CUDA tensors");
        const int64_t rows = K.size(-3), Hkv = K.size(-2), d = K.size(-1);
        need(Hkv <= INT_MAX && d <= INT_MAX && K.size(0) <= INT_MAX, "K and V: too large");
        a.n_layers = K.dim() == 4 ? static_cast<int>(K.size(0)) : 1;
        a.Hkv = static_cast<int>(Hkv);
        a.d = static_cast<int>(d);
        a.page_size = small(v[1], "page_size");
        a.dtype = dtype_code(K);
        a.n_rows = rows;
        a.K = K.data_ptr();
        a.V = V.data_ptr();
        a.row_layer_stride = rows * Hkv * d;
        a.block_table = packed<int32_t>(v[2], "block_table", at::kInt, false, &table);
        a.first = packed<int32_t>(v[3], "first", at::kInt, false, &first);
        a.start = packed<int32_t>(v[4], "start", at::kInt, false, &start);
        const int64_t B = first->numel();
        need(B <= INT_MAX && table->dim() == 2 && table->size(0) == B && table->size(1) <= INT_MAX && start->numel() == B + 1,
             "block_table [B, max_pages], first [B] and start [B + 1] disagree about B");
        a.B = static_cast<int>(B);
        a.max_pages = static_cast<int>(table->size(1));
        const Pool p = pool(v[0], a.page_size, Hkv, d, a.n_layers);
        a.pages = p.p; a.n_pages = p.n_pages; a.page_layer_stride = p.layer_bytes;
        return a;
    });
}

// Q, Kt, Vt, pages, page_size, block_table, cache_len, max_cache_len, O, workspace, mask, n_nodes, lse, scale
PyObject* cache_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return cache_call(args, n, 17, [](PyObject* const* v) {
        radar_cache_attn_args a = {};
        const at::Tensor &Q = *tensor(v[0], "Q"), &Kt = *tensor(v[1], "Kt"), &Vt = *tensor(v[2], "Vt"), *table, *len, *O, *mask, *nodes, *lse, *ws;
        need(Q.dim() == 4 && Kt.dim() == 4 && Q.scalar_type() == at::kBFloat16 && Kt.scalar_type() == at::kBFloat16 && Vt.scalar_type() == at::kBFloat16,
             "Q, Kt and Vt: expected bfloat16 [B, rows, heads, d]");
        const int64_t B = Q.size(0), rows = Q.size(1), Hq = Q.size(2), Hkv = Kt.size(2), d = Q.size(3);
        need(B <= INT_MAX && rows <= INT_MAX && Hq <= INT_MAX && d <= INT_MAX, "Q: too large");
        a.O = packed(v[8], "O", at::kBFloat16, false, &O);
        need(Kt.sizes() == Vt.sizes() && Kt.size(0) == B && Kt.size(1) == rows && Kt.size(3) == d && O->sizes() == Q.sizes() && same_strides(Kt, Vt),
             "Q, O, Kt and Vt disagree in shape or strides");
        need(B == 1 || rows == 1 || (Q.stride(0) == rows * Q.stride(1) && Kt.stride(0) == rows * Kt.stride(1)),
             "Q, Kt, Vt: the rows of a sequence must follow those of the one before");
        a.B = static_cast<int>(B); a.Hq = static_cast<int>(Hq); a.Hkv = static_cast<int>(Hkv); a.d = static_cast<int>(d); a.rows = static_cast<int>(rows);
        a.dtype = RADAR_BF16;
        a.Q = strided_rows(Q, 4, "Q");
        a.Kt = strided_rows(Kt, 4, "Kt");
        a.Vt = strided_rows(Vt, 4, "Vt");
        auto stride = [&](const at::Tensor& t) { return rows > 1 ? t.stride(1) : B > 1 ? t.stride(0) : t.size(2) * d; };
        a.q_row_stride = stride(Q);
        a.kv_row_stride = stride(Kt);
        a.page_size = small(v[4], "page_size");
        a.block_table = packed<int32_t>(v[5], "block_table", at::kInt, false, &table);
        a.cache_len = packed<int32_t>(v[6], "cache_len", at::kInt, false, &len);
        a.max_cache_len = small(v[7], "max_cache_len");
        a.workspace = packed(v[9], "workspace", at::kByte, false, &ws);
        a.workspace_bytes = static_cast<size_t>(ws->numel());
        a.mask = reinterpret_cast<const uint64_t*>(packed<int64_t>(v[10], "mask", at::kLong, true, &mask));
        a.n_nodes = packed<int32_t>(v[11], "n_nodes", at::kInt, true, &nodes);
        a.lse = packed<float>(v[12], "lse", at::kFloat, true, &lse);
        const double scale = PyFloat_AsDouble(v[13]);
        if (scale == -1.0 && PyErr_Occurred()) throw Bad();
        a.scale = static_cast<float>(scale);
        need(table->dim() == 2 && table->size(0) == B && table->size(1) <= INT_MAX && len->numel() == B && (nodes == nullptr || nodes->numel() == B) &&
                 (mask == nullptr || (mask->dim() == 2 && mask->size(0) == B && mask->size(1) == rows)) &&
                 (lse == nullptr || (lse->dim() == 3 && lse->size(0) == B && lse->size(1) == Hq && lse->size(2) == rows)),
             "block_table, cache_len, n_nodes, mask or lse disagree with Q");
        a.max_pages = static_cast<int>(table->size(1));
        const Pool p = pool(v[3], a.page_size, Hkv, d, 1);
        a.pages = p.p; a.n_pages = p.n_pages;
        return a;
    });
}

// ---- rows with positions and the paged cache: as above, behind the number of the current device, which every tensor has to be on --------
thread_local int current_device = -1;
void here(const at::Tensor* t, const char* name) {
    if (t != nullptr && t->device().index() != current_device) { PyErr_Format(PyExc_ValueError, "%s: not on the current device", name); throw Bad(); }
}
const at::Tensor* rows_of(PyObject* v, const char* name, int64_t min_dim, int64_t max_dim) {
    const at::Tensor* t = tensor(v, name, true);
    if (t == nullptr) return nullptr;
    here(t, name);
    if (t->dim() < min_dim || t->dim() > max_dim) { PyErr_Format(PyExc_ValueError, "%s: a tensor of another number of dimensions", name); throw Bad(); }
    strided_rows(*t, t->dim(), name);
    for (int64_t i = 0; i < t->dim(); ++i) need(t->size(i) <= INT_MAX, "rows, heads or channels: more than an int counts");
    return t;
}
template <typename T>
T* packed_here(PyObject* v, const char* name, at::ScalarType dtype, bool optional = false, const at::Tensor** out = nullptr) {
    const at::Tensor* t;
    T* p = packed<T>(v, name, dtype, optional, &t);
    here(t, name);
    if (out != nullptr) *out = t;
    return p;
}
int64_t row_stride(const at::Tensor& t) { return t.size(-3) > 1 ? t.stride(-3) : t.size(-2) * t.size(-1); }
int64_t layer_stride(const at::Tensor& t) { return t.dim() == 4 && t.size(0) > 1 ? t.stride(0) : 0; }

// pos, inv_freq, pair_axis, neighbours
void rotation(PyObject* const* v, int64_t n, radar_rotation& r) {
    const at::Tensor *pos, *freq, *axis;
    r.pos = packed_here<int32_t>(v[0], "pos", at::kInt, true, &pos);
    if (pos == nullptr) return;
    need(pos->dim() == 1 || pos->dim() == 2, "pos: expected [rows] or [axes, rows]");
    need(pos->size(-1) >= n, "pos: fewer positions than rows");
    r.pos_stride = pos->size(-1);
    r.n_axes = pos->dim() == 2 ? static_cast<int>(pos->size(0)) : 1;
    r.inv_freq = packed_here<float>(v[1], "inv_freq", at::kFloat, false, &freq);
    need(freq->numel() <= INT_MAX, "inv_freq: too large");
    r.n_pairs = static_cast<int>(freq->numel());
    r.pair_axis = packed_here<uint8_t>(v[2], "pair_axis", at::kByte, true, &axis);
    need(axis == nullptr || axis->numel() == freq->numel(), "pair_axis and inv_freq disagree");
    const int on = PyObject_IsTrue(v[3]);
    if (on < 0) throw Bad();
    r.neighbours = on;
}
int set_device(PyObject* v) { return current_device = small(v, "device"); }

// device, Q, Q_out, K, K_out, pos, inv_freq, pair_axis, neighbours, inverse
PyObject* rotate(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return cache_call(args, n, 13, [](PyObject* const* v) {
        radar_rotate_args a = {};
        set_device(v[0]);
        const at::Tensor *Q = rows_of(v[1], "Q", 3, 3), *Qo = rows_of(v[2], "Q_out", 3, 3), *K = rows_of(v[3], "K", 3, 3), *Ko = rows_of(v[4], "K_out", 3, 3);
        const at::Tensor* X = Q != nullptr ? Q : K;
        need(X != nullptr, "Q or K: expected a tensor");
        need((Q == nullptr) == (Qo == nullptr) && (K == nullptr) == (Ko == nullptr), "Q_out and K_out: one for each of Q and K");
        for (const at::Tensor* t : {Q, Qo, K, Ko})
            need(t == nullptr || (t->scalar_type() == X->scalar_type() && t->size(0) == X->size(0) && t->size(2) == X->size(2)), "Q, K and their outputs disagree in rows, d or dtype");
        need((Q == nullptr || Q->sizes() == Qo->sizes()) && (K == nullptr || K->sizes() == Ko->sizes()), "Q_out and K_out: the shapes of Q and K");
        a.dtype = dtype_code(*X);
        a.n_rows = X->size(0);
        a.d = static_cast<int>(X->size(2));
        if (Q != nullptr) { a.Hq = static_cast<int>(Q->size(1)); a.Q = Q->data_ptr(); a.Q_out = Qo->data_ptr(); a.q_row_stride = row_stride(*Q); a.q_out_row_stride = row_stride(*Qo); }
        if (K != nullptr) { a.Hkv = static_cast<int>(K->size(1)); a.K = K->data_ptr(); a.K_out = Ko->data_ptr(); a.k_row_stride = row_stride(*K); a.k_out_row_stride = row_stride(*Ko); }
        rotation(v + 5, a.n_rows, a.rotation);
        need(v[5] != Py_None, "pos: expected a tensor");
        const int on = PyObject_IsTrue(v[9]);
        if (on < 0) throw Bad();
        a.inverse = on;
        return a;
    });
}

// device, K, V, slots, src_row, Kc, Vc, Q, Q_out, pos, inv_freq, pair_axis, neighbours
PyObject* paged_store(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return cache_call(args, n, 16, [](PyObject* const* v) {
        radar_paged_store_args a = {};
        set_device(v[0]);
        const at::Tensor *K = rows_of(v[1], "K", 3, 4), *V = rows_of(v[2], "V", 3, 4), *slots, *src, *Kc, *Vc;
        need(K != nullptr && V != nullptr, "K, V: expected tensors");
        need(K->sizes() == V->sizes() && K->scalar_type() == V->scalar_type() && same_strides(*K, *V), "K and V must share shape, dtype and strides");
        const bool layers = K->dim() == 4;
        a.n_layers = layers ? static_cast<int>(K->size(0)) : 1;
        a.Hkv = static_cast<int>(K->size(-2));
        a.d = static_cast<int>(K->size(-1));
        a.dtype = dtype_code(*K);
        a.n_rows = K->size(-3);
        a.K = K->data_ptr(); a.V = V->data_ptr();
        a.kv_row_stride = row_stride(*K); a.kv_layer_stride = layer_stride(*K);
        a.slots = packed_here<int64_t>(v[3], "slots", at::kLong, false, &slots);
        a.src_row = packed_here<int32_t>(v[4], "src_row", at::kInt, true, &src);
        a.n_tokens = slots->numel();
        need((src == nullptr ? a.n_rows : src->numel()) >= a.n_tokens, "fewer rows (or entries of src_row) than slots");
        a.Kc = packed_here<void>(v[5], "Kc", K->scalar_type(), false, &Kc);
        a.Vc = packed_here<void>(v[6], "Vc", K->scalar_type(), false, &Vc);
        const int64_t row = static_cast<int64_t>(a.Hkv) * a.d, layer = a.n_layers > 0 ? Kc->numel() / a.n_layers : 0;
        need(Kc->dim() >= 3 && Kc->sizes() == Vc->sizes() && Kc->size(-1) == a.d && Kc->size(-2) == a.Hkv && (!layers || (Kc->dim() >= 4 && Kc->size(0) == a.n_layers)),
             "Kc, Vc: expected [cache rows, Hkv, d] (the rows in as many dimensions as there are), behind the layers' dimension if K has one");
        a.cache_rows = row > 0 ? layer / row : 0;
        a.cache_layer_stride = a.n_layers > 1 ? layer : 0;
        const at::Tensor *Q = rows_of(v[7], "Q", 3, 4), *Qo = rows_of(v[8], "Q_out", 3, 4);
        need((Q == nullptr) == (Qo == nullptr), "Q_out: one for Q, and none without");
        if (Q != nullptr) {
            need(Q->dim() == K->dim() && Qo->dim() == K->dim() && Q->scalar_type() == K->scalar_type() && Qo->scalar_type() == K->scalar_type() && Q->size(-3) == a.n_rows &&
                     Q->size(-1) == a.d && Qo->size(-1) == a.d && Qo->size(-2) == Q->size(-2) && Qo->size(-3) >= a.n_tokens && (!layers || (Q->size(0) == a.n_layers && Qo->size(0) == a.n_layers)),
                 "Q and Q_out disagree with K in layers, rows, d or dtype");
            a.Hq = static_cast<int>(Q->size(-2));
            a.Q = Q->data_ptr(); a.Q_out = Qo->data_ptr();
            a.q_row_stride = row_stride(*Q); a.q_layer_stride = layer_stride(*Q);
            a.q_out_row_stride = row_stride(*Qo); a.q_out_layer_stride = layer_stride(*Qo);
        }
        rotation(v + 9, a.n_tokens, a.rotation);
        return a;
    });
}

// device, Q, q_start, Kc, Vc, page_size, block_table, cache_len, max_new, max_cache_len, O, workspace, lse, scale
PyObject* chunk_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return cache_call(args, n, 17, [](PyObject* const* v) {
        radar_chunk_attn_args a = {};
        set_device(v[0]);
        const at::Tensor *Q = rows_of(v[1], "Q", 3, 3), *start, *Kc, *Vc, *table, *len, *O, *lse, *ws;
        need(Q != nullptr, "Q: expected a tensor");
        a.dtype = dtype_code(*Q);
        a.Hq = static_cast<int>(Q->size(1));
        a.d = static_cast<int>(Q->size(2));
        a.n_rows = Q->size(0);
        a.Q = Q->data_ptr();
        a.q_row_stride = row_stride(*Q);
        a.q_start = packed_here<int32_t>(v[2], "q_start", at::kInt, false, &start);
        a.Kc = packed_here<void>(v[3], "Kc", Q->scalar_type(), false, &Kc);
        a.Vc = packed_here<void>(v[4], "Vc", Q->scalar_type(), false, &Vc);
        need(Kc->dim() >= 3 && Kc->sizes() == Vc->sizes() && Kc->size(-1) == a.d && Kc->size(-2) > 0 && Kc->size(-2) <= INT_MAX && a.d > 0,
             "Kc, Vc: expected [cache rows, Hkv, d] (the rows in as many dimensions as there are) with the d of Q");
        a.Hkv = static_cast<int>(Kc->size(-2));
        a.cache_rows = Kc->numel() / (Kc->size(-2) * a.d);
        a.page_size = small(v[5], "page_size");
        a.block_table = packed_here<int32_t>(v[6], "block_table", at::kInt, false, &table);
        a.cache_len = packed_here<int32_t>(v[7], "cache_len", at::kInt, false, &len);
        a.max_new = small(v[8], "max_new");
        a.max_cache_len = small(v[9], "max_cache_len");
        a.O = packed_here<void>(v[10], "O", Q->scalar_type(), false, &O);
        a.workspace = packed_here<void>(v[11], "workspace", at::kByte, false, &ws);
        a.workspace_bytes = static_cast<size_t>(ws->numel());
        a.lse = packed_here<float>(v[12], "lse", at::kFloat, true, &lse);
        const double scale = PyFloat_AsDouble(v[13]);
        if (scale == -1.0 && PyErr_Occurred()) throw Bad();
        a.scale = static_cast<float>(scale);
        const int64_t B = len->numel();
        need(B <= INT_MAX && start->numel() == B + 1 && table->dim() == 2 && table->size(0) == B && table->size(1) <= INT_MAX, "q_start [B + 1], block_table [B, max_pages] and cache_len [B] disagree about B");
        need(O->sizes() == Q->sizes() && (lse == nullptr || (lse->dim() == 2 && lse->size(0) == a.n_rows && lse->size(1) == a.Hq)), "O and lse [rows, Hq]: the shape of Q");
        a.B = static_cast<int>(B);
        a.max_pages = static_cast<int>(table->size(1));
        return a;
    });
}

#define RADAR_FASTCALL(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef cache_methods[] = {RADAR_FASTCALL(cache_extend), RADAR_FASTCALL(cache_store), RADAR_FASTCALL(cache_load), RADAR_FASTCALL(cache_attention),
                               RADAR_FASTCALL(rotate), RADAR_FASTCALL(paged_store), RADAR_FASTCALL(chunk_attention), {nullptr, nullptr, 0, nullptr}};

PyType_Slot filler_slots[] = {{Py_tp_new, reinterpret_cast<void*>(filler_new)},
                              {Py_tp_call, reinterpret_cast<void*>(filler_call)},
                              {Py_tp_dealloc, reinterpret_cast<void*>(filler_dealloc)},
                              {0, nullptr}};
PyType_Spec filler_spec = {"_marshal.Filler", sizeof(Filler), 0, Py_TPFLAGS_DEFAULT, filler_slots};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, cache_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
    PyObject* m = PyModule_Create(&module_def);
    if (m == nullptr) return nullptr;
    PyObject* type = PyType_FromSpec(&filler_spec);
    if (type == nullptr || PyModule_AddStringConstant(m, "BUILT_FOR", RADAR_BUILT_FOR) != 0 || PyModule_AddObject(m, "Filler", type) != 0) {
        Py_XDECREF(type);
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
