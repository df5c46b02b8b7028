// Argument marshalling of the paged-cache operations for torch tensors: checks, outputs, device, stream, and the call of the C
// entry point (include/nnc.h).  These calls are short on the device (3 to 12 us for a decoding step's), so what the host does
// for each counts: through Python and ctypes it was 6 to 11 us, here it is mostly the launch itself.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <optional>
#include <utility>
#include <vector>

#include "../../include/nnc.h"

namespace {

decltype(&nnc_op_rope) call_rope;
decltype(&nnc_op_kv_write_paged) call_write;
decltype(&nnc_op_kv_read_paged) call_read;
decltype(&nnc_op_attn_decode_paged) call_attn;
PyObject *error_class;   // NncError(status, detail)

struct Refused {};   // a Python error is set

[[noreturn]] void refuse(const char *what) {
    PyErr_SetString(PyExc_ValueError, what);
    throw Refused();
}

const at::Tensor &tensor(PyObject *o, const char *what) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: a tensor", what);
        throw Refused();
    }
    return THPVariable_Unpack(o);
}

int type_of(at::ScalarType t) {
    return t == at::kFloat ? NNC_F32 : t == at::kBFloat16 ? NNC_BF16 : t == at::kHalf ? NNC_F16 : -1;
}

// [tokens][heads][head_dim] with contiguous heads
struct Rows {
    int type;
    int64_t tokens, heads, d, row, head;
    bool like(const Rows &o) const { return type == o.type && tokens == o.tokens && heads == o.heads && d == o.d; }
};

Rows rows_of(const at::Tensor &t, int device, const char *what) {
    Rows r{};
    r.type = type_of(t.scalar_type());
    if (r.type < 0 || t.dim() != 3 || !t.is_cuda() || t.get_device() != device) {
        PyErr_Format(PyExc_ValueError, "%s: [tokens][heads][head_dim] of float32, bfloat16 or float16 on one CUDA device with the other tensors of the call", what);
        throw Refused();
    }
    r.tokens = t.size(0); r.heads = t.size(1); r.d = t.size(2);
    if (t.stride(2) != 1 && r.d > 1) {
        PyErr_Format(PyExc_ValueError, "%s: elements of a head next to each other", what);
        throw Refused();
    }
    if (r.tokens > INT32_MAX || r.heads > INT32_MAX || r.d > INT32_MAX) refuse("sizes: 32-bit numbers");
    r.head = r.heads > 1 ? t.stride(1) : r.d;            // strides that nothing is reached by do not count
    r.row = r.tokens > 1 ? t.stride(0) : r.heads * r.head;
    return r;
}

const int32_t *index_of(const at::Tensor &t, int64_t n, int device, const char *what) {
    if (t.scalar_type() != at::kInt || t.dim() != 1 || t.size(0) != n || !t.is_contiguous() || !t.is_cuda() || t.get_device() != device) {
        PyErr_Format(PyExc_ValueError, "%s: %lld contiguous int32 numbers on the call's CUDA device", what, (long long)n);
        throw Refused();
    }
    return static_cast<const int32_t *>(t.data_ptr());
}

// no two elements share memory, as far as sorted strides show it
bool disjoint(const at::Tensor &t) {
    if (t.is_contiguous()) return true;
    std::vector<std::pair<int64_t, int64_t>> dims;
    for (int64_t i = 0; i < t.dim(); ++i)
        if (t.size(i) > 1) dims.emplace_back(t.stride(i), t.size(i));
    std::sort(dims.begin(), dims.end());
    int64_t span = 1;
    for (auto &d : dims) {
        if (d.first < span) return false;
        span += d.first * (d.second - 1);
    }
    return true;
}

// Memory that a call reads or writes: `size` bytes from `base` plus every sum of its steps, each taken 0 .. count - 1 times.
struct Region {
    struct Step { int64_t bytes, count; };
    int64_t base, size;
    Step steps[2];
    bool empty() const { return size == 0 || steps[0].count == 0 || steps[1].count == 0; }
    int64_t end() const { return base + steps[0].bytes * (steps[0].count - 1) + steps[1].bytes * (steps[1].count - 1) + size; }
};

Region region_of(const at::Tensor &t, const Rows &r) {
    const int64_t el = t.element_size();
    return {reinterpret_cast<int64_t>(t.data_ptr()), r.d * el, {{r.row * el, r.tokens}, {r.head * el, r.heads}}};
}

Region pool_of(const nnc_paged_kv &c, const void *pool) {   // as far as pages reach
    const int64_t bytes = (c.type == NNC_E4M3 ? 1 : 2) * (int64_t)c.n_kv_heads * c.page_size * c.head_dim * c.n_pages;
    return {reinterpret_cast<int64_t>(pool), bytes, {{0, 1}, {0, 1}}};
}

struct Term { int64_t bytes, lo, hi; };   // taken lo .. hi times

// whether apart + (a sum of the terms from `at` on) can lie in [lo, hi].  Terms are sorted, longest first, so that each leaves few choices.
bool reaches(int64_t apart, const Term *at, const Term *end, int64_t lo, int64_t hi) {
    if (at == end) return lo <= apart && apart <= hi;
    int64_t least = 0, most = 0;
    for (const Term *t = at + 1; t != end; ++t) { least += t->lo * t->bytes; most += t->hi * t->bytes; }
    auto floor_div = [](int64_t a, int64_t b) { return a / b - (a % b != 0 && a < 0); };
    const int64_t first = std::max(at->lo, -floor_div(apart + most - lo, at->bytes)), last = std::min(at->hi, floor_div(hi - apart - least, at->bytes));
    for (int64_t n = first; n <= last; ++n)
        if (reaches(apart + n * at->bytes, at + 1, end, lo, hi)) return true;
    return false;
}

// A tensor that a call writes to.  Where autograd keeps it for a backward pass, that pass has to see that it changed.
void written(const at::Tensor &t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
void writable(const at::Tensor &t) {
    if (t.requires_grad() && c10::GradMode::is_enabled()) refuse("out: no tensor that requires a gradient");
}

// whether two regions have a byte in common, exactly
bool meet(const Region &a, const Region &b) {
    if (a.empty() || b.empty() || a.end() <= b.base || b.end() <= a.base) return false;
    Term terms[4];
    int n = 0;
    auto add = [&](const Region::Step &s, int64_t lo, int64_t hi) {
        if (s.bytes == 0 || s.count == 1) return;
        for (int i = 0; i < n; ++i)
            if (terms[i].bytes == s.bytes) { terms[i].lo += lo; terms[i].hi += hi; return; }   // the difference of the two alone matters
        terms[n++] = {s.bytes, lo, hi};
    };
    for (const Region::Step &s : a.steps) add(s, 0, s.count - 1);
    for (const Region::Step &s : b.steps) add(s, 1 - s.count, 0);
    std::sort(terms, terms + n, [](const Term &x, const Term &y) { return x.bytes > y.bytes; });
    return reaches(a.base - b.base, terms, terms + n, 1 - a.size, b.size - 1);
}

// out may be `in` itself, and otherwise has nothing in common with it
void apart_or_same(const Region &out, const Region &in, const char *refusal) {
    bool same = out.base == in.base;
    for (int i = 0; i < 2; ++i) same = same && out.steps[i].bytes == in.steps[i].bytes;
    if (!same && meet(out, in)) refuse(refusal);
}

void raise_status(int status, const char *what) {
    PyObject *e = PyObject_CallFunction(error_class, "is", status, what);
    if (e) {
        PyErr_SetObject(error_class, e);
        Py_DECREF(e);
    }
    throw Refused();
}

// the call, on `device` and its current stream
template <typename F> void launch(int device, const char *what, F call) {
    int status = 0;
    {
        std::optional<c10::cuda::CUDAGuard> guard;
        if (c10::cuda::current_device() != device) guard.emplace(static_cast<c10::DeviceIndex>(device));
        void *stream = c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream();
        Py_BEGIN_ALLOW_THREADS
        status = call(stream);
        Py_END_ALLOW_THREADS
    }
    if (status) raise_status(status, what);
}

const nnc_paged_kv &cache_of(PyObject *address) {
    void *p = PyLong_AsVoidPtr(address);
    if (!p) refuse("cache: a PagedKV");
    return *static_cast<const nnc_paged_kv *>(p);
}

bool truth(PyObject *o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Refused();
    return v != 0;
}

float number(PyObject *o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused();
    return static_cast<float>(v);
}

PyObject *pair(const at::Tensor &a, const at::Tensor &b) {
    PyObject *t = PyTuple_New(2);
    if (!t) throw Refused();
    PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(a));
    PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(b));
    return t;
}

// rope(x, positions, freq, interleaved, amplitude, inverse, out or None)
PyObject *rope(PyObject *const *a) {
    const at::Tensor &x = tensor(a[0], "x"), &positions = tensor(a[1], "positions"), &freq = tensor(a[2], "freq");
    if (!x.is_cuda()) refuse("x: a CUDA tensor");
    const int device = static_cast<int>(x.get_device());
    const Rows in = rows_of(x, device, "x");
    if (freq.scalar_type() != at::kDouble || freq.dim() != 1 || !freq.is_contiguous() || !freq.is_cuda() || freq.get_device() != device || freq.size(0) > (1 << 20))
        refuse("freq: contiguous float64 numbers on the call's CUDA device");
    const int32_t *pos = index_of(positions, in.tokens, device, "positions");
    at::Tensor out;
    Rows to{};
    if (a[6] == Py_None) {
        out = at::empty({in.tokens, in.heads, in.d}, x.options());
        to = in;
        to.head = in.d;
        to.row = in.heads * in.d;
    } else {
        out = tensor(a[6], "out");
        to = rows_of(out, device, "out");
        writable(out);
        if (!to.like(in) || !disjoint(out)) refuse("out: x's shape and type, no rows that overlap");
        apart_or_same(region_of(out, to), region_of(x, in), "out: x itself, or memory that x has no part of");
    }
    const bool interleaved = truth(a[3]), inverse = truth(a[5]);
    const float amplitude = number(a[4]);
    launch(device, "nnc_op_rope", [&](void *stream) {
        return call_rope(x.data_ptr(), out.data_ptr(), in.type, (int32_t)in.tokens, (int32_t)in.heads, (int32_t)in.d, in.row, in.head, to.row, to.head, pos,
                         static_cast<const double *>(freq.data_ptr()), (int32_t)(2 * freq.size(0)), interleaved, inverse, amplitude, stream);
    });
    if (a[6] != Py_None) {
        written(out);
        Py_INCREF(a[6]);
        return a[6];
    }
    return THPVariable_Wrap(out);
}

// kv_write(cache, device, k, v, pos, seq or None)
PyObject *kv_write(PyObject *const *a) {
    const nnc_paged_kv &c = cache_of(a[0]);
    const int device = (int)PyLong_AsLong(a[1]);
    const at::Tensor &k = tensor(a[2], "k"), &v = tensor(a[3], "v"), &pos = tensor(a[4], "pos");
    const Rows rk = rows_of(k, device, "k"), rv = rows_of(v, device, "v");
    if (!rv.like(rk) || rv.row != rk.row || rv.head != rk.head || rk.heads != c.n_kv_heads || rk.d != c.head_dim)
        refuse("k, v: [tokens][n_kv_heads][head_dim] of the cache, of one type with the same strides");
    for (const void *pool : {c.k, c.v})
        for (const at::Tensor *t : {&k, &v})
            if (meet(region_of(*t, rk), pool_of(c, pool))) refuse("k, v: memory that the cache has no part of");
    const int32_t *at_pos = index_of(pos, rk.tokens, device, "pos");
    const int32_t *at_seq = a[5] == Py_None ? nullptr : index_of(tensor(a[5], "seq"), rk.tokens, device, "seq");
    launch(device, "nnc_op_kv_write_paged", [&](void *stream) {
        return call_write(&c, k.data_ptr(), v.data_ptr(), rk.type, (int32_t)rk.tokens, rk.row, rk.head, at_pos, at_seq, stream);
    });
    Py_RETURN_NONE;
}

// kv_read(cache, device, pos, seq or None, dtype or None, k or None, v or None)
PyObject *kv_read(PyObject *const *a) {
    const nnc_paged_kv &c = cache_of(a[0]);
    const int device = (int)PyLong_AsLong(a[1]);
    const at::Tensor &pos = tensor(a[2], "pos");
    if (pos.dim() != 1) refuse("pos: contiguous int32 numbers");
    const int64_t tokens = pos.size(0);
    at::ScalarType dtype = c.type == NNC_F16 ? at::kHalf : at::kBFloat16;
    if (a[4] != Py_None) {
        if (!THPDtype_Check(a[4])) refuse("dtype: float32, bfloat16 or float16");
        dtype = reinterpret_cast<THPDtype *>(a[4])->scalar_type;
        if (type_of(dtype) < 0) refuse("dtype: float32, bfloat16 or float16");
    }
    at::Tensor k, v;
    Rows r{};
    if ((a[5] == Py_None) != (a[6] == Py_None)) refuse("out: two tensors, or None");
    if (a[5] == Py_None) {
        const auto options = at::TensorOptions().dtype(dtype).device(at::kCUDA, static_cast<c10::DeviceIndex>(device));
        k = at::empty({tokens, c.n_kv_heads, c.head_dim}, options);
        v = at::empty({tokens, c.n_kv_heads, c.head_dim}, options);
        r = rows_of(k, device, "out");
    } else {
        k = tensor(a[5], "out");
        v = tensor(a[6], "out");
        r = rows_of(k, device, "out");
        writable(k);
        writable(v);
        const Rows rv = rows_of(v, device, "out");
        if (!rv.like(r) || rv.row != r.row || rv.head != r.head || r.tokens != tokens || r.heads != c.n_kv_heads || r.d != c.head_dim ||
            (a[4] != Py_None && r.type != type_of(dtype)) || !disjoint(k) || !disjoint(v))
            refuse("out: two tensors [tokens][n_kv_heads][head_dim] of one type with the same strides, no rows that overlap");
        if (meet(region_of(k, r), region_of(v, r))) refuse("out: two tensors with no memory in common");
        for (const void *pool : {c.k, c.v})
            for (const at::Tensor *t : {&k, &v})
                if (meet(region_of(*t, r), pool_of(c, pool))) refuse("out: memory that the cache has no part of");
    }
    const int32_t *at_pos = index_of(pos, tokens, device, "pos");
    const int32_t *at_seq = a[3] == Py_None ? nullptr : index_of(tensor(a[3], "seq"), tokens, device, "seq");
    launch(device, "nnc_op_kv_read_paged", [&](void *stream) {
        return call_read(&c, k.data_ptr(), v.data_ptr(), r.type, (int32_t)tokens, r.row, r.head, at_pos, at_seq, stream);
    });
    if (a[5] != Py_None) {
        written(k);
        written(v);
    }
    return pair(k, v);
}

// attn(cache, device, q, lens, scale or None, window, scratch or None, out or None, want_lse)
PyObject *attn(PyObject *const *a) {
    const nnc_paged_kv &c = cache_of(a[0]);
    const int device = (int)PyLong_AsLong(a[1]);
    const at::Tensor &q = tensor(a[2], "q"), &lens = tensor(a[3], "lens");
    const Rows in = rows_of(q, device, "q");
    if (in.d != c.head_dim || in.head != in.d) refuse("q: [batch][n_q_heads][head_dim] of the cache's head_dim, heads next to each other");
    const int32_t *at_lens = index_of(lens, in.tokens, device, "lens");
    const float scale = a[4] == Py_None ? static_cast<float>(1.0 / std::sqrt(static_cast<double>(in.d))) : number(a[4]);
    const long long window = PyLong_AsLongLong(a[5]);
    if (window == -1 && PyErr_Occurred()) throw Refused();
    if (window < 0 || window > INT32_MAX) refuse("window: 0 or a number of positions");
    at::Tensor out, lse, scratch;
    Rows to = in;
    to.row = in.heads * in.d;
    if (a[7] == Py_None) {
        out = at::empty({in.tokens, in.heads, in.d}, q.options());
    } else {
        out = tensor(a[7], "out");
        to = rows_of(out, device, "out");
        writable(out);
        if (!to.like(in) || to.head != in.d || !disjoint(out)) refuse("out: q's shape and type, heads next to each other, no rows that overlap");
        apart_or_same(region_of(out, to), region_of(q, in), "out: q itself, or memory that q has no part of");
        for (const void *pool : {c.k, c.v})
            if (meet(region_of(out, to), pool_of(c, pool))) refuse("out: memory that the cache has no part of");
    }
    const bool want_lse = truth(a[8]);
    if (want_lse) lse = at::empty({in.tokens, in.heads}, q.options().dtype(at::kFloat));
    if (a[6] == Py_None) {   // the tickets alone have to be zero
        scratch = at::empty({(int64_t)NNC_ATTN_PAGED_SCRATCH_BYTES}, q.options().dtype(at::kByte));
        scratch.narrow(0, 0, NNC_ATTN_PAGED_TICKET_BYTES).zero_();
    } else {
        scratch = tensor(a[6], "scratch");
        if (!scratch.is_cuda() || scratch.get_device() != device || !scratch.is_contiguous()) refuse("scratch: a contiguous tensor on the call's CUDA device (attn_paged_scratch)");
    }
    launch(device, "nnc_op_attn_decode_paged", [&](void *stream) {
        return call_attn(q.data_ptr(), &c, at_lens, out.data_ptr(), want_lse ? static_cast<float *>(lse.data_ptr()) : nullptr, in.type, (int32_t)in.tokens,
                         (int32_t)in.heads, in.row, to.row, scale, (int32_t)window, scratch.data_ptr(), scratch.nbytes(), stream);
    });
    if (a[7] != Py_None) written(out);
    if (want_lse) return pair(out, lse);
    return THPVariable_Wrap(out);
}

template <PyObject *(*F)(PyObject *const *), int N> PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments, got %zd", N, n);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Refused &) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// bind(addresses of the four entry points, NncError)
PyObject *bind(PyObject *const *a) {
    void *p[4];
    for (int i = 0; i < 4; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) refuse("bind: addresses");
    }
    call_rope = reinterpret_cast<decltype(call_rope)>(p[0]);
    call_write = reinterpret_cast<decltype(call_write)>(p[1]);
    call_read = reinterpret_cast<decltype(call_read)>(p[2]);
    call_attn = reinterpret_cast<decltype(call_attn)>(p[3]);
    Py_XDECREF(error_class);
    Py_INCREF(a[4]);
    error_class = a[4];
    Py_RETURN_NONE;
}

#define NNC_ENTRY(name, n) {#name, (PyCFunction)(void *)entry<name, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {NNC_ENTRY(bind, 5), NNC_ENTRY(rope, 7), NNC_ENTRY(kv_write, 6), NNC_ENTRY(kv_read, 7), NNC_ENTRY(attn, 9), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
