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
decltype(&nnc_op_page_bounds) call_bounds;
decltype(&nnc_op_score_pages) call_score;
decltype(&nnc_op_select_pages) call_select;
decltype(&nnc_op_attn_selected_paged) call_selected;
decltype(&nnc_op_attn_prefix_paged) call_prefix;
decltype(&nnc_attn_prefix_scratch_bytes) prefix_scratch_bytes;
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

// contiguous int32 numbers, one for every element of `shape`
const int32_t *indices_of(const at::Tensor &t, at::IntArrayRef shape, int device, const char *what) {
    if (t.scalar_type() != at::kInt || t.sizes() != shape || !t.is_contiguous() || !t.is_cuda() || t.get_device() != device) {
        PyErr_Format(PyExc_ValueError, "%s on the call's CUDA device", what);
        throw Refused();
    }
    return static_cast<const int32_t *>(t.data_ptr());
}

int32_t whole(PyObject *o, long long least, const char *refusal) {
    const long long n = PyLong_AsLongLong(o);
    if (n == -1 && PyErr_Occurred()) throw Refused();
    if (n < least || n > INT32_MAX) refuse(refusal);
    return static_cast<int32_t>(n);
}

// What the attentions of one token per sequence have in common: queries, scale, results, scratch.
struct Attention {
    const nnc_paged_kv &c;
    int device;
    const at::Tensor &q;
    Rows in, to;
    at::Tensor out, lse, scratch;
    PyObject *given;   // out, or None
    bool want_lse;
    float scale;

    Attention(PyObject *cache, PyObject *index, PyObject *queries, PyObject *scale_or_none, PyObject *out_or_none, PyObject *want)
        : c(cache_of(cache)), device((int)PyLong_AsLong(index)), q(tensor(queries, "q")), in(rows_of(q, device, "q")), to(in), given(out_or_none) {
        if (in.d != c.head_dim || in.head != in.d) refuse("q: [batch][n_q_heads][head_dim] of the cache's head_dim, heads next to each other");
        scale = scale_or_none == Py_None ? static_cast<float>(1.0 / std::sqrt(static_cast<double>(in.d))) : number(scale_or_none);
        to.row = in.heads * in.d;
        if (given == Py_None) {
            out = at::empty({in.tokens, in.heads, in.d}, q.options());
        } else {
            out = tensor(given, "out");
            to = rows_of(out, device, "out");
            writable(out);
            if (!to.like(in) || to.head != in.d || !disjoint(out)) refuse("out: q's shape and type, heads next to each other, no rows that overlap");
            apart_or_same(region_of(out, to), region_of(q, in), "out: q itself, or memory that q has no part of");
            for (const void *pool : {c.k, c.v})
                if (meet(region_of(out, to), pool_of(c, pool))) refuse("out: memory that the cache has no part of");
        }
        want_lse = truth(want);
        if (want_lse) lse = at::empty({in.tokens, in.heads}, q.options().dtype(at::kFloat));
    }

    // scratch of the caller's, or of the call's own, whose first `zeros` bytes have to be zero
    void take_scratch(PyObject *o, int64_t bytes, int64_t zeros, const char *refusal) {
        if (o == Py_None) {
            scratch = at::empty({bytes}, q.options().dtype(at::kByte));
            scratch.narrow(0, 0, zeros).zero_();
        } else {
            scratch = tensor(o, "scratch");
            if (!scratch.is_cuda() || scratch.get_device() != device || !scratch.is_contiguous()) refuse(refusal);
        }
    }
    float *lse_at() const { return want_lse ? static_cast<float *>(lse.data_ptr()) : nullptr; }
    PyObject *result() const {
        if (given != Py_None) written(out);
        return want_lse ? pair(out, lse) : THPVariable_Wrap(out);
    }
};
constexpr const char *kPagedScratch = "scratch: a contiguous tensor on the call's CUDA device (attn_paged_scratch)";

// attn(cache, device, q, lens, scale or None, window, scratch or None, out or None, want_lse)
PyObject *attn(PyObject *const *a) {
    Attention x(a[0], a[1], a[2], a[4], a[7], a[8]);
    const int32_t *at_lens = index_of(tensor(a[3], "lens"), x.in.tokens, x.device, "lens");
    const int32_t window = whole(a[5], 0, "window: 0 or a number of positions");
    x.take_scratch(a[6], NNC_ATTN_PAGED_SCRATCH_BYTES, NNC_ATTN_PAGED_TICKET_BYTES, kPagedScratch);
    launch(x.device, "nnc_op_attn_decode_paged", [&](void *stream) {
        return call_attn(x.q.data_ptr(), &x.c, at_lens, x.out.data_ptr(), x.lse_at(), x.in.type, (int32_t)x.in.tokens, (int32_t)x.in.heads, x.in.row, x.to.row,
                         x.scale, window, x.scratch.data_ptr(), x.scratch.nbytes(), stream);
    });
    return x.result();
}

// attn_selected(cache, device, q, lens, pages, counts, scale or None, scratch or None, out or None, want_lse)
PyObject *attn_selected(PyObject *const *a) {
    Attention x(a[0], a[1], a[2], a[6], a[8], a[9]);
    const int32_t *at_lens = index_of(tensor(a[3], "lens"), x.in.tokens, x.device, "lens");
    const at::Tensor &pages = tensor(a[4], "pages"), &counts = tensor(a[5], "counts");
    const int64_t list_len = pages.dim() == 3 ? pages.size(2) : 0;
    if (list_len < 1 || list_len > INT32_MAX) refuse("pages: contiguous int32 [batch][n_kv_heads][entries]");
    const int32_t *at_pages = indices_of(pages, {x.in.tokens, x.c.n_kv_heads, list_len}, x.device, "pages: contiguous int32 [batch][n_kv_heads][entries]");
    const int32_t *at_counts = indices_of(counts, {x.in.tokens, x.c.n_kv_heads}, x.device, "counts: contiguous int32 [batch][n_kv_heads]");
    x.take_scratch(a[7], NNC_ATTN_PAGED_SCRATCH_BYTES, NNC_ATTN_PAGED_TICKET_BYTES, kPagedScratch);
    launch(x.device, "nnc_op_attn_selected_paged", [&](void *stream) {
        return call_selected(x.q.data_ptr(), &x.c, at_lens, at_pages, at_counts, (int32_t)list_len, x.out.data_ptr(), x.lse_at(), x.in.type, (int32_t)x.in.tokens,
                             (int32_t)x.in.heads, x.in.row, x.to.row, x.scale, x.scratch.data_ptr(), x.scratch.nbytes(), stream);
    });
    return x.result();
}

// attn_prefix(cache, device, q, lens, starts, shared, scale or None, scratch or None, out or None, want_lse)
PyObject *attn_prefix(PyObject *const *a) {
    Attention x(a[0], a[1], a[2], a[6], a[8], a[9]);
    const int32_t *at_lens = index_of(tensor(a[3], "lens"), x.in.tokens, x.device, "lens");
    const at::Tensor &starts = tensor(a[4], "starts"), &shared = tensor(a[5], "shared");
    const int64_t groups = shared.dim() == 1 ? shared.size(0) : -1;
    if (groups < 0 || groups > x.in.tokens || (groups == 0 && x.in.tokens > 0)) refuse("shared: contiguous int32 numbers, one a group, at most one group a sequence");
    const int32_t *at_starts = index_of(starts, groups + 1, x.device, "starts"), *at_shared = index_of(shared, groups, x.device, "shared");
    // (0 bytes for sizes that the call refuses)
    const int64_t bytes = (int64_t)prefix_scratch_bytes((int32_t)x.in.tokens, (int32_t)x.in.heads, (int32_t)x.in.d);
    x.take_scratch(a[7], std::max<int64_t>(bytes, NNC_ATTN_PAGED_TICKET_BYTES), NNC_ATTN_PAGED_TICKET_BYTES,
                   "scratch: a contiguous tensor on the call's CUDA device (attn_prefix_scratch)");
    launch(x.device, "nnc_op_attn_prefix_paged", [&](void *stream) {
        return call_prefix(x.q.data_ptr(), &x.c, at_lens, at_starts, at_shared, (int32_t)groups, x.out.data_ptr(), x.lse_at(), x.in.type, (int32_t)x.in.tokens,
                           (int32_t)x.in.heads, x.in.row, x.to.row, x.scale, x.scratch.data_ptr(), x.scratch.nbytes(), stream);
    });
    return x.result();
}

// a cache's bounds: [n_pages][n_kv_heads][2][head_dim]
const at::Tensor &bounds_of(PyObject *o, const nnc_paged_kv &c, int device) {
    const at::Tensor &t = tensor(o, "bounds");
    const at::ScalarType type = c.type == NNC_F16 ? at::kHalf : at::kBFloat16;
    if (t.scalar_type() != type || t.sizes() != at::IntArrayRef({c.n_pages, c.n_kv_heads, 2, c.head_dim}) || !t.is_contiguous() || !t.is_cuda() || t.get_device() != device)
        refuse("bounds: contiguous [n_pages][n_kv_heads][2][head_dim] of the cache's type (bfloat16 for float8_e4m3fn) on the cache's device (page_bounds)");
    return t;
}

// page_bounds(cache, device, bounds, lens, first or None)
PyObject *page_bounds(PyObject *const *a) {
    const nnc_paged_kv &c = cache_of(a[0]);
    const int device = (int)PyLong_AsLong(a[1]);
    const at::Tensor &bounds = bounds_of(a[2], c, device), &lens = tensor(a[3], "lens");
    writable(bounds);
    const int64_t batch = lens.dim() == 1 ? lens.size(0) : 0;
    if (batch > INT32_MAX) refuse("sizes: 32-bit numbers");
    const int32_t *at_lens = index_of(lens, batch, device, "lens"), *at_first = a[4] == Py_None ? nullptr : index_of(tensor(a[4], "first"), batch, device, "first");
    const Region whole_bounds = {reinterpret_cast<int64_t>(bounds.data_ptr()), (int64_t)bounds.nbytes(), {{0, 1}, {0, 1}}};
    for (const void *pool : {c.k, c.v})
        if (meet(whole_bounds, pool_of(c, pool))) refuse("bounds: memory that the cache has no part of");
    launch(device, "nnc_op_page_bounds", [&](void *stream) { return call_bounds(&c, bounds.data_ptr(), at_lens, at_first, (int32_t)batch, stream); });
    written(bounds);
    Py_INCREF(a[2]);
    return a[2];
}

// score_pages(cache, device, q, bounds, lens)
PyObject *score_pages(PyObject *const *a) {
    const nnc_paged_kv &c = cache_of(a[0]);
    const int device = (int)PyLong_AsLong(a[1]);
    const at::Tensor &q = tensor(a[2], "q"), &bounds = bounds_of(a[3], c, device);
    const Rows in = rows_of(q, device, "q");
    if (in.d != c.head_dim || in.head != in.d) refuse("q: [batch][n_q_heads][head_dim] of the cache's head_dim, heads next to each other");
    const int32_t *at_lens = index_of(tensor(a[4], "lens"), in.tokens, device, "lens");
    at::Tensor scores = at::empty({in.tokens, c.n_kv_heads, c.pages_per_seq}, q.options().dtype(at::kFloat));
    launch(device, "nnc_op_score_pages", [&](void *stream) {
        return call_score(q.data_ptr(), &c, bounds.data_ptr(), at_lens, static_cast<float *>(scores.data_ptr()), in.type, (int32_t)in.tokens, (int32_t)in.heads, in.row, stream);
    });
    return THPVariable_Wrap(scores);
}

// select_pages(scores, lens, page_size, n, first, last)
PyObject *select_pages(PyObject *const *a) {
    const at::Tensor &scores = tensor(a[0], "scores"), &lens = tensor(a[1], "lens");
    if (scores.scalar_type() != at::kFloat || scores.dim() != 3 || !scores.is_contiguous() || !scores.is_cuda()) refuse("scores: contiguous float32 [batch][n_kv_heads][pages] on a CUDA device");
    const int device = static_cast<int>(scores.get_device());
    const int64_t batch = scores.size(0), heads = scores.size(1), columns = scores.size(2);
    if (batch > INT32_MAX || heads > INT32_MAX || columns > INT32_MAX) refuse("sizes: 32-bit numbers");
    const int32_t *at_lens = index_of(lens, batch, device, "lens");
    const int32_t page_size = whole(a[2], 1, "page_size: a cache's"), n = whole(a[3], 1, "n: a number of pages");
    const int32_t first = whole(a[4], 0, "first, last: numbers of pages"), last = whole(a[5], 0, "first, last: numbers of pages");
    at::Tensor pages = at::empty({batch, heads, n}, scores.options().dtype(at::kInt)), counts = at::empty({batch, heads}, scores.options().dtype(at::kInt));
    launch(device, "nnc_op_select_pages", [&](void *stream) {
        return call_select(static_cast<const float *>(scores.data_ptr()), at_lens, static_cast<int32_t *>(pages.data_ptr()), static_cast<int32_t *>(counts.data_ptr()),
                           (int32_t)batch, (int32_t)heads, (int32_t)columns, page_size, n, first, last, stream);
    });
    return pair(pages, counts);
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

// bind(addresses of the entry points, NncError)
PyObject *bind(PyObject *const *a) {
    void *p[10];
    for (int i = 0; i < 10; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) refuse("bind: addresses");
    }
    call_rope = reinterpret_cast<decltype(call_rope)>(p[0]);
    call_write = reinterpret_cast<decltype(call_write)>(p[1]);
    call_read = reinterpret_cast<decltype(call_read)>(p[2]);
    call_attn = reinterpret_cast<decltype(call_attn)>(p[3]);
    call_bounds = reinterpret_cast<decltype(call_bounds)>(p[4]);
    call_score = reinterpret_cast<decltype(call_score)>(p[5]);
    call_select = reinterpret_cast<decltype(call_select)>(p[6]);
    call_selected = reinterpret_cast<decltype(call_selected)>(p[7]);
    call_prefix = reinterpret_cast<decltype(call_prefix)>(p[8]);
    prefix_scratch_bytes = reinterpret_cast<decltype(prefix_scratch_bytes)>(p[9]);
    Py_XDECREF(error_class);
    Py_INCREF(a[10]);
    error_class = a[10];
    Py_RETURN_NONE;
}

#define NNC_ENTRY(name, n) {#name, (PyCFunction)(void *)entry<name, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {NNC_ENTRY(bind, 11), NNC_ENTRY(rope, 7), NNC_ENTRY(kv_write, 6), NNC_ENTRY(kv_read, 7), NNC_ENTRY(attn, 9),
                         NNC_ENTRY(page_bounds, 5), NNC_ENTRY(score_pages, 5), NNC_ENTRY(select_pages, 6), NNC_ENTRY(attn_selected, 10), NNC_ENTRY(attn_prefix, 10), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
