// Python side of the page operators: checks of the tensors, allocation of the results, the call.  A Python-level check of
// twenty arguments takes longer than a small kernel runs; here all of it takes about as long as the launch.  The library's
// entry points are handed over as addresses (bind), so that this module works with whichever copy of the library
// binding.py has loaded.  Every function returns its result, or the xsv_status as an int where the library refused the call.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/core/grad_mode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <initializer_list>
#include <stdexcept>
#include <string>
#include <vector>

#include "../../include/xsv.h"

namespace {

decltype(&xsv_qk_norm_rope) f_norm;
decltype(&xsv_page_plan) f_plan;
decltype(&xsv_page_append) f_append;
decltype(&xsv_page_read) f_read;
decltype(&xsv_page_attention_planned) f_attention;
decltype(&xsv_page_attention_workspace) f_workspace;

[[noreturn]] void refuse(const std::string& what) { throw std::invalid_argument("xsv: " + what); }

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) refuse(std::string(name) + " must be a tensor");
    return THPVariable_Unpack(o);
}
const at::Tensor* maybe(PyObject* o, const char* name) { return o == Py_None ? nullptr : &tensor(o, name); }
std::string seen(const at::Tensor& t) {
    std::string s = std::string(c10::toString(t.scalar_type())) + " [";
    for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
    return s + "] on " + t.device().str();
}
// The address of a contiguous tensor of this type, device and shape (-1: any size).
void* flat(const at::Tensor& t, const char* name, at::ScalarType type, c10::Device dev, std::initializer_list<int64_t> shape) {
    bool ok = t.scalar_type() == type && t.device() == dev && t.is_contiguous() && t.dim() == (int64_t)shape.size();
    int64_t i = 0;
    for (int64_t n : shape) { ok = ok && (n < 0 || t.size(i) == n); ++i; }
    if (!ok) {
        std::string want;
        for (int64_t n : shape) want += (want.empty() ? "" : ", ") + (n < 0 ? std::string("any") : std::to_string(n));
        refuse(std::string(name) + " must be a contiguous " + c10::toString(type) + " tensor of shape [" + want + "] on " + dev.str() + ", not " + seen(t));
    }
    return t.data_ptr();
}
int* ints(const at::Tensor& t, const char* name, c10::Device dev, std::initializer_list<int64_t> shape) {
    return static_cast<int*>(flat(t, name, at::kInt, dev, shape));
}
// Rows [tokens, heads, head_dim] whose heads are contiguous, at any stride.
struct Rows { void* p = nullptr; int64_t stride = 0; };
Rows rows(const at::Tensor& t, const char* name, at::ScalarType type, c10::Device dev, int64_t n, int64_t h, int64_t d) {
    if (t.scalar_type() != type || t.device() != dev || t.dim() != 3 || t.size(0) != n || t.size(1) != h || t.size(2) != d)
        refuse(std::string(name) + " must be a " + c10::toString(type) + " tensor [" + std::to_string(n) + ", " + std::to_string(h) + ", " + std::to_string(d) + "] on " +
               dev.str() + ", not " + seen(t));
    if (n > 0 && ((d > 1 && t.stride(2) != 1) || (h > 1 && t.stride(1) != d))) refuse(std::string(name) + " needs contiguous heads and channels");
    return {t.data_ptr(), n > 1 ? t.stride(0) : h * d};
}
xsv_dtype dtype_of(const at::Tensor& t) {
    if (t.scalar_type() == at::kHalf) return XSV_F16;
    if (t.scalar_type() == at::kBFloat16) return XSV_BF16;
    refuse(std::string("unsupported dtype ") + c10::toString(t.scalar_type()));
}
int int_of(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); refuse("an integer argument is needed"); }
    if (v > INT32_MAX || v < INT32_MIN) refuse("an integer argument is out of range");
    return (int)v;
}
float float_of(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); refuse("a number is needed"); }
    return (float)v;
}
// The tensors' device made current, and its current stream.
struct Here {
    c10::Device dev;
    c10::cuda::OptionalCUDAGuard guard;
    void* stream;
    explicit Here(const at::Tensor& t) : dev(t.device()) {
        if (!t.is_cuda()) refuse("CUDA tensors are needed");
        guard.set_device(dev);
        stream = c10::cuda::getCurrentCUDAStream(dev.index()).stream();
    }
};
int small(int64_t n) {
    if (n > INT32_MAX) refuse("a size is out of range");
    return (int)n;
}
at::Tensor empty(const at::Tensor& like, at::IntArrayRef shape) { return at::empty(shape, like.options().requires_grad(false).memory_format(c10::MemoryFormat::Contiguous)); }

// Elements [off, off + n) of a list, over the same storage (integers: nothing for autograd to know).
at::Tensor part_of(const at::Tensor& t, int64_t off, int64_t n) {
    at::Tensor part = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(t.storage()), t.key_set(), t.dtype());
    part.unsafeGetTensorImpl()->set_storage_offset(off);
    part.unsafeGetTensorImpl()->set_sizes_contiguous({n});
    return part;
}

xsv_page_pool pool_of(const at::Tensor& pages, const at::Tensor& tail) {
    if (pages.dim() != 3 || tail.dim() != 5) refuse("pages are [pages, kv_heads, 72 * head_dim], k_tail is [sequences, 2, kv_heads, 64, head_dim]");
    const int64_t n = pages.size(0), h = pages.size(1), seqs = tail.size(0), d = tail.size(4);
    xsv_page_pool p;
    p.dtype = dtype_of(tail);
    p.records = flat(pages, "pages", at::kByte, pages.device(), {n, h, 72 * d});
    p.k_tail = flat(tail, "k_tail", tail.scalar_type(), pages.device(), {seqs, 2, h, XSV_PAGE_TOKENS, d});
    p.n_pages = n;
    p.max_seqs = small(seqs);
    p.kv_heads = small(h);
    p.head_dim = (int)d;
    return p;
}

// There is no backward: results of inputs that need a gradient say so when one is asked for, instead of passing for constants.
void no_backward(const char* call, std::initializer_list<const at::Tensor*> from, std::initializer_list<at::Tensor> to) {
    if (!at::GradMode::is_enabled()) return;
    std::vector<at::Tensor> need;
    for (const at::Tensor* t : from)
        if (t && t->requires_grad()) need.push_back(*t);
    if (need.empty()) return;
    const std::shared_ptr<torch::autograd::Node> node(new torch::autograd::NotImplemented(call, torch::autograd::collect_next_edges(need)), torch::autograd::deleteNode);
    for (const at::Tensor& t : to)
        if (t.defined()) torch::autograd::set_history(t, node);
}

PyObject* wrap(std::initializer_list<at::Tensor> ts) {
    PyObject* tuple = PyTuple_New((Py_ssize_t)ts.size());
    Py_ssize_t i = 0;
    for (const at::Tensor& t : ts) PyTuple_SET_ITEM(tuple, i++, THPVariable_Wrap(t));
    return tuple;
}
PyObject* status(xsv_status s) { return PyLong_FromLong((long)s); }

// ------------------------------------------------------------------ the calls
PyObject* norm_rope(PyObject* const* a) {
    const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k");
    const at::Tensor* v = maybe(a[2], "v");
    if (q.dim() != 3 || k.dim() != 3) refuse("q and k are [tokens, heads, head_dim]");
    Here here(q);
    const at::ScalarType type = q.scalar_type();
    const int64_t n = q.size(0), hq = q.size(1), hk = k.size(1), d = q.size(2);
    const xsv_dtype dt = dtype_of(q);
    const Rows rq = rows(q, "q", type, here.dev, n, hq, d), rk = rows(k, "k", type, here.dev, n, hk, d);
    const Rows rv = v ? rows(*v, "v", type, here.dev, n, hk, d) : Rows{};
    const int norm = int_of(a[3]), rope = int_of(a[9]);
    void* w[4];
    for (int i = 0; i < 4; ++i) {
        const at::Tensor* t = maybe(a[4 + i], "a weight");
        w[i] = t ? flat(*t, "a weight", type, here.dev, {d}) : nullptr;
    }
    int rotary = 0;
    const float* freq = nullptr;
    const int* pos = nullptr;
    if (rope != XSV_ROPE_NONE) {
        const at::Tensor *f = maybe(a[10], "inv_freq"), *p = maybe(a[11], "positions");
        if (!f || !p) refuse("rope needs inv_freq and positions");
        const int64_t nf = rope == XSV_ROPE_2D ? d / 4 : f->dim() == 1 ? f->size(0) : -1;
        rotary = (int)(rope == XSV_ROPE_2D ? d : 2 * nf);
        freq = static_cast<const float*>(flat(*f, "inv_freq", at::kFloat, here.dev, {nf}));
        pos = rope == XSV_ROPE_2D ? ints(*p, "positions", here.dev, {n, 2}) : ints(*p, "positions", here.dev, {n});
    }
    const int truth = PyObject_IsTrue(a[12]);
    if (truth < 0) { PyErr_Clear(); refuse("head_major must be true or false"); }
    const bool head_major = truth == 1;
    const at::Tensor qo = head_major ? empty(q, {hq, n, d}) : empty(q, {n, hq, d}), ko = head_major ? empty(q, {hk, n, d}) : empty(q, {n, hk, d});
    const at::Tensor vo = v ? empty(ko, ko.sizes()) : at::Tensor();
    const xsv_status s = f_norm(rq.p, rk.p, rv.p, rq.stride, rk.stride, rv.stride, small(n), small(hq), small(hk), (int)d, dt, (xsv_norm)norm, w[0], w[1], w[2], w[3],
                                float_of(a[8]), (xsv_rope)rope, rotary, freq, pos, head_major ? XSV_HEAD_MAJOR : XSV_TOKEN_MAJOR, qo.data_ptr(), ko.data_ptr(),
                                v ? vo.data_ptr() : nullptr, here.stream);
    if (s != XSV_OK) return status(s);
    no_backward("qk_norm_rope", {&q, &k, v, maybe(a[4], ""), maybe(a[5], ""), maybe(a[6], ""), maybe(a[7], "")}, {qo, ko, vo});
    return v ? wrap({qo, ko, vo}) : wrap({qo, ko});
}

PyObject* plan(PyObject* const* a) {
    const at::Tensor &cached = tensor(a[0], "cached_len"), &fresh = tensor(a[1], "new_len"), &table = tensor(a[2], "block_table"),
                     &ring = tensor(a[3], "free_ring"), &state = tensor(a[4], "ring_state");
    Here here(cached);
    const int most = int_of(a[5]);
    const int64_t n = cached.dim() == 1 ? cached.size(0) : -1;
    int *pc = ints(cached, "cached_len", here.dev, {n}), *pf = ints(fresh, "new_len", here.dev, {n}), *pt = ints(table, "block_table", here.dev, {n, -1}),
        *pr = ints(ring, "free_ring", here.dev, {-1}), *ps = ints(state, "ring_state", here.dev, {-1});
    if (state.size(0) < 2 || most < 0) refuse("ring_state holds head and count; max_tokens is not negative");
    const int64_t sizes[6] = {4, n + 1, n, most, most, most};
    const at::Tensor one = empty(cached, {4 + 2 * n + 1 + 3 * (int64_t)most});      // one allocation for all outputs
    int* at0 = one.data_ptr<int>();
    at::Tensor out[6];
    int* p[6];
    int64_t off = 0;
    for (int i = 0; i < 6; ++i) {
        out[i] = part_of(one, off, sizes[i]);
        p[i] = at0 + off;
        off += sizes[i];
    }
    const xsv_status s = f_plan(pc, pf, small(n), pt, small(table.size(1)), pr, small(ring.size(0)), ps, p[0], p[1], p[2], p[3], p[4], p[5], most, here.stream);
    if (s != XSV_OK) return status(s);
    return wrap({out[1], out[2], out[3], out[4], out[5], out[0]});
}

PyObject* append(PyObject* const* a) {
    const at::Tensor &pages = tensor(a[0], "pages"), &tail = tensor(a[1], "k_tail"), &K = tensor(a[2], "K"), &V = tensor(a[3], "V"), &slot = tensor(a[4], "slot_map"),
                     &seq = tensor(a[5], "token_seq"), &cu = tensor(a[6], "cu_new"), &total = tensor(a[7], "total_len");
    Here here(pages);
    const xsv_page_pool pool = pool_of(pages, tail);
    if (K.dim() != 3 || total.dim() != 1) refuse("K is [tokens, kv_heads, head_dim], total_len a list");
    const int64_t n = K.size(0), seqs = total.size(0);
    const Rows rk = rows(K, "K", tail.scalar_type(), here.dev, n, pool.kv_heads, pool.head_dim), rv = rows(V, "V", tail.scalar_type(), here.dev, n, pool.kv_heads, pool.head_dim);
    const int *psl = ints(slot, "slot_map", here.dev, {-1}), *pse = ints(seq, "token_seq", here.dev, {-1});
    if (slot.size(0) < n || seq.size(0) < n) refuse("the plan lists fewer tokens than K and V hold");
    return status(f_append(&pool, rk.p, rv.p, rk.stride, rv.stride, small(n), psl, pse, ints(cu, "cu_new", here.dev, {seqs + 1}), ints(total, "total_len", here.dev, {seqs}),
                           small(seqs), here.stream));
}

PyObject* read(PyObject* const* a) {
    const at::Tensor &pages = tensor(a[0], "pages"), &tail = tensor(a[1], "k_tail"), &table = tensor(a[2], "block_table"), &total = tensor(a[3], "total_len"),
                     &seq = tensor(a[4], "token_seq"), &pos = tensor(a[5], "positions");
    Here here(pages);
    const xsv_page_pool pool = pool_of(pages, tail);
    if (total.dim() != 1 || seq.dim() != 1) refuse("total_len and token_seq are lists");
    const int64_t n = seq.size(0), seqs = total.size(0);
    const int *pt = ints(table, "block_table", here.dev, {seqs, -1}), *pl = ints(total, "total_len", here.dev, {seqs}), *ps = ints(seq, "token_seq", here.dev, {n}),
              *pp = ints(pos, "positions", here.dev, {n});
    const at::Tensor K = empty(tail, {n, pool.kv_heads, pool.head_dim}), V = empty(tail, {n, pool.kv_heads, pool.head_dim});
    const xsv_status s = f_read(&pool, pt, small(table.size(1)), pl, small(seqs), ps, pp, small(n), K.data_ptr(), V.data_ptr(), here.stream);
    return s != XSV_OK ? status(s) : wrap({K, V});
}

PyObject* attention(PyObject* const* a) {
    const at::Tensor &Q = tensor(a[0], "Q"), &pages = tensor(a[1], "pages"), &tail = tensor(a[2], "k_tail"), &table = tensor(a[3], "block_table"), &cu = tensor(a[4], "cu_new"),
                     &total = tensor(a[5], "total_len");
    const at::Tensor *out = maybe(a[9], "out"), *slot = maybe(a[10], "slot_map");
    Here here(pages);
    const xsv_page_pool pool = pool_of(pages, tail);
    if (Q.dim() != 3 || total.dim() != 1) refuse("Q is [tokens, heads, head_dim], total_len a list");
    const int64_t n = Q.size(0), heads = Q.size(1), seqs = total.size(0);
    const int max_new = int_of(a[6]), window = int_of(a[8]);
    const float scale = a[7] == Py_None ? 1.f / std::sqrt((float)pool.head_dim) : float_of(a[7]);
    const Rows rq = rows(Q, "Q", tail.scalar_type(), here.dev, n, heads, pool.head_dim);
    const int *pt = ints(table, "block_table", here.dev, {seqs, -1}), *pc = ints(cu, "cu_new", here.dev, {seqs + 1}), *pl = ints(total, "total_len", here.dev, {seqs});
    const int* ps = slot ? ints(*slot, "slot_map", here.dev, {-1}) : nullptr;
    if (slot && slot->size(0) < n) refuse("slot_map lists fewer tokens than Q holds");
    const at::Tensor to = out ? *out : empty(Q, Q.sizes());
    void* po = flat(to, "out", Q.scalar_type(), here.dev, {n, heads, pool.head_dim});
    const size_t need = f_workspace(small(n), small(seqs), max_new, small(heads), pool.kv_heads, pool.head_dim);
    const at::Tensor space = empty(pages, {(int64_t)need});
    const xsv_status s = f_attention(&pool, rq.p, rq.stride, small(n), small(heads), pt, small(table.size(1)), pc, pl, ps, small(seqs), max_new, scale, window, po, space.data_ptr(), need, here.stream);
    if (s != XSV_OK) return status(s);
    if (out) { Py_INCREF(a[9]); return a[9]; }
    no_backward("page_attention", {&Q}, {to});
    return THPVariable_Wrap(to);
}

template <PyObject* (*F)(PyObject* const*), int N> PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments are needed, not %zd", N, n);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const std::invalid_argument& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const c10::OutOfMemoryError& e) {
        PyErr_SetString(PyExc_MemoryError, e.what_without_backtrace());
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    void* p[6];
    if (n != 6) { PyErr_SetString(PyExc_TypeError, "six addresses are needed"); return nullptr; }
    for (int i = 0; i < 6; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    f_norm = (decltype(f_norm))p[0];
    f_plan = (decltype(f_plan))p[1];
    f_append = (decltype(f_append))p[2];
    f_read = (decltype(f_read))p[3];
    f_attention = (decltype(f_attention))p[4];
    f_workspace = (decltype(f_workspace))p[5];
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
                         {"norm_rope", (PyCFunction)(void (*)(void))entry<norm_rope, 13>, METH_FASTCALL, nullptr},
                         {"plan", (PyCFunction)(void (*)(void))entry<plan, 6>, METH_FASTCALL, nullptr},
                         {"append", (PyCFunction)(void (*)(void))entry<append, 8>, METH_FASTCALL, nullptr},
                         {"read", (PyCFunction)(void (*)(void))entry<read, 6>, METH_FASTCALL, nullptr},
                         {"attention", (PyCFunction)(void (*)(void))entry<attention, 11>, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "xsv_pages", "Argument checks and calls of the page operators; used by binding.py.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit_xsv_pages() { return PyModule_Create(&module); }
