// CPython binding of the decoding operators' C ABI (profk.h).  A decoding step makes these calls on small tensors, where
// the caller's time is mostly argument handling: through ctypes and Python checks a call took 17-32 us on the host for
// 8 us of device time, through this module 7-10 with the Python call around it.  It checks and marshals arguments and allocates outputs, nothing else;
// refusals are raised as the package's ProfkError.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <array>
#include <cmath>
#include <initializer_list>
#include <stdexcept>
#include <string>
#include <utility>

#include "profk.h"

namespace {

PyObject* g_error = nullptr;      // ProfkError
PyObject* g_no_memory = nullptr;  // torch.OutOfMemoryError

struct Refusal { std::string what; };
[[noreturn]] void refuse(const std::string& what) { throw Refusal{what}; }
void need(bool ok, const char* what) {
    if (!ok) refuse(what);
}
void status(int code, const char* call) {
    if (code != PROFK_OK) refuse(std::string(call) + ": " + profk_strerror(code) + " (" + std::to_string(code) + ")");
}

// Runs `f`, with no C++ exception crossing into the interpreter.
template <typename F>
PyObject* guarded(F&& f) {
    try {
        return f();
    } catch (const Refusal& r) {
        PyErr_SetString(g_error, r.what.c_str());
    } catch (const c10::OutOfMemoryError& e) {
        PyErr_SetString(g_no_memory, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

const at::Tensor& tensor(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) refuse(std::string(what) + " must be a tensor");
    return THPVariable_Unpack(o);
}
const at::Tensor* optional(PyObject* o, const char* what) { return o == Py_None ? nullptr : &tensor(o, what); }
int64_t integer(PyObject* o, const char* what) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        refuse(std::string(what) + " must be an integer");
    }
    return v;
}
double real(PyObject* o, const char* what) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        refuse(std::string(what) + " must be a number");
    }
    return v;
}

at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, c10::Device device) { return at::detail::empty_cuda(sizes, type, device, std::nullopt); }
PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }
PyObject* none() { Py_RETURN_NONE; }
PyObject* pack(std::initializer_list<PyObject*> items) {
    PyObject* t = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    for (PyObject* o : items) PyTuple_SET_ITEM(t, i++, o);
    return t;
}

// Refuses a tensor whose derivative the call would drop: one with a tangent (forward mode), or that requires a gradient in
// grad mode (`logprobs` is differentiable, and calls this module with grad mode off).
void no_derivative(const at::Tensor* t, const char* what) {
    if (!t) return;
    if (t->_fw_grad(0).defined()) refuse(std::string(what) + " carries a tangent: there is no forward-mode derivative");
    if (t->requires_grad() && at::GradMode::is_enabled())
        refuse(std::string(what) + " requires a gradient, which this call does not have: detach it, or call under torch.no_grad()");
}

// Tells autograd that a tensor was written (inference tensors have no version to raise).
void written(const at::Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// Whether consecutive elements of the last dimension lie together.
bool dense_rows(const at::Tensor& t) { return t.size(-1) <= 1 || t.stride(-1) == 1; }

// An optional tensor of one value per row (or per row and alternative).
template <typename P>
P* of_row(const at::Tensor* t, const char* what, at::ScalarType type, at::IntArrayRef shape, c10::Device device) {
    if (!t) return nullptr;
    if (t->scalar_type() != type || t->sizes() != shape || t->device() != device || !t->is_contiguous())
        refuse(std::string(what) + " must be a contiguous " + c10::toString(type) + " tensor with one value per row, on the logits' device");
    return static_cast<P*>(t->data_ptr());
}

// ---- log probabilities -----------------------------------------------------------------------

struct Matrix { int64_t rows, cols, stride; };

// (rows, V) view of (..., V) with dense, evenly spaced rows that do not overlap.
Matrix matrix(const at::Tensor& x) {
    need(x.is_cuda(), "logits must be a CUDA tensor");
    need(x.dim() >= 1 && x.numel() > 0, "logits must have at least one row and one column");
    need(dense_rows(x), "logits must have dense rows that do not overlap");
    const int64_t cols = x.size(-1);
    int64_t rows = 1, stride = cols;
    bool first = true;
    for (int64_t d = x.dim() - 2; d >= 0; --d) {
        if (x.size(d) == 1) continue;
        if (first) {
            stride = x.stride(d);
            first = false;
        } else {
            need(x.stride(d) == stride * rows, "logits: the leading dimensions must be evenly spaced");
        }
        rows *= x.size(d);
    }
    need(stride >= cols, "logits must have dense rows that do not overlap");
    return {rows, cols, stride};
}

int dtype_index(at::ScalarType t) {
    switch (t) {
        case at::kFloat: return 0;
        case at::kBFloat16: return 1;
        case at::kHalf: return 2;
        default: refuse(std::string("unsupported dtype ") + c10::toString(t) + ": float32, bfloat16 and float16 only");
    }
}

// (logits, tokens, k, temperature, entropy) -> (logprob, lse, entropy, top_logprobs, top_tokens, lse_rest)
PyObject* logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        need(n == 5, "logprobs takes five arguments");
        const at::Tensor& x = tensor(a[0], "logits");
        const at::Tensor* tokens = optional(a[1], "tokens");
        const int64_t k = integer(a[2], "k");
        const double temperature = real(a[3], "temperature");
        const bool entropy = a[4] == Py_True;
        no_derivative(&x, "logits");
        const Matrix m = matrix(x);
        const int type = dtype_index(x.scalar_type());
        const c10::Device dev = x.device();
        const at::IntArrayRef lead = x.sizes().slice(0, x.dim() - 1);
        const int64_t* tok = of_row<int64_t>(tokens, "tokens", at::kLong, lead, dev);
        const c10::cuda::CUDAGuard guard(dev);
        const at::Tensor lse = fresh(lead, at::kFloat, dev), rest = fresh(lead, at::kFloat, dev);
        at::Tensor logprob, ent, top_lp, top_tok;
        if (tok) logprob = fresh(lead, at::kFloat, dev);
        if (entropy) ent = fresh(lead, at::kFloat, dev);
        if (k > 0) {
            c10::SmallVector<int64_t, 8> shape(lead.begin(), lead.end());
            shape.push_back(k);
            top_lp = fresh(shape, at::kFloat, dev);
            top_tok = fresh(shape, at::kLong, dev);
        }
        auto f32 = [](const at::Tensor& t) { return t.defined() ? static_cast<float*>(t.data_ptr()) : nullptr; };
        int64_t* tt = top_tok.defined() ? static_cast<int64_t*>(top_tok.data_ptr()) : nullptr;
        void* stream = c10::cuda::getCurrentCUDAStream(dev.index()).stream();
        const void* p = x.data_ptr();
        const int code = type == 0   ? profk_logprobs_f32((const float*)p, m.rows, m.cols, m.stride, tok, k, temperature, stream, f32(logprob), f32(lse), f32(rest), f32(ent), f32(top_lp), tt)
                         : type == 1 ? profk_logprobs_bf16(p, m.rows, m.cols, m.stride, tok, k, temperature, stream, f32(logprob), f32(lse), f32(rest), f32(ent), f32(top_lp), tt)
                                     : profk_logprobs_f16(p, m.rows, m.cols, m.stride, tok, k, temperature, stream, f32(logprob), f32(lse), f32(rest), f32(ent), f32(top_lp), tt);
        status(code, "profk_logprobs");
        auto give = [](const at::Tensor& t) { return t.defined() ? wrap(t) : none(); };
        return pack({give(logprob), wrap(lse), give(ent), give(top_lp), give(top_tok), wrap(rest)});
    });
}

// (logits, lse, lse_rest, tokens, grad_logprob, entropy, grad_entropy, grad_lse, top_tokens, grad_top, temperature) -> gradient
PyObject* logprobs_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        need(n == 11, "logprobs_backward takes eleven arguments");
        const at::Tensor& x = tensor(a[0], "logits");
        const at::Tensor* top = optional(a[8], "top_tokens");
        const at::Tensor* g_top = optional(a[9], "grad_top");
        const double temperature = real(a[10], "temperature");
        no_derivative(&x, "logits");
        for (const auto& [i, what] : {std::pair{1, "lse"}, {2, "lse_rest"}, {4, "grad_logprob"}, {5, "entropy"}, {6, "grad_entropy"}, {7, "grad_lse"}, {9, "grad_top"}})
            no_derivative(optional(a[i], what), what);
        const Matrix m = matrix(x);
        const int type = dtype_index(x.scalar_type());
        const c10::Device dev = x.device();
        const at::IntArrayRef lead = x.sizes().slice(0, x.dim() - 1);
        auto row = [&](int i, const char* what) { return of_row<const float>(optional(a[i], what), what, at::kFloat, lead, dev); };
        const float *lse = row(1, "lse"), *rest = row(2, "lse_rest"), *g_lp = row(4, "grad_logprob"), *ent = row(5, "entropy"),
                    *g_ent = row(6, "grad_entropy"), *g_lse = row(7, "grad_lse");
        const int64_t* tok = of_row<const int64_t>(optional(a[3], "tokens"), "tokens", at::kLong, lead, dev);
        need(!g_top || top, "grad_top needs top_tokens");
        int64_t k = 0;
        const int64_t* top_p = nullptr;
        const float* g_top_p = nullptr;
        if (g_top) {
            need(top->dim() == x.dim(), "top_tokens must be of shape (..., k)");
            k = top->size(-1);
            c10::SmallVector<int64_t, 8> shape(lead.begin(), lead.end());
            shape.push_back(k);
            top_p = of_row<const int64_t>(top, "top_tokens", at::kLong, shape, dev);
            g_top_p = of_row<const float>(g_top, "grad_top", at::kFloat, shape, dev);
            if (k == 0) g_top_p = nullptr;
        }
        const c10::cuda::CUDAGuard guard(dev);
        const at::Tensor grad = fresh(x.sizes(), x.scalar_type(), dev);
        void* stream = c10::cuda::getCurrentCUDAStream(dev.index()).stream();
        const void* p = x.data_ptr();
        void* g = grad.data_ptr();
        const int code = type == 0   ? profk_logprobs_backward_f32((const float*)p, m.rows, m.cols, m.stride, temperature, lse, rest, tok, g_lp, ent, g_ent, g_lse, k, top_p, g_top_p, stream, (float*)g, m.cols)
                         : type == 1 ? profk_logprobs_backward_bf16(p, m.rows, m.cols, m.stride, temperature, lse, rest, tok, g_lp, ent, g_ent, g_lse, k, top_p, g_top_p, stream, g, m.cols)
                                     : profk_logprobs_backward_f16(p, m.rows, m.cols, m.stride, temperature, lse, rest, tok, g_lp, ent, g_ent, g_lse, k, top_p, g_top_p, stream, g, m.cols);
        status(code, "profk_logprobs_backward");
        return wrap(grad);
    });
}

// ---- paged cache -----------------------------------------------------------------------------

const int32_t* ints(const at::Tensor& t, const char* what, int64_t dims, c10::Device device) {
    if (!t.is_cuda() || t.scalar_type() != at::kInt || t.dim() != dims || t.device() != device || (t.numel() > 0 && !dense_rows(t)))
        refuse(std::string(what) + " must be a dense int32 tensor of " + std::to_string(dims) + " dimension(s) on " + device.str());
    return static_cast<const int32_t*>(t.data_ptr());
}
// Checks a page table; returns its row stride.
int64_t table_stride(const at::Tensor& t, c10::Device device) {
    ints(t, "tables", 2, device);
    const int64_t width = t.size(1), stride = t.size(0) > 1 ? t.stride(0) : width;
    need(width >= 1 && stride >= width, "tables must have rows of at least one entry that do not overlap");
    return stride;
}

// A cache (layers, 2, pages, kv_heads, page_size, dim) with dense rows.
profk_pool_t pool_of(const at::Tensor& t) {
    need(t.is_cuda(), "pool must be a CUDA tensor");
    need(t.dim() == 6 && t.size(1) == 2 && t.numel() > 0, "pool must be of shape (layers, 2, pages, kv_heads, page_size, dim)");
    need(dense_rows(t), "pool must have dense rows");
    const int64_t b = (int64_t)t.element_size();
    return profk_pool_t{t.data_ptr(), t.size(0), t.size(3), t.size(4), t.size(5) * b, t.stride(0) * b, t.stride(1) * b, t.stride(2) * b, t.stride(3) * b, t.stride(4) * b};
}

// (pool, tables, lengths, refs, parents, grow, page_size, past_room) -> (tables, lengths, refs, missing); page_size < 0: the pool's
PyObject* pages_fork(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded([&]() -> PyObject* {
        need(n_args == 8, "pages_fork takes eight arguments");
        const at::Tensor* pool = optional(a[0], "pool");
        no_derivative(pool, "pool");
        const at::Tensor &tables = tensor(a[1], "tables"), &lengths = tensor(a[2], "lengths"), &refs = tensor(a[3], "refs"), &parents = tensor(a[4], "parents");
        const int64_t grow = integer(a[5], "grow");
        int64_t page_size = integer(a[6], "page_size");
        need(refs.is_cuda(), "refs must be a CUDA tensor");
        const c10::Device dev = refs.device();
        const int32_t *refs_p = ints(refs, "refs", 1, dev), *lengths_p = ints(lengths, "lengths", 1, dev), *parents_p = ints(parents, "parents", 1, dev);
        const int64_t stride = table_stride(tables, dev), n_old = tables.size(0), width = tables.size(1), n = parents.size(0), pages = refs.size(0);
        need(lengths.size(0) == n_old, "tables and lengths must have the same number of sequences");
        profk_pool_t desc{};
        if (pool) {
            desc = pool_of(*pool);
            need(pool->device() == dev && pool->size(2) == pages && (page_size < 0 || page_size == desc.page_size),
                 "pool must hold as many pages as refs counts, of page_size tokens, on the same device");
            page_size = desc.page_size;
        } else {
            need(page_size >= 0, "without a pool the page_size must be given");
        }
        size_t bytes = 0;
        status(profk_pages_fork_workspace_bytes(n_old, n, pages, page_size, grow, &bytes), "profk_pages_fork");
        const c10::cuda::CUDAGuard guard(dev);
        const at::Tensor ws = fresh({(int64_t)bytes}, at::kByte, dev), new_tables = fresh({n, width}, at::kInt, dev), new_lengths = fresh({n}, at::kInt, dev),
                         new_refs = fresh({pages}, at::kInt, dev), missing = fresh({}, at::kInt, dev);
        void* stream = c10::cuda::getCurrentCUDAStream(dev.index()).stream();
        status(profk_pages_fork_ex(pool ? &desc : nullptr, static_cast<const int32_t*>(tables.data_ptr()), n_old, width, stride, lengths_p, refs_p, pages, parents_p, n,
                                page_size, grow, a[7] == Py_True ? PROFK_FORK_PAST_ROOM : 0, ws.data_ptr(), bytes, stream, static_cast<int32_t*>(new_tables.data_ptr()),
                                static_cast<int32_t*>(new_lengths.data_ptr()), static_cast<int32_t*>(new_refs.data_ptr()),
                                static_cast<int32_t*>(missing.data_ptr())),
               "profk_pages_fork");
        if (pool) written(*pool);
        return pack({wrap(new_tables), wrap(new_lengths), wrap(new_refs), wrap(missing)});
    });
}

// (pool, tables, refs) -> (tables, refs, page_map, live)
PyObject* pages_compact(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded([&]() -> PyObject* {
        need(n_args == 3, "pages_compact takes three arguments");
        const at::Tensor* pool = optional(a[0], "pool");
        no_derivative(pool, "pool");
        const at::Tensor &tables = tensor(a[1], "tables"), &refs = tensor(a[2], "refs");
        need(refs.is_cuda(), "refs must be a CUDA tensor");
        const c10::Device dev = refs.device();
        const int32_t* refs_p = ints(refs, "refs", 1, dev);
        const int64_t stride = table_stride(tables, dev), n = tables.size(0), width = tables.size(1), pages = refs.size(0);
        profk_pool_t desc{};
        if (pool) {
            desc = pool_of(*pool);
            need(pool->device() == dev && pool->size(2) == pages, "pool must hold as many pages as refs counts, on the same device");
        }
        size_t bytes = 0;
        status(profk_pages_compact_workspace_bytes(pages, &bytes), "profk_pages_compact");
        const c10::cuda::CUDAGuard guard(dev);
        const at::Tensor ws = fresh({(int64_t)bytes}, at::kByte, dev), new_tables = fresh({n, width}, at::kInt, dev), new_refs = fresh({pages}, at::kInt, dev),
                         page_map = fresh({pages}, at::kInt, dev), live = fresh({}, at::kInt, dev);
        void* stream = c10::cuda::getCurrentCUDAStream(dev.index()).stream();
        status(profk_pages_compact(pool ? &desc : nullptr, static_cast<const int32_t*>(tables.data_ptr()), n, width, stride, refs_p, pages, ws.data_ptr(), bytes, stream,
                                   static_cast<int32_t*>(new_tables.data_ptr()), static_cast<int32_t*>(new_refs.data_ptr()),
                                   static_cast<int32_t*>(page_map.data_ptr()), static_cast<int32_t*>(live.data_ptr())),
               "profk_pages_compact");
        if (pool) written(*pool);
        return pack({wrap(new_tables), wrap(new_refs), wrap(page_map), wrap(live)});
    });
}

// (pool, src, dst)
PyObject* pages_copy(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded([&]() -> PyObject* {
        need(n_args == 3, "pages_copy takes three arguments");
        const at::Tensor &pool = tensor(a[0], "pool"), &src = tensor(a[1], "src"), &dst = tensor(a[2], "dst");
        no_derivative(&pool, "pool");
        const profk_pool_t desc = pool_of(pool);
        const c10::Device dev = pool.device();
        const int32_t *src_p = ints(src, "src", 1, dev), *dst_p = ints(dst, "dst", 1, dev);
        need(src.size(0) == dst.size(0), "src and dst must have the same length");
        const c10::cuda::CUDAGuard guard(dev);
        status(profk_pages_copy(&desc, pool.size(2), src_p, dst_p, src.size(0), c10::cuda::getCurrentCUDAStream(dev.index()).stream()), "profk_pages_copy");
        written(pool);
        return none();
    });
}

// One layer's keys and values (pages, kv_heads, page_size, dim).
void pages_pair(const at::Tensor& k, const at::Tensor& v) {
    need(k.is_cuda() && v.is_cuda(), "k_pages and v_pages must be CUDA tensors");
    need(k.dim() == 4 && k.sizes() == v.sizes() && k.scalar_type() == v.scalar_type() && k.device() == v.device() && k.numel() > 0,
         "k_pages and v_pages must be alike, of shape (pages, kv_heads, page_size, dim)");
    need(dense_rows(k) && dense_rows(v), "k_pages and v_pages must have dense rows");
}
profk_page_strides_t strides_of(const at::Tensor& t, int64_t unit) { return {t.stride(0) * unit, t.stride(1) * unit, t.stride(2) * unit}; }

// (k_pages, v_pages, tables, lengths, k, v); k, v: (seqs, [tokens,] kv_heads, dim)
PyObject* pages_append(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded([&]() -> PyObject* {
        need(n_args == 6, "pages_append takes six arguments");
        const at::Tensor &kp = tensor(a[0], "k_pages"), &vp = tensor(a[1], "v_pages"), &tables = tensor(a[2], "tables"), &lengths = tensor(a[3], "lengths"),
                         &k = tensor(a[4], "k"), &v = tensor(a[5], "v");
        for (const auto& [t, what] : {std::pair{&kp, "k_pages"}, {&vp, "v_pages"}, {&k, "k"}, {&v, "v"}}) no_derivative(t, what);
        pages_pair(kp, vp);
        const c10::Device dev = kp.device();
        const int64_t stride = table_stride(tables, dev), seqs = tables.size(0), width = tables.size(1), dims = k.dim();
        const int32_t* lengths_p = ints(lengths, "lengths", 1, dev);
        need((dims == 3 || dims == 4) && k.sizes() == v.sizes() && k.size(0) == seqs && k.size(dims - 2) == kp.size(1) && k.size(dims - 1) == kp.size(3) &&
                 lengths.size(0) == seqs,
             "k and v must be of shape (seqs, [tokens,] kv_heads, dim), one sequence per row of the tables");
        need(k.scalar_type() == kp.scalar_type() && v.scalar_type() == kp.scalar_type() && k.device() == dev && v.device() == dev && dense_rows(k) && dense_rows(v),
             "k and v must have the pages' type and device, and dense rows");
        const int64_t b = (int64_t)k.element_size(), tokens = dims == 4 ? k.size(1) : 1;
        const int64_t ks[3] = {k.stride(0) * b, dims == 4 ? k.stride(1) * b : 0, k.stride(dims - 2) * b};
        const int64_t vs[3] = {v.stride(0) * b, dims == 4 ? v.stride(1) * b : 0, v.stride(dims - 2) * b};
        const profk_page_strides_t kps = strides_of(kp, b), vps = strides_of(vp, b);
        const c10::cuda::CUDAGuard guard(dev);
        status(profk_pages_append(k.data_ptr(), v.data_ptr(), ks, vs, kp.data_ptr(), vp.data_ptr(), &kps, &vps, static_cast<const int32_t*>(tables.data_ptr()), stride,
                                  lengths_p, seqs, tokens, kp.size(1), kp.size(3) * b, kp.size(2), kp.size(0), width,
                                  c10::cuda::getCurrentCUDAStream(dev.index()).stream()),
               "profk_pages_append");
        written(kp);
        written(vp);
        return none();
    });
}

// (q, k_pages, v_pages, tables, lengths, scale) -> (out, lse); scale None: dim ** -0.5
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded([&]() -> PyObject* {
        need(n_args == 6, "paged_attention takes six arguments");
        const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k_pages"), &v = tensor(a[2], "v_pages"), &tables = tensor(a[3], "tables"),
                         &lengths = tensor(a[4], "lengths");
        for (const auto& [t, what] : {std::pair{&q, "q"}, {&k, "k_pages"}, {&v, "v_pages"}}) no_derivative(t, what);
        need(q.is_cuda(), "q must be a CUDA tensor");
        pages_pair(k, v);
        need(q.dim() == 3 && q.numel() > 0 && dense_rows(q), "q must be of shape (seqs, heads, dim) with dense rows");
        const c10::Device dev = q.device();
        const int64_t seqs = q.size(0), heads = q.size(1), dim = q.size(2), stride = table_stride(tables, dev);
        const int32_t* lengths_p = ints(lengths, "lengths", 1, dev);
        need(k.scalar_type() == q.scalar_type() && k.device() == dev && k.size(3) == dim && heads % k.size(1) == 0 && tables.size(0) == seqs && lengths.size(0) == seqs,
             "q, pages, tables and lengths do not belong together (type, device, dim, heads or sequences differ)");
        need(q.scalar_type() == at::kBFloat16 || q.scalar_type() == at::kHalf, "unsupported dtype: bfloat16 and float16 only");
        const double scale = a[5] == Py_None ? 1.0 / std::sqrt((double)dim) : real(a[5], "scale");
        const c10::cuda::CUDAGuard guard(dev);
        size_t bytes = 0;
        status(profk_paged_attention_workspace_bytes(dim, &bytes), "profk_paged_attention");
        const at::Tensor ws = fresh({(int64_t)bytes}, at::kByte, dev), out = fresh({seqs, heads, dim}, q.scalar_type(), dev), lse = fresh({seqs, heads}, at::kFloat, dev);
        const profk_page_strides_t ks = strides_of(k, 1), vs = strides_of(v, 1);
        auto* call = q.scalar_type() == at::kHalf ? &profk_paged_attention_f16 : &profk_paged_attention_bf16;
        status(call(q.data_ptr(), q.stride(0), q.stride(1), k.data_ptr(), v.data_ptr(), &ks, &vs, static_cast<const int32_t*>(tables.data_ptr()), stride, lengths_p, seqs,
                    heads, k.size(1), dim, k.size(2), k.size(0), tables.size(1), scale, ws.data_ptr(), bytes,
                    c10::cuda::getCurrentCUDAStream(dev.index()).stream(), out.data_ptr(), static_cast<float*>(lse.data_ptr())),
               "profk_paged_attention");
        return pack({wrap(out), wrap(lse)});
    });
}

// ---- prompts and drafts ----------------------------------------------------------------------

using Strides3 = std::array<int64_t, 3>;

int64_t stride_of(const at::Tensor& t, int64_t d) { return t.size(d) > 1 ? t.stride(d) : 0; }

const double* frequencies_of(const at::Tensor& t, c10::Device device) {
    no_derivative(&t, "frequencies");
    need(t.is_cuda() && t.device() == device && t.scalar_type() == at::kDouble && t.dim() == 1 && t.numel() > 0 && t.is_contiguous(),
         "frequencies must be a contiguous float64 tensor of one dimension on the same device");
    return static_cast<const double*>(t.data_ptr());
}

// (x, positions, frequencies, interleaved, magnitude, inverse) -> turned
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded([&]() -> PyObject* {
        need(n_args == 6, "rotary takes six arguments");
        const at::Tensor &x = tensor(a[0], "x"), &positions = tensor(a[1], "positions"), &frequencies = tensor(a[2], "frequencies");
        no_derivative(&x, "x");
        need(x.is_cuda() && x.dim() >= 2, "x must be a CUDA tensor (..., heads, dim)");
        const int type = dtype_index(x.scalar_type());
        const c10::Device dev = x.device();
        need(x.numel() == 0 || dense_rows(x), "x must have dense heads");
        need(positions.is_cuda() && positions.device() == dev && positions.scalar_type() == at::kLong && positions.dim() <= x.dim() - 2,
             "positions must be an int64 tensor that broadcasts to x's leading dimensions, on the same device");
        const double magnitude = real(a[4], "magnitude");
        profk_rotary_t how{frequencies_of(frequencies, dev), frequencies.numel(), a[3] == Py_True, a[5] == Py_True, magnitude};
        // the leading dimensions as two evenly spaced levels, of x and positions alike
        int64_t sizes[2] = {1, 1}, xs[2] = {0, 0}, ps[2] = {0, 0};
        int level = 2;
        for (int64_t d = x.dim() - 3; d >= 0; --d) {
            const int64_t pd = d - (x.dim() - 2 - positions.dim()), n = x.size(d);
            need(pd < 0 || positions.size(pd) == n || positions.size(pd) == 1, "positions must be an int64 tensor that broadcasts to x's leading dimensions, on the same device");
            if (n == 1) continue;
            const int64_t x_step = x.stride(d), p_step = pd >= 0 && positions.size(pd) > 1 ? positions.stride(pd) : 0;
            if (level < 2 && x_step == xs[level] * sizes[level] && p_step == ps[level] * sizes[level]) {
                sizes[level] *= n;
                continue;
            }
            need(--level >= 0, "x: the leading dimensions must be evenly spaced on two levels at most");
            sizes[level] = n;
            xs[level] = x_step;
            ps[level] = p_step;
        }
        const c10::cuda::CUDAGuard guard(dev);
        const at::Tensor out = fresh(x.sizes(), x.scalar_type(), dev);
        if (x.numel() == 0) return wrap(out);
        const int64_t strides[3] = {xs[0], xs[1], stride_of(x, x.dim() - 2)};
        auto* call = type == 0 ? &profk_rotary_f32 : type == 1 ? &profk_rotary_bf16 : &profk_rotary_f16;
        status(call(x.data_ptr(), sizes[0], sizes[1], x.size(-2), x.size(-1), strides, static_cast<const int64_t*>(positions.data_ptr()), ps, &how,
                    c10::cuda::getCurrentCUDAStream(dev.index()).stream(), out.data_ptr()),
               "profk_rotary");
        return wrap(out);
    });
}

// The rows of new tokens: (seqs, [tokens,] heads, dim), or (rows, heads, dim) where `starts` tells the sequences apart.
struct NewRows {
    int64_t rows;
    const int32_t* starts;
};
NewRows new_rows(const at::Tensor& t, const char* what, const at::Tensor* starts, int64_t seqs, c10::Device device) {
    if (starts) {
        need(t.dim() == 3, "with starts, rows of new tokens must be of shape (rows, heads, dim)");
        const int32_t* p = ints(*starts, "starts", 1, device);
        need(starts->size(0) == seqs + 1, "starts must have one entry more than there are sequences");
        return {t.size(0), p};
    }
    if (!((t.dim() == 3 || t.dim() == 4) && t.size(0) == seqs)) refuse(std::string(what) + " must be of shape (seqs, [tokens,] heads, dim), one sequence per row of the tables");
    if (t.dim() == 3) return {seqs, nullptr};
    return {seqs * t.size(1), nullptr};
}
Strides3 row_strides(const at::Tensor& t, bool ragged) {
    if (ragged) return {0, stride_of(t, 0), stride_of(t, 1)};
    if (t.dim() == 3) return {stride_of(t, 0), 0, stride_of(t, 1)};
    return {stride_of(t, 0), stride_of(t, 1), stride_of(t, 2)};
}

// (k_pages, v_pages, tables, lengths, q, k, v, frequencies, starts, positions, interleaved, magnitude) -> turned q
PyObject* pages_append_rotary(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded([&]() -> PyObject* {
        need(n_args == 12, "pages_append_rotary takes twelve arguments");
        const at::Tensor &kp = tensor(a[0], "k_pages"), &vp = tensor(a[1], "v_pages"), &tables = tensor(a[2], "tables"), &lengths = tensor(a[3], "lengths"),
                         &k = tensor(a[5], "k"), &v = tensor(a[6], "v"), &frequencies = tensor(a[7], "frequencies");
        const at::Tensor *q = optional(a[4], "q"), *starts = optional(a[8], "starts"), *positions = optional(a[9], "positions");
        const double magnitude = real(a[11], "magnitude");
        for (const auto& [t, what] : {std::pair{&kp, "k_pages"}, {&vp, "v_pages"}, {&k, "k"}, {&v, "v"}}) no_derivative(t, what);
        no_derivative(q, "q");
        pages_pair(kp, vp);
        const c10::Device dev = kp.device();
        const int type = dtype_index(kp.scalar_type());
        const int64_t stride = table_stride(tables, dev), seqs = tables.size(0), width = tables.size(1);
        const int32_t* lengths_p = ints(lengths, "lengths", 1, dev);
        need(lengths.size(0) == seqs, "tables and lengths must have the same number of sequences");
        const NewRows rows = new_rows(k, "k", starts, seqs, dev);
        const int64_t d = k.dim();
        need(k.sizes() == v.sizes() && k.size(d - 2) == kp.size(1) && k.size(d - 1) == kp.size(3), "k and v must be alike, with the pages' kv_heads and dim");
        for (const at::Tensor* t : {&k, &v, q}) {
            if (!t) continue;
            need(t->scalar_type() == kp.scalar_type() && t->device() == dev && (t->numel() == 0 || dense_rows(*t)), "q, k and v must have the pages' type and device, and dense heads");
        }
        if (q) need(q->dim() == d && q->sizes().slice(0, d - 2) == k.sizes().slice(0, d - 2) && q->size(d - 1) == k.size(d - 1) && q->size(d - 2) > 0, "q must have the same tokens and dim as k");
        const int64_t* pos_p = nullptr;
        int64_t pos_strides[2] = {0, 0};
        if (positions) {
            need(positions->is_cuda() && positions->device() == dev && positions->scalar_type() == at::kLong && positions->sizes() == k.sizes().slice(0, d - 2),
                 "positions must be an int64 tensor with one value per token, on the pages' device");
            pos_p = static_cast<const int64_t*>(positions->data_ptr());
            pos_strides[0] = starts ? 0 : stride_of(*positions, 0);
            pos_strides[1] = starts ? stride_of(*positions, 0) : d == 4 ? stride_of(*positions, 1) : 0;
        }
        profk_rotary_t how{frequencies_of(frequencies, dev), frequencies.numel(), a[10] == Py_True, 0, magnitude};
        const c10::cuda::CUDAGuard guard(dev);
        at::Tensor out;
        if (q) out = fresh(q->sizes(), q->scalar_type(), dev);
        if (rows.rows > 0) {
            const Strides3 qs = q ? row_strides(*q, starts) : Strides3{}, ks = row_strides(k, starts), vs = row_strides(v, starts);
            const profk_page_strides_t kps = strides_of(kp, 1), vps = strides_of(vp, 1);
            auto* call = type == 0 ? &profk_pages_append_rotary_f32 : type == 1 ? &profk_pages_append_rotary_bf16 : &profk_pages_append_rotary_f16;
            status(call(q ? q->data_ptr() : nullptr, qs.data(), k.data_ptr(), ks.data(), v.data_ptr(), vs.data(), kp.data_ptr(), vp.data_ptr(), &kps, &vps,
                        static_cast<const int32_t*>(tables.data_ptr()), stride, lengths_p, rows.starts, seqs, rows.rows, q ? q->size(d - 2) : 0, kp.size(1), kp.size(3),
                        kp.size(2), kp.size(0), width, pos_p, pos_strides, &how, c10::cuda::getCurrentCUDAStream(dev.index()).stream(),
                        q ? out.data_ptr() : nullptr),
                   "profk_pages_append_rotary");
            written(kp);
            written(vp);
        }
        return q ? wrap(out) : none();
    });
}

// (q, k_pages, v_pages, tables, lengths, starts, scale) -> (out, lse); scale None: dim ** -0.5
PyObject* paged_attention_chunk(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded([&]() -> PyObject* {
        need(n_args == 7, "paged_attention_chunk takes seven arguments");
        const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k_pages"), &v = tensor(a[2], "v_pages"), &tables = tensor(a[3], "tables"),
                         &lengths = tensor(a[4], "lengths");
        const at::Tensor* starts = optional(a[5], "starts");
        for (const auto& [t, what] : {std::pair{&q, "q"}, {&k, "k_pages"}, {&v, "v_pages"}}) no_derivative(t, what);
        need(q.is_cuda(), "q must be a CUDA tensor");
        pages_pair(k, v);
        const c10::Device dev = q.device();
        const int64_t stride = table_stride(tables, dev), seqs = tables.size(0), d = q.dim();
        const int32_t* lengths_p = ints(lengths, "lengths", 1, dev);
        need(lengths.size(0) == seqs, "tables and lengths must have the same number of sequences");
        need(starts ? d == 3 : d == 4, "q must be of shape (seqs, tokens, heads, dim), or with starts (rows, heads, dim)");
        const NewRows rows = new_rows(q, "q", starts, seqs, dev);
        const int64_t heads = q.size(d - 2), dim = q.size(d - 1);
        need(q.numel() == 0 || dense_rows(q), "q must have dense heads");
        need(heads > 0 && k.scalar_type() == q.scalar_type() && k.device() == dev && k.size(3) == dim && heads % k.size(1) == 0,
             "q and pages do not belong together (type, device, dim or heads differ)");
        need(q.scalar_type() == at::kBFloat16 || q.scalar_type() == at::kHalf, "unsupported dtype: bfloat16 and float16 only");
        const double scale = a[6] == Py_None ? 1.0 / std::sqrt((double)dim) : real(a[6], "scale");
        const c10::cuda::CUDAGuard guard(dev);
        const at::Tensor out = fresh(q.sizes(), q.scalar_type(), dev), lse = fresh(q.sizes().slice(0, d - 1), at::kFloat, dev);
        if (rows.rows == 0) return pack({wrap(out), wrap(lse)});
        size_t bytes = 0;
        status(profk_paged_attention_chunk_workspace_bytes(dim, &bytes), "profk_paged_attention_chunk");
        const at::Tensor ws = fresh({(int64_t)bytes}, at::kByte, dev);
        const Strides3 qs = row_strides(q, starts);
        const profk_page_strides_t ks = strides_of(k, 1), vs = strides_of(v, 1);
        auto* call = q.scalar_type() == at::kHalf ? &profk_paged_attention_chunk_f16 : &profk_paged_attention_chunk_bf16;
        status(call(q.data_ptr(), qs.data(), k.data_ptr(), v.data_ptr(), &ks, &vs, static_cast<const int32_t*>(tables.data_ptr()), stride, lengths_p, rows.starts, seqs,
                    rows.rows, heads, k.size(1), dim, k.size(2), k.size(0), tables.size(1), scale, ws.data_ptr(), bytes,
                    c10::cuda::getCurrentCUDAStream(dev.index()).stream(), out.data_ptr(), static_cast<float*>(lse.data_ptr())),
               "profk_paged_attention_chunk");
        return pack({wrap(out), wrap(lse)});
    });
}

// Something of n values per row of logits, or (of one dimension) the same for all rows: its stride between rows; null: not given.
template <typename P>
const P* beside_rows(const at::Tensor* t, const char* what, at::ScalarType type, at::IntArrayRef lead, c10::Device device, int64_t* n, int64_t* stride) {
    if (!t) return nullptr;
    const int64_t d = t->dim();
    bool ok = t->is_cuda() && t->device() == device && t->scalar_type() == type && d >= 1 && (t->numel() == 0 || dense_rows(*t));
    ok = ok && (d == 1 || t->sizes().slice(0, d - 1) == lead);
    if (!ok) refuse(std::string(what) + " must be a " + c10::toString(type) + " tensor with dense rows, one for each row of logits or one for all, on the logits' device");
    *n = t->size(-1);
    *stride = 0;
    int64_t rows = 1;
    bool first = true;
    for (int64_t i = d - 2; i >= 0; --i) {
        if (t->size(i) == 1) continue;
        if (first) *stride = t->stride(i);
        else if (t->stride(i) != *stride * rows) refuse(std::string(what) + ": the leading dimensions must be evenly spaced");
        first = false;
        rows *= t->size(i);
    }
    return static_cast<const P*>(t->data_ptr());
}

// (logits, tokens, lengths, prompts, repetition, frequency, presence, bias_tokens, bias_values, mask, out) -> adjusted
PyObject* adjust_logits(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded([&]() -> PyObject* {
        need(n_args == 11, "adjust_logits takes eleven arguments");
        const at::Tensor& x = tensor(a[0], "logits");
        const at::Tensor *tokens = optional(a[1], "tokens"), *lengths = optional(a[2], "lengths"), *prompts = optional(a[3], "prompts"), *bias_tokens = optional(a[7], "bias_tokens"),
                         *bias_values = optional(a[8], "bias_values"), *mask = optional(a[9], "mask"), *given = optional(a[10], "out");
        no_derivative(&x, "logits");
        no_derivative(bias_values, "bias_values");
        no_derivative(given, "out");
        const int type = dtype_index(x.scalar_type());
        const c10::Device dev = x.device();
        need(x.is_cuda() && x.dim() >= 1, "logits must be a CUDA tensor (..., V)");
        const at::IntArrayRef lead = x.sizes().slice(0, x.dim() - 1);
        profk_adjust_t how{};
        int64_t n = 0, words = 0;
        how.tokens = beside_rows<int64_t>(tokens, "tokens", at::kLong, lead, dev, &how.history, &how.token_stride);
        need(tokens || (!lengths && !prompts), "lengths and prompts need tokens");
        how.lengths = of_row<const int32_t>(lengths, "lengths", at::kInt, lead, dev);
        how.prompts = of_row<const int32_t>(prompts, "prompts", at::kInt, lead, dev);
        auto number = [&](int i, const char* what, const float** rows, double* value) {
            if (!THPVariable_Check(a[i])) {
                *value = real(a[i], what);
                if (!std::isfinite((float)*value)) refuse(std::string(what) + " must be finite");
                return;
            }
            const at::Tensor& t = THPVariable_Unpack(a[i]);
            no_derivative(&t, what);
            *rows = of_row<const float>(&t, what, at::kFloat, lead, dev);
        };
        number(4, "repetition", &how.repetition, &how.repetition_value);
        number(5, "frequency", &how.frequency, &how.frequency_value);
        number(6, "presence", &how.presence, &how.presence_value);
        need(how.repetition || (float)how.repetition_value > 0.0f, "repetition must be positive");
        need((bias_tokens != nullptr) == (bias_values != nullptr), "bias_tokens and bias_values belong together");
        how.bias_tokens = beside_rows<int64_t>(bias_tokens, "bias_tokens", at::kLong, lead, dev, &how.biases, &how.bias_token_stride);
        how.bias_values = beside_rows<float>(bias_values, "bias_values", at::kFloat, lead, dev, &n, &how.bias_value_stride);
        need(n == how.biases, "bias_tokens and bias_values must have the same length");
        how.mask = beside_rows<uint32_t>(mask, "mask", at::kInt, lead, dev, &words, &how.mask_stride);
        if (mask) need(words == (x.size(-1) + 31) / 32, "mask must have ceil(V / 32) words");
        if (given) need(given->is_cuda() && given->device() == dev && given->scalar_type() == x.scalar_type() && given->sizes() == x.sizes(), "out must be like logits");
        const c10::cuda::CUDAGuard guard(dev);
        const at::Tensor out = given ? *given : fresh(x.sizes(), x.scalar_type(), dev);
        if (x.numel() == 0) return wrap(out);
        const Matrix m = matrix(x), o = given ? matrix(*given) : Matrix{m.rows, m.cols, m.cols};
        if (given && out.data_ptr() != x.data_ptr()) {
            const int64_t b = (int64_t)x.element_size();
            const char *x0 = static_cast<const char*>(x.data_ptr()), *o0 = static_cast<const char*>(out.data_ptr());
            need(x0 + ((m.rows - 1) * m.stride + m.cols) * b <= o0 || o0 + ((o.rows - 1) * o.stride + o.cols) * b <= x0, "out must be logits itself or not overlap it");
        }
        auto* call = type == 0 ? &profk_adjust_logits_f32 : type == 1 ? &profk_adjust_logits_bf16 : &profk_adjust_logits_f16;
        status(call(x.data_ptr(), m.rows, m.cols, m.stride, &how, c10::cuda::getCurrentCUDAStream(dev.index()).stream(), out.data_ptr(), o.stride), "profk_adjust_logits");
        if (given) written(out);
        return wrap(out);
    });
}

// (ProfkError, torch.OutOfMemoryError): the exceptions to raise
PyObject* set_errors(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 2) throw std::invalid_argument("set_errors takes two arguments");
        Py_INCREF(a[0]);
        Py_XSETREF(g_error, a[0]);
        Py_INCREF(a[1]);
        Py_XSETREF(g_no_memory, a[1]);
        return none();
    });
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {FAST(logprobs), FAST(logprobs_backward), FAST(pages_fork), FAST(pages_compact), FAST(pages_copy), FAST(pages_append), FAST(paged_attention),
                           FAST(rotary), FAST(pages_append_rotary), FAST(paged_attention_chunk), FAST(adjust_logits), FAST(set_errors), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_decode", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__decode(void) {
    PyObject* m = PyModule_Create(&g_module);
    if (m && PyModule_AddStringConstant(m, "built_for", PROFK_BINDING_FOR) != 0) Py_CLEAR(m);      // (the build looks for it in the file)
    return m;
}
