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
                           FAST(set_errors), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_decode", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__decode(void) {
    PyObject* m = PyModule_Create(&g_module);
    if (m && PyModule_AddStringConstant(m, "built_for", PROFK_BINDING_FOR) != 0) Py_CLEAR(m);      // (the build looks for it in the file)
    return m;
}
