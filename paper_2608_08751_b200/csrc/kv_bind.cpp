// Argument marshalling of the block-cache operators for Python: tensors in, pointers and strides out to the C-ABI
// library.  A decode step makes five calls of a few microseconds of GPU time each; checked and marshalled in Python
// through ctypes a call took 27-39 us of host time, here it takes a few.  No step of the computation runs here.
//
// The module is handed the C functions' addresses once (`init`), so that it serves the regular and the checked
// library alike.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/AutogradState.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdarg>
#include <initializer_list>
#include <optional>

#include "../../include/ivf_b200.h"

namespace {

decltype(&ivf_kv_tables) f_tables = nullptr;
decltype(&ivf_kv_append) f_append = nullptr;
decltype(&ivf_kv_summarize) f_summarize = nullptr;
decltype(&ivf_kv_select) f_select = nullptr;
decltype(&ivf_kv_attend) f_attend = nullptr;
decltype(&ivf_kv_attend_chunk) f_chunk = nullptr;
decltype(&ivf_kv_attend_chunk_workspace) f_chunk_workspace = nullptr;
decltype(&ivf_kv_fork) f_fork = nullptr;
decltype(&ivf_kv_compact) f_compact = nullptr;
decltype(&ivf_kv_pages_workspace) f_pages_workspace = nullptr;
decltype(&ivf_kv_copy) f_copy = nullptr;
decltype(&ivf_last_error) f_last_error = nullptr;
PyObject* g_error = nullptr;  // IvfError

struct Refused {};  // a Python error is set

[[noreturn]] void refuse(PyObject* type, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    PyErr_FormatV(type, fmt, ap);
    va_end(ap);
    throw Refused();
}

void check(int rc) {
    if (rc == IVF_OK) return;
    PyObject* e = PyObject_CallFunction(g_error, "is", rc, f_last_error());
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    throw Refused();
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "%s must be a torch.Tensor, not %s", name, Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}
bool given(PyObject* o) { return o != Py_None; }
int64_t whole(PyObject* o, const char* name) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused();
    (void)name;
    return v;
}
int small(PyObject* o, const char* name) {
    const int64_t v = whole(o, name);
    if (v < INT32_MIN || v > INT32_MAX) refuse(PyExc_ValueError, "%s = %lld is out of range", name, static_cast<long long>(v));
    return static_cast<int>(v);
}
float real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused();
    return static_cast<float>(v);
}

int type16(const at::Tensor& t, const char* name) {
    if (t.scalar_type() == at::kHalf) return IVF_F16;
    if (t.scalar_type() == at::kBFloat16) return IVF_BF16;
    refuse(PyExc_TypeError, "%s must be float16 or bfloat16, got %s", name, c10::toString(t.scalar_type()));
}

// Neither mode of differentiation is dropped without a word.
void no_grad(const at::Tensor& t, const char* name) {
    if (t.requires_grad() && c10::GradMode::is_enabled())
        refuse(PyExc_ValueError, "%s requires grad: the block-cache operators compute no gradients", name);
    if (c10::AutogradState::get_tls_state().get_fw_grad_mode() && t._fw_grad(0).defined())
        refuse(PyExc_ValueError, "%s carries a forward-mode tangent: the block-cache operators compute no gradients", name);
}
// A tensor that the call writes into: whoever saved it for a backward pass finds out.  (Inference tensors count nothing.)
void written(const at::Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// A contiguous CUDA tensor of this type, device and shape.
void* dense(const at::Tensor& t, const char* name, at::ScalarType type, c10::Device dev, std::initializer_list<int64_t> shape) {
    if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous())
        refuse(PyExc_ValueError, "%s must be a contiguous CUDA tensor of %s", name, c10::toString(type));
    if (t.device() != dev) refuse(PyExc_ValueError, "%s is on %s, the other tensors on %s", name, t.device().str().c_str(), dev.str().c_str());
    if (t.sizes() != at::IntArrayRef(shape)) {
        std::string want;
        for (int64_t s : shape) want += (want.empty() ? "" : ", ") + std::to_string(s);
        refuse(PyExc_ValueError, "%s must have the shape [%s]", name, want.c_str());
    }
    no_grad(t, name);
    return t.numel() ? t.data_ptr() : nullptr;
}

// A CUDA tensor whose last axis is contiguous.
void* strided(const at::Tensor& t, const char* name, int dim, at::ScalarType type, c10::Device dev, int64_t* stride = nullptr) {
    if (t.dim() != dim || !t.is_cuda() || t.device() != dev || t.scalar_type() != type || (t.numel() && t.size(dim - 1) > 1 && t.stride(dim - 1) != 1))
        refuse(PyExc_ValueError, "%s must be a %d-D CUDA tensor of %s on %s with a contiguous last axis", name, dim, c10::toString(type),
               dev.str().c_str());
    for (int i = 1; i < dim; ++i)  // the library takes these as 32-bit numbers
        if (t.size(i) > INT32_MAX) refuse(PyExc_ValueError, "%s: axis %d has %lld elements", name, i, static_cast<long long>(t.size(i)));
    if (stride)
        for (int i = 0; i < dim - 1; ++i) stride[i] = t.size(i) > 1 ? t.stride(i) : 0;  // an axis of one element may carry any stride
    no_grad(t, name);
    return t.numel() ? t.data_ptr() : nullptr;
}

void same_shape(const at::Tensor& a, const at::Tensor& b, const char* what) {
    if (a.sizes() != b.sizes()) refuse(PyExc_ValueError, "shape mismatch: %s", what);
}

ivf_kv_cache cache_of(const at::Tensor& k, const at::Tensor* v) {
    ivf_kv_cache c;
    c.dtype = static_cast<ivf_dtype>(type16(k, "k_cache"));
    c.k = strided(k, "k_cache", 4, k.scalar_type(), k.device(), c.k_stride);
    c.v = c.k;
    for (int i = 0; i < 3; ++i) c.v_stride[i] = c.k_stride[i];
    if (v) {
        c.v = strided(*v, "v_cache", 4, k.scalar_type(), k.device(), c.v_stride);
        same_shape(k, *v, "k_cache and v_cache must both be [num_pages, kv_heads, page_size, head_dim]");
    }
    c.num_pages = k.size(0);
    c.n_kv_heads = static_cast<int>(k.size(1));
    c.page_size = static_cast<int>(k.size(2));
    c.head_dim = static_cast<int>(k.size(3));
    return c;
}

struct Table {
    int32_t* p;
    int64_t stride;
    int n, columns;
};
Table table_of(const at::Tensor& t, c10::Device dev) {
    Table r;
    int64_t s;
    r.p = static_cast<int32_t*>(strided(t, "table", 2, at::kInt, dev, &s));
    if (t.size(0) > INT32_MAX) refuse(PyExc_ValueError, "table: at most 2^31 - 1 rows");
    r.n = static_cast<int>(t.size(0));
    r.columns = static_cast<int>(t.size(1));
    r.stride = r.n > 1 ? s : r.columns;
    return r;
}

at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type, c10::Device dev) {
    return at::empty(shape, at::TensorOptions().dtype(type).device(dev));
}
// A contiguous tensor over part of a buffer's storage.
at::Tensor part(const at::Tensor& buf, int64_t byte, int64_t n, at::ScalarType type) {
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(buf.storage()), buf.key_set(), c10::scalarTypeToTypeMeta(type));
    t.unsafeGetTensorImpl()->set_storage_offset(byte / static_cast<int64_t>(c10::elementSize(type)));
    t.unsafeGetTensorImpl()->set_sizes_contiguous({n});
    return t;
}
void* stream_of(c10::Device dev) { return c10::cuda::getCurrentCUDAStream(dev.index()).stream(); }
template <typename T>
T* as(void* p) { return static_cast<T*>(p); }

#define NEEDS(n)                                                                              \
    if (nargs != (n)) {                                                                       \
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", (n), nargs);          \
        return nullptr;                                                                       \
    }
#define BEGIN    \
    HANDLE_TH_ERRORS \
    try {
#define END              \
    }                    \
    catch (const Refused&) { \
        return nullptr;  \
    }                    \
    END_HANDLE_TH_ERRORS

// (cached, fresh, free_pages, table, page_size, max_tokens, max_touched or None, plan or None) -> the plan's eight tensors
PyObject* kv_tables(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    NEEDS(8)
    BEGIN
    const at::Tensor& table = tensor(a[3], "table");
    const c10::Device dev = table.device();
    const Table tb = table_of(table, dev);
    const int64_t n = tb.n;
    const auto* cached = as<int32_t>(dense(tensor(a[0], "cached"), "cached", at::kInt, dev, {n}));
    const auto* fresh_ = as<int32_t>(dense(tensor(a[1], "fresh"), "fresh", at::kInt, dev, {n}));
    const at::Tensor& free_t = tensor(a[2], "free_pages");
    const auto* free_p = as<int32_t>(dense(free_t, "free_pages", at::kInt, dev, {free_t.numel()}));
    if (free_t.numel() > INT32_MAX) refuse(PyExc_ValueError, "free_pages: at most 2^31 - 1 pages");
    const int page = small(a[4], "page_size");
    const int64_t tokens = whole(a[5], "max_tokens");
    if (tokens < 0) refuse(PyExc_ValueError, "max_tokens must not be negative");
    at::Tensor out[8];
    int64_t touched = 0;
    if (given(a[7])) {
        if (!PyTuple_Check(a[7]) || PyTuple_GET_SIZE(a[7]) != 8) refuse(PyExc_TypeError, "plan must be what an earlier call returned");
        for (int i = 0; i < 8; ++i) out[i] = tensor(PyTuple_GET_ITEM(a[7], i), "plan");
        touched = given(a[6]) ? whole(a[6], "max_touched") : out[5].numel();
        dense(out[0], "plan.kv_lens", at::kInt, dev, {n});
        dense(out[1], "plan.token_start", at::kInt, dev, {n + 1});
        dense(out[2], "plan.token_req", at::kInt, dev, {tokens});
        dense(out[3], "plan.token_pos", at::kInt, dev, {tokens});
        dense(out[4], "plan.token_slot", at::kLong, dev, {tokens});
        dense(out[5], "plan.touched_page", at::kInt, dev, {touched});
        dense(out[6], "plan.touched_fill", at::kInt, dev, {touched});
        dense(out[7], "plan.used", at::kInt, dev, {1});
    } else {
        touched = given(a[6]) ? whole(a[6], "max_touched") : tokens / (page > 0 ? page : 1) + 2 * n;
        if (touched < 0) refuse(PyExc_ValueError, "max_touched must not be negative");
        // one allocation: the 8-byte slots first, then the 4-byte arrays
        const int64_t sizes[8] = {n, n + 1, tokens, tokens, tokens, touched, touched, 1};
        const at::Tensor buf = fresh({4 * (2 * n + 1 + 4 * tokens + 2 * touched + 1)}, at::kByte, dev);
        int64_t at_byte = 8 * tokens;
        for (int i = 0; i < 8; ++i) {
            const bool slots = i == 4;
            out[i] = part(buf, slots ? 0 : at_byte, sizes[i], slots ? at::kLong : at::kInt);
            if (!slots) at_byte += 4 * sizes[i];
        }
    }
    const c10::cuda::CUDAGuard guard(dev);
    auto i32 = [&](int i) { return static_cast<int32_t*>(out[i].data_ptr()); };
    check(f_tables(cached, fresh_, static_cast<int>(n), page, free_p, static_cast<int>(free_t.numel()), tb.p, tb.stride, tb.columns, i32(0), i32(1),
                   i32(2), i32(3), static_cast<int64_t*>(out[4].data_ptr()), tokens, i32(5), i32(6), touched, i32(7), stream_of(dev)));
    written(table);
    if (given(a[7])) {
        for (const at::Tensor& t : out) written(t);
        Py_INCREF(a[7]);
        return a[7];
    }
    PyObject* r = PyTuple_New(8);
    for (int i = 0; r && i < 8; ++i) PyTuple_SET_ITEM(r, i, THPVariable_Wrap(out[i]));
    return r;
    END
}

// (q, k, v, k_cache, v_cache, token_pos, token_slot, rotary, interleaved, q_weight, k_weight, eps, q_out) -> q_out
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    NEEDS(13)
    BEGIN
    const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v");
    const at::Tensor &kc = tensor(a[3], "k_cache"), &vc = tensor(a[4], "v_cache");
    const ivf_kv_cache c = cache_of(kc, &vc);
    const c10::Device dev = kc.device();
    const at::ScalarType type = kc.scalar_type();
    int64_t qs[2], ks[2], vs[2], os[2];
    const void* qp = strided(q, "q", 3, type, dev, qs);
    const void* kp = strided(k, "k", 3, type, dev, ks);
    const void* vp = strided(v, "v", 3, type, dev, vs);
    const int64_t n = q.size(0), heads = q.size(1), d = q.size(2);
    if (k.size(0) != n || k.size(1) != c.n_kv_heads || d != c.head_dim || k.size(2) != d)
        refuse(PyExc_ValueError, "shape mismatch between q, k, v and the caches");
    same_shape(k, v, "k and v");
    const auto* pos = as<int32_t>(dense(tensor(a[5], "token_pos"), "token_pos", at::kInt, dev, {n}));
    const auto* slot = as<int64_t>(dense(tensor(a[6], "token_slot"), "token_slot", at::kLong, dev, {n}));
    const float* rotary = nullptr;
    int64_t n_pos = 0, rot = 0;
    if (given(a[7])) {
        const at::Tensor& r = tensor(a[7], "rotary");
        if (r.dim() != 2) refuse(PyExc_ValueError, "rotary must be [n_pos, rot_dim]");
        n_pos = r.size(0), rot = r.size(1);
        rotary = as<float>(dense(r, "rotary", at::kFloat, dev, {n_pos, rot}));
        if (n_pos > INT32_MAX || rot > INT32_MAX) refuse(PyExc_ValueError, "rotary is too large");
    }
    const int pairs = PyObject_IsTrue(a[8]);
    if (pairs < 0) return nullptr;
    const auto* qw = given(a[9]) ? as<float>(dense(tensor(a[9], "q_weight"), "q_weight", at::kFloat, dev, {d})) : nullptr;
    const auto* kw = given(a[10]) ? as<float>(dense(tensor(a[10], "k_weight"), "k_weight", at::kFloat, dev, {d})) : nullptr;
    const float eps = real(a[11]);
    const at::Tensor out = given(a[12]) ? tensor(a[12], "q_out") : fresh({n, heads, d}, type, dev);
    void* op = strided(out, "q_out", 3, type, dev, os);
    same_shape(out, q, "q_out and q");
    const c10::cuda::CUDAGuard guard(dev);
    check(f_append(qp, qs, kp, ks, vp, vs, n, static_cast<int>(heads), &c, pos, slot, rotary, static_cast<int>(n_pos), static_cast<int>(rot), pairs,
                   qw, kw, eps, op, os, stream_of(dev)));
    written(kc);
    written(vc);
    if (given(a[12])) written(out);
    return THPVariable_Wrap(out);
    END
}

// (k_cache, pages, fills, codes, scales)
PyObject* kv_summarize(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    NEEDS(5)
    BEGIN
    const at::Tensor& kc = tensor(a[0], "k_cache");
    const ivf_kv_cache c = cache_of(kc, nullptr);
    const c10::Device dev = kc.device();
    const at::Tensor& pages = tensor(a[1], "pages");
    const int64_t n = pages.numel();
    const auto* pp = as<int32_t>(dense(pages, "pages", at::kInt, dev, {n}));
    const auto* fp = as<int32_t>(dense(tensor(a[2], "fills"), "fills", at::kInt, dev, {n}));
    auto* codes = as<int8_t>(dense(tensor(a[3], "codes"), "codes", at::kChar, dev, {c.num_pages, c.n_kv_heads, c.head_dim}));
    auto* scales = as<float>(dense(tensor(a[4], "scales"), "scales", at::kFloat, dev, {c.num_pages, c.n_kv_heads}));
    const c10::cuda::CUDAGuard guard(dev);
    check(f_summarize(&c, pp, fp, n, codes, scales, stream_of(dev)));
    written(tensor(a[3], "codes"));
    written(tensor(a[4], "scales"));
    Py_RETURN_NONE;
    END
}

// (q, codes, scales, table, token_req, token_pos, page_size, n_select, n_first, n_last, out) -> out
PyObject* kv_select(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    NEEDS(11)
    BEGIN
    const at::Tensor& q = tensor(a[0], "q");
    const int type = type16(q, "q");
    const c10::Device dev = q.device();
    int64_t qs[2];
    const void* qp = strided(q, "q", 3, q.scalar_type(), dev, qs);
    const int64_t n = q.size(0), heads = q.size(1), d = q.size(2);
    const at::Tensor& ct = tensor(a[1], "codes");
    if (ct.dim() != 3 || ct.size(2) != d) refuse(PyExc_ValueError, "codes must be [num_pages, kv_heads, head_dim]");
    const int64_t pages = ct.size(0), kv = ct.size(1);
    const auto* codes = as<int8_t>(dense(ct, "codes", at::kChar, dev, {pages, kv, d}));
    const auto* scales = as<float>(dense(tensor(a[2], "scales"), "scales", at::kFloat, dev, {pages, kv}));
    const Table tb = table_of(tensor(a[3], "table"), dev);
    const auto* req = as<int32_t>(dense(tensor(a[4], "token_req"), "token_req", at::kInt, dev, {n}));
    const auto* pos = as<int32_t>(dense(tensor(a[5], "token_pos"), "token_pos", at::kInt, dev, {n}));
    const int page = small(a[6], "page_size"), take = small(a[7], "n_select"), first = small(a[8], "n_first"), last = small(a[9], "n_last");
    if (take < 1) refuse(PyExc_ValueError, "n_select must be positive");
    const at::Tensor out = given(a[10]) ? tensor(a[10], "out") : fresh({n, kv, take}, at::kInt, dev);
    auto* op = as<int32_t>(dense(out, "out", at::kInt, dev, {n, kv, take}));
    const c10::cuda::CUDAGuard guard(dev);
    check(f_select(qp, qs, static_cast<ivf_dtype>(type), n, static_cast<int>(heads), static_cast<int>(kv), static_cast<int>(d), codes, scales, pages,
                   tb.p, tb.stride, tb.n, tb.columns, page, req, pos, take, first, last, op, stream_of(dev)));
    if (given(a[10])) written(out);
    return THPVariable_Wrap(out);
    END
}

// (q, k_cache, v_cache, table, token_req, token_pos, selected, scale, out, want_lse) -> (out, lse or None)
PyObject* kv_attend(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    NEEDS(10)
    BEGIN
    const at::Tensor &q = tensor(a[0], "q"), &kc = tensor(a[1], "k_cache"), &vc = tensor(a[2], "v_cache");
    const ivf_kv_cache c = cache_of(kc, &vc);
    const c10::Device dev = kc.device();
    int64_t qs[2], os[2];
    const void* qp = strided(q, "q", 3, kc.scalar_type(), dev, qs);
    const int64_t n = q.size(0), heads = q.size(1), d = q.size(2);
    if (d != c.head_dim) refuse(PyExc_ValueError, "head_dim mismatch between q and the caches");
    const Table tb = table_of(tensor(a[3], "table"), dev);
    const auto* req = as<int32_t>(dense(tensor(a[4], "token_req"), "token_req", at::kInt, dev, {n}));
    const auto* pos = as<int32_t>(dense(tensor(a[5], "token_pos"), "token_pos", at::kInt, dev, {n}));
    const at::Tensor& st = tensor(a[6], "selected");
    if (st.dim() != 3) refuse(PyExc_ValueError, "selected must be [n, kv_heads, n_select]");
    const auto* sel = as<int32_t>(dense(st, "selected", at::kInt, dev, {n, c.n_kv_heads, st.size(2)}));
    const float scale = real(a[7]);
    const at::Tensor out = given(a[8]) ? tensor(a[8], "out") : fresh({n, heads, d}, kc.scalar_type(), dev);
    void* op = strided(out, "out", 3, kc.scalar_type(), dev, os);
    same_shape(out, q, "out and q");
    const int want = PyObject_IsTrue(a[9]);
    if (want < 0) return nullptr;
    at::Tensor lse;
    if (want) lse = fresh({n, heads}, at::kFloat, dev);
    const c10::cuda::CUDAGuard guard(dev);
    check(f_attend(qp, qs, n, static_cast<int>(heads), &c, tb.p, tb.stride, tb.n, tb.columns, req, pos, sel,
                   static_cast<int>(std::min<int64_t>(st.size(2), INT32_MAX)), scale, op, os,
                   want && lse.numel() ? lse.data_ptr<float>() : nullptr, stream_of(dev)));
    if (given(a[8])) written(out);
    PyObject* r = PyTuple_New(2);
    if (!r) return nullptr;
    PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(out));
    if (want) PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(lse));
    else {
        Py_INCREF(Py_None);
        PyTuple_SET_ITEM(r, 1, Py_None);
    }
    return r;
    END
}

// Scratch memory of one call: the allocator hands it out again to later work of the same stream only, and a captured graph keeps its own.
at::Tensor scratch(int64_t bytes, c10::Device dev) { return fresh({bytes}, at::kByte, dev); }

// (q, k_cache, v_cache, table, token_start, kv_lens, scale, cap, slopes, window, prefix, out, want_lse) -> (out, lse or None)
PyObject* kv_attend_chunk(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    NEEDS(13)
    BEGIN
    const at::Tensor &q = tensor(a[0], "q"), &kc = tensor(a[1], "k_cache"), &vc = tensor(a[2], "v_cache");
    const ivf_kv_cache c = cache_of(kc, &vc);
    const c10::Device dev = kc.device();
    int64_t qs[2], os[2];
    const void* qp = strided(q, "q", 3, kc.scalar_type(), dev, qs);
    const int64_t n = q.size(0), heads = q.size(1), d = q.size(2);
    if (d != c.head_dim) refuse(PyExc_ValueError, "head_dim mismatch between q and the caches");
    const Table tb = table_of(tensor(a[3], "table"), dev);
    const auto* start = as<int32_t>(dense(tensor(a[4], "token_start"), "token_start", at::kInt, dev, {tb.n + int64_t{1}}));
    const auto* lens = as<int32_t>(dense(tensor(a[5], "kv_lens"), "kv_lens", at::kInt, dev, {tb.n}));
    const float scale = real(a[6]), cap = real(a[7]);
    const auto* slopes = given(a[8]) ? as<float>(dense(tensor(a[8], "slopes"), "slopes", at::kFloat, dev, {heads})) : nullptr;
    const int window = small(a[9], "window");
    const auto* prefix = given(a[10]) ? as<int32_t>(dense(tensor(a[10], "prefix"), "prefix", at::kInt, dev, {tb.n})) : nullptr;
    const at::Tensor out = given(a[11]) ? tensor(a[11], "out") : fresh({n, heads, d}, kc.scalar_type(), dev);
    void* op = strided(out, "out", 3, kc.scalar_type(), dev, os);
    same_shape(out, q, "out and q");
    const int want = PyObject_IsTrue(a[12]);
    if (want < 0) return nullptr;
    const c10::cuda::CUDAGuard guard(dev);
    at::Tensor lse, work;
    if (want) lse = fresh({n, heads}, at::kFloat, dev);
    int64_t bytes = 0;
    check(f_chunk_workspace(n, static_cast<int>(heads), &c, tb.n, &bytes));
    if (bytes) work = scratch(bytes, dev);
    check(f_chunk(qp, qs, n, static_cast<int>(heads), &c, tb.p, tb.stride, tb.n, tb.columns, start, lens, scale, cap, slopes, window, prefix, op, os,
                  want && lse.numel() ? lse.data_ptr<float>() : nullptr, bytes ? work.data_ptr() : nullptr, bytes, stream_of(dev)));
    if (given(a[11])) written(out);
    PyObject* r = PyTuple_New(2);
    if (!r) return nullptr;
    PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(out));
    if (want) PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(lse));
    else {
        Py_INCREF(Py_None);
        PyTuple_SET_ITEM(r, 1, Py_None);
    }
    return r;
    END
}

// (table, kv_lens, parent, keep, num_pages, page_size, fork or None) -> the seven tensors of a fork
PyObject* kv_fork(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    NEEDS(7)
    BEGIN
    const at::Tensor& table = tensor(a[0], "table");
    const c10::Device dev = table.device();
    const Table tb = table_of(table, dev);
    const auto* lens = as<int32_t>(dense(tensor(a[1], "kv_lens"), "kv_lens", at::kInt, dev, {tb.n}));
    const at::Tensor& pt = tensor(a[2], "parent");
    const int64_t n = pt.numel();
    if (n > INT32_MAX) refuse(PyExc_ValueError, "parent: at most 2^31 - 1 rows");
    const auto* parent = as<int32_t>(dense(pt, "parent", at::kInt, dev, {n}));
    const auto* keep = given(a[3]) ? as<int32_t>(dense(tensor(a[3], "keep"), "keep", at::kInt, dev, {n})) : nullptr;
    const int64_t pages = whole(a[4], "num_pages");
    const int page = small(a[5], "page_size");
    if (pages < 0 || pages > INT32_MAX) refuse(PyExc_ValueError, "num_pages = %lld is out of range", static_cast<long long>(pages));
    const c10::cuda::CUDAGuard guard(dev);
    at::Tensor out[7];
    int64_t stride = tb.columns;
    if (given(a[6])) {
        if (!PyTuple_Check(a[6]) || PyTuple_GET_SIZE(a[6]) != 7) refuse(PyExc_TypeError, "fork must be what an earlier call returned");
        for (int i = 0; i < 7; ++i) out[i] = tensor(PyTuple_GET_ITEM(a[6], i), "fork");
        strided(out[0], "fork.table", 2, at::kInt, dev, &stride);
        if (out[0].size(0) != n || out[0].size(1) != tb.columns) refuse(PyExc_ValueError, "fork.table must have a row for each parent and the table's columns");
        if (n <= 1) stride = tb.columns;
        static const char* const names[] = {"", "fork.kv_lens", "fork.copy_from", "fork.copy_to", "fork.copy_fill"};
        for (int i = 1; i < 5; ++i) dense(out[i], names[i], at::kInt, dev, {n});
        dense(out[5], "fork.free_pages", at::kInt, dev, {pages});
        dense(out[6], "fork.n_free", at::kInt, dev, {1});
    } else {
        out[0] = fresh({n, tb.columns}, at::kInt, dev);
        const at::Tensor buf = fresh({4 * (4 * n + pages + 1)}, at::kByte, dev);
        for (int i = 1; i < 5; ++i) out[i] = part(buf, 4 * (i - 1) * n, n, at::kInt);
        out[5] = part(buf, 16 * n, pages, at::kInt);
        out[6] = part(buf, 16 * n + 4 * pages, 1, at::kInt);
    }
    int64_t bytes = 0;
    at::Tensor work;
    check(f_pages_workspace(static_cast<int>(n), tb.columns, pages, &bytes));
    if (bytes) work = scratch(bytes, dev);
    auto i32 = [&](int i) { return out[i].numel() ? static_cast<int32_t*>(out[i].data_ptr()) : nullptr; };
    check(f_fork(tb.p, tb.stride, lens, tb.n, tb.columns, parent, keep, static_cast<int>(n), pages, page, i32(0), stride, i32(1), i32(2), i32(3), i32(4),
                 i32(5), i32(6), bytes ? work.data_ptr() : nullptr, bytes, stream_of(dev)));
    if (given(a[6])) {
        for (const at::Tensor& t : out) written(t);
        Py_INCREF(a[6]);
        return a[6];
    }
    PyObject* r = PyTuple_New(7);
    for (int i = 0; r && i < 7; ++i) PyTuple_SET_ITEM(r, i, THPVariable_Wrap(out[i]));
    return r;
    END
}

// (table, kv_lens, num_pages, page_size, max_moves or None, out or None) -> (table, copy_from, copy_to, n_held)
PyObject* kv_compact(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    NEEDS(6)
    BEGIN
    const at::Tensor& table = tensor(a[0], "table");
    const c10::Device dev = table.device();
    const Table tb = table_of(table, dev);
    const auto* lens = as<int32_t>(dense(tensor(a[1], "kv_lens"), "kv_lens", at::kInt, dev, {tb.n}));
    const int64_t pages = whole(a[2], "num_pages");
    const int page = small(a[3], "page_size");
    if (pages < 0 || pages > INT32_MAX) refuse(PyExc_ValueError, "num_pages = %lld is out of range", static_cast<long long>(pages));
    const int64_t moves = given(a[4]) ? whole(a[4], "max_moves") : pages;
    if (moves < 0 || moves > INT32_MAX) refuse(PyExc_ValueError, "max_moves = %lld is out of range", static_cast<long long>(moves));
    const at::Tensor out = given(a[5]) ? tensor(a[5], "out") : table;
    const Table to = table_of(out, dev);
    if (to.n != tb.n || to.columns != tb.columns) refuse(PyExc_ValueError, "out must have the table's shape");
    const c10::cuda::CUDAGuard guard(dev);
    const at::Tensor buf = fresh({4 * (2 * moves + 1)}, at::kByte, dev);
    const at::Tensor lists[3] = {part(buf, 0, moves, at::kInt), part(buf, 4 * moves, moves, at::kInt), part(buf, 8 * moves, 1, at::kInt)};
    int64_t bytes = 0;
    at::Tensor work;
    check(f_pages_workspace(tb.n, tb.columns, pages, &bytes));
    if (bytes) work = scratch(bytes, dev);
    auto i32 = [&](int i) { return lists[i].numel() ? static_cast<int32_t*>(lists[i].data_ptr()) : nullptr; };
    check(f_compact(tb.p, tb.stride, lens, tb.n, tb.columns, pages, page, to.p, to.stride, i32(0), i32(1), moves, i32(2), bytes ? work.data_ptr() : nullptr,
                    bytes, stream_of(dev)));
    written(out);
    PyObject* r = PyTuple_New(4);
    if (!r) return nullptr;
    PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(out));
    for (int i = 0; i < 3; ++i) PyTuple_SET_ITEM(r, i + 1, THPVariable_Wrap(lists[i]));
    return r;
    END
}

// (k_cache, v_cache, copy_from, copy_to, copy_fill or None, codes or None, scales or None)
PyObject* kv_copy(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    NEEDS(7)
    BEGIN
    const at::Tensor &kc = tensor(a[0], "k_cache"), &vc = tensor(a[1], "v_cache");
    const ivf_kv_cache c = cache_of(kc, &vc);
    const c10::Device dev = kc.device();
    const at::Tensor& from = tensor(a[2], "copy_from");
    const int64_t n = from.numel();
    const auto* fp = as<int32_t>(dense(from, "copy_from", at::kInt, dev, {n}));
    const auto* tp = as<int32_t>(dense(tensor(a[3], "copy_to"), "copy_to", at::kInt, dev, {n}));
    const auto* fill = given(a[4]) ? as<int32_t>(dense(tensor(a[4], "copy_fill"), "copy_fill", at::kInt, dev, {n})) : nullptr;
    if (given(a[5]) != given(a[6])) refuse(PyExc_ValueError, "codes and scales: both or neither");
    int8_t* codes = nullptr;
    float* scales = nullptr;
    if (given(a[5])) {
        codes = as<int8_t>(dense(tensor(a[5], "codes"), "codes", at::kChar, dev, {c.num_pages, c.n_kv_heads, c.head_dim}));
        scales = as<float>(dense(tensor(a[6], "scales"), "scales", at::kFloat, dev, {c.num_pages, c.n_kv_heads}));
    }
    const c10::cuda::CUDAGuard guard(dev);
    check(f_copy(&c, fp, tp, fill, n, codes, scales, stream_of(dev)));
    written(kc);
    written(vc);
    if (given(a[5])) {
        written(tensor(a[5], "codes"));
        written(tensor(a[6], "scales"));
    }
    Py_RETURN_NONE;
    END
}

// (addresses of the library's functions in the order below; the error class)
PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    constexpr int kFunctions = 12;
    NEEDS(kFunctions + 1)
    void* f[kFunctions];
    for (int i = 0; i < kFunctions; ++i) {
        f[i] = PyLong_AsVoidPtr(a[i]);
        if (!f[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null function address");
            return nullptr;
        }
    }
    f_tables = reinterpret_cast<decltype(f_tables)>(f[0]);
    f_append = reinterpret_cast<decltype(f_append)>(f[1]);
    f_summarize = reinterpret_cast<decltype(f_summarize)>(f[2]);
    f_select = reinterpret_cast<decltype(f_select)>(f[3]);
    f_attend = reinterpret_cast<decltype(f_attend)>(f[4]);
    f_chunk = reinterpret_cast<decltype(f_chunk)>(f[5]);
    f_chunk_workspace = reinterpret_cast<decltype(f_chunk_workspace)>(f[6]);
    f_fork = reinterpret_cast<decltype(f_fork)>(f[7]);
    f_compact = reinterpret_cast<decltype(f_compact)>(f[8]);
    f_pages_workspace = reinterpret_cast<decltype(f_pages_workspace)>(f[9]);
    f_copy = reinterpret_cast<decltype(f_copy)>(f[10]);
    f_last_error = reinterpret_cast<decltype(f_last_error)>(f[11]);
    Py_INCREF(a[kFunctions]);
    Py_XSETREF(g_error, a[kFunctions]);
    Py_RETURN_NONE;
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(kv_tables), METHOD(kv_append), METHOD(kv_summarize), METHOD(kv_select), METHOD(kv_attend), METHOD(kv_attend_chunk),
                         METHOD(kv_fork), METHOD(kv_compact), METHOD(kv_copy), METHOD(init),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kv_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kv_bind(void) { return PyModule_Create(&module); }
