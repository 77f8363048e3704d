// Argument checks that the block-cache entry points share, before any CUDA call.  Included once by each translation unit
// with such entry points, behind its `fail` (which sets the calling thread's error text and returns the code).
#pragma once

namespace {

inline bool kv_page_ok(int page_size) { return page_size == 16 || page_size == 32 || page_size == 64 || page_size == 128; }
inline int kv_shift(int page_size) { return page_size == 16 ? 4 : page_size == 32 ? 5 : page_size == 64 ? 6 : 7; }
inline bool kv_misaligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

int kv_check_page(int page_size) {
    if (!kv_page_ok(page_size)) return fail(IVF_ERR_UNSUPPORTED, "page_size = %d: must be 16, 32, 64 or 128", page_size);
    return IVF_OK;
}
int kv_check_dim(int dim) {
    if (dim < 16 || dim > kKvMaxDim || dim % 16 != 0)
        return fail(IVF_ERR_UNSUPPORTED, "head_dim = %d: must be a multiple of 16 in [16, %d]", dim, kKvMaxDim);
    return IVF_OK;
}
int kv_check_heads(int n_heads, int n_kv_heads) {
    if (n_kv_heads < 1 || n_heads < n_kv_heads || n_heads % n_kv_heads != 0)
        return fail(IVF_ERR_INVALID_ARG, "%d query heads, %d kv heads: the second must divide the first", n_heads, n_kv_heads);
    if (n_heads / n_kv_heads > kKvMaxGroup || n_kv_heads > 1024)
        return fail(IVF_ERR_UNSUPPORTED, "%d query heads, %d kv heads: at most %d to a group and 1024 groups", n_heads, n_kv_heads, kKvMaxGroup);
    return IVF_OK;
}
int kv_check_rows(const char* what, const void* p, const int64_t* stride, int n) {
    if (!p || !stride) return fail(IVF_ERR_INVALID_ARG, "%s: null pointer argument", what);
    if (kv_misaligned(p, 16)) return fail(IVF_ERR_INVALID_ARG, "%s must be 16-byte aligned", what);
    for (int i = 0; i < n; ++i)
        if (stride[i] < 0 || stride[i] % 8 != 0)
            return fail(IVF_ERR_INVALID_ARG, "%s: stride %lld must be a non-negative multiple of 8 elements", what, (long long)stride[i]);
    return IVF_OK;
}
// A tensor that is written: no two elements in one place.  Axes of one element do not count, the others lie within each other.
int kv_check_apart(const char* what, const int64_t* stride, std::initializer_list<int64_t> size, int dim) {
    std::pair<int64_t, int64_t> axis[3];
    int n = 0, i = 0;
    for (int64_t s : size) {
        if (s > 1) axis[n++] = {stride[i], s};
        ++i;
    }
    std::sort(axis, axis + n);
    int64_t span = dim;
    for (i = 0; i < n; ++i) {
        if (axis[i].first < span)
            return fail(IVF_ERR_INVALID_ARG, "%s is written: its stride of %lld elements must not be below %lld", what, (long long)axis[i].first, (long long)span);
        span += (axis[i].second - 1) * axis[i].first;
    }
    return IVF_OK;
}
int kv_check_cache(const ivf_kv_cache* c, bool keys, bool values) {
    if (!c) return fail(IVF_ERR_INVALID_ARG, "null cache descriptor");
    if (c->dtype != IVF_F16 && c->dtype != IVF_BF16)
        return fail(IVF_ERR_INVALID_ARG, "element type %d: caches are IVF_F16 or IVF_BF16", static_cast<int>(c->dtype));
    int rc = kv_check_page(c->page_size);
    if (rc == IVF_OK) rc = kv_check_dim(c->head_dim);
    if (rc != IVF_OK) return rc;
    if (c->num_pages < 0 || c->num_pages > 0x7FFFFFFF)
        return fail(IVF_ERR_INVALID_ARG, "num_pages = %lld", (long long)c->num_pages);
    if (keys && (rc = kv_check_rows("key cache", c->k, c->k_stride, 3)) != IVF_OK) return rc;
    if (values && (rc = kv_check_rows("value cache", c->v, c->v_stride, 3)) != IVF_OK) return rc;
    return IVF_OK;
}
// Whether `bytes` at `p` share memory with one of `n` rows of `row` bytes, `step` apart.
bool kv_over_rows(const void* p, int64_t bytes, const void* rows, int64_t row, int64_t step, int64_t n) {
    const int64_t at = static_cast<int64_t>(reinterpret_cast<uintptr_t>(p)) - static_cast<int64_t>(reinterpret_cast<uintptr_t>(rows));
    if (bytes <= 0 || row <= 0 || n < 1 || at + bytes <= 0 || at >= (n - 1) * step + row) return false;
    if (at < 0) return true;
    const int64_t k = at / step;
    return at - k * step < row || (k + 1 < n && at + bytes > (k + 1) * step);
}
KvPlane kv_plane(void* base, const int64_t* s) { return KvPlane{base, s[0], s[1], s[2]}; }

}  // namespace
