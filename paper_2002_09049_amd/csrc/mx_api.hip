// C ABI of the microscaled operators (mpq_mx_*, declared in include/mpq.h):
// argument checks, workspaces and launches.  Checks run before any HIP call.
#include <math.h>

#include "internal.hpp"
#include "mpq.h"

using mpq::fail;
using mpq::hip_fail;

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 40;       // rows, tokens and slots
constexpr int64_t kMaxStride = (int64_t)1 << 40;

bool known_dtype(int dtype) { return dtype == MPQ_F32 || dtype == MPQ_F16 || dtype == MPQ_BF16; }
int dtype_bytes(int dtype) { return dtype == MPQ_F32 ? 4 : 2; }
bool aligned(const void *p, int to) { return (uintptr_t)p % to == 0; }

int check_dtype(int dtype, const char *name)
{
    if (known_dtype(dtype)) return MPQ_OK;
    return fail(MPQ_ERR_INVALID_ARG, "%s must be MPQ_F32, MPQ_F16 or MPQ_BF16 (got %d)", name, dtype);
}

// A matrix of rows of d values, ld apart.
int check_matrix(const void *p, int dtype, int64_t rows, int64_t d, int64_t ld, const char *name)
{
    if (ld < d || ld > kMaxStride)
        return fail(MPQ_ERR_INVALID_ARG, "%s: ld must be in [%lld, 2^40] (got %lld)", name, (long long)d,
                    (long long)ld);
    if (rows > 0 && !p) return fail(MPQ_ERR_INVALID_ARG, "%s must not be NULL", name);
    if (!aligned(p, dtype_bytes(dtype)))
        return fail(MPQ_ERR_INVALID_ARG, "%s must be aligned to its element", name);
    return MPQ_OK;
}

int check_fp4_rows(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t d, const char *name)
{
    if (rows < 0 || rows > kMaxRows)
        return fail(MPQ_ERR_INVALID_ARG, "%s: rows must be in [0, 2^40] (got %lld)", name, (long long)rows);
    if (d < 1 || d > MPQ_MX_MAX_D)
        return fail(MPQ_ERR_INVALID_ARG, "d must be in [1, %d] (got %lld)", MPQ_MX_MAX_D, (long long)d);
    if (rows * mpq::mx_row(d) > ((int64_t)1 << 42))
        return fail(MPQ_ERR_INVALID_ARG, "%s: more than 2^42 elements", name);
    if (rows > 0 && (!codes || !scales))
        return fail(MPQ_ERR_INVALID_ARG, "%s: codes and scales must not be NULL", name);
    if (!aligned(codes, 16) || !aligned(scales, 4))
        return fail(MPQ_ERR_INVALID_ARG, "%s: codes must be 16-byte and scales 4-byte aligned", name);
    return MPQ_OK;
}

// The workspace of a call: the caller's, or stream-ordered scratch that is
// given back after the call's launches.
class Workspace {
public:
    int open(void *own, int64_t own_bytes, size_t need, hipStream_t s)
    {
        if (own) {
            if (!aligned(own, 16)) return fail(MPQ_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
            if (own_bytes < 0 || (size_t)own_bytes < need)
                return fail(MPQ_ERR_INVALID_ARG, "workspace of %lld bytes is too small (%zu needed)",
                            (long long)own_bytes, need);
            p_ = own;
            return MPQ_OK;
        }
        if (need == 0) return MPQ_OK;
        const hipError_t e = mpq::scratch_alloc(&p_, need, s);
        if (e != hipSuccess) {
            p_ = nullptr;
            (void)hipGetLastError();
            return fail(MPQ_ERR_NOMEM, "scratch allocation of %zu bytes failed: %s", need, hipGetErrorString(e));
        }
        stream_ = s;
        scratch_ = true;
        return MPQ_OK;
    }
    hipError_t close()
    {
        if (!scratch_) return hipSuccess;
        scratch_ = false;
        return mpq::scratch_free(p_, stream_);
    }
    uint8_t *get() const { return (uint8_t *)p_; }

private:
    void *p_ = nullptr;
    hipStream_t stream_ = nullptr;
    bool scratch_ = false;
};

int done(hipError_t e, hipError_t freed, const char *what)
{
    if (e != hipSuccess) return hip_fail(e, what);
    if (freed != hipSuccess) return hip_fail(freed, "hipFreeAsync");
    return MPQ_OK;
}

int check_product(int64_t n, const uint8_t *w_codes, const uint8_t *w_scales, int64_t c_out, int64_t d,
                  const float *bias, const void *Y, int dtype, int64_t ld)
{
    if (n < 0 || n > MPQ_MX_MAX_N)
        return fail(MPQ_ERR_INVALID_ARG, "n must be in [0, %d] (got %lld)", MPQ_MX_MAX_N, (long long)n);
    int rc = check_dtype(dtype, "dtype");
    if (rc == MPQ_OK) rc = check_fp4_rows(w_codes, w_scales, c_out, d, "weights");
    if (rc == MPQ_OK) rc = check_matrix(Y, dtype, c_out > 0 ? n : 0, c_out, ld, "Y");
    if (rc == MPQ_OK && !aligned(bias, 4)) rc = fail(MPQ_ERR_INVALID_ARG, "bias must be 4-byte aligned");
    return rc;
}

mpq::MxProduct product(const uint8_t *xc, const uint8_t *xs, int64_t n, const uint8_t *wc, const uint8_t *ws,
                       int64_t c_out, int64_t d, const float *bias, void *Y, int dtype, int64_t ld)
{
    mpq::MxProduct p = {};
    p.xc = xc;
    p.xs = xs;
    p.wc = wc;
    p.ws = ws;
    p.bias = bias;
    p.Y = Y;
    p.dtype = dtype;
    p.nb = (int)(mpq::mx_row(d) / MPQ_MX_BLOCK);
    p.n = n;
    p.c = c_out;
    p.ldy = ld;
    return p;
}

// Bytes of n quantized rows of d: the codes, then the scales, 16-byte pieces.
size_t fp4_bytes(int64_t n, int64_t d)
{
    const int64_t w = mpq::mx_row(d);
    return (size_t)(n * (w / 2) + (n * (w / MPQ_MX_BLOCK) + 15) / 16 * 16);
}

// The workspace of a linear call: its quantized tokens, where they are not
// quantized inside the product.
size_t linear_bytes(int64_t n, int64_t d) { return mpq::mx_quantizes_inside(n) ? 0 : fp4_bytes(n, d); }

int view_cache(const mpq_mx_cache *c, mpq::MxCacheView *v)
{
    if (!c) return fail(MPQ_ERR_INVALID_ARG, "cache must not be NULL");
    if (c->format != MPQ_MX_FP4 && c->format != MPQ_MX_FP8)
        return fail(MPQ_ERR_INVALID_ARG, "cache format must be MPQ_MX_FP4 or MPQ_MX_FP8 (got %d)", c->format);
    if (c->head_dim < 1 || c->head_dim > MPQ_MX_MAX_HEAD_DIM)
        return fail(MPQ_ERR_INVALID_ARG, "head_dim must be in [1, %d] (got %d)", MPQ_MX_MAX_HEAD_DIM, c->head_dim);
    if (c->page_size < 16 || c->page_size > MPQ_MX_MAX_PAGE || c->page_size % 16 != 0)
        return fail(MPQ_ERR_INVALID_ARG, "page_size must be a multiple of 16 of at most %d (got %d)", MPQ_MX_MAX_PAGE,
                    c->page_size);
    if (c->kv_heads < 1 || c->kv_heads > 65535)
        return fail(MPQ_ERR_INVALID_ARG, "kv_heads must be in [1, 65535] (got %d)", c->kv_heads);
    if (c->n_pages < 1 || c->n_pages > 0x7fffffff || c->n_pages * c->page_size >= kMaxRows)
        return fail(MPQ_ERR_INVALID_ARG, "n_pages must be in [1, 2^31) with n_pages * page_size < 2^40 (got %lld)",
                    (long long)c->n_pages);
    if (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales)
        return fail(MPQ_ERR_INVALID_ARG, "the cache's arrays must not be NULL");
    if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scales, 4) || !aligned(c->v_scales, 4))
        return fail(MPQ_ERR_INVALID_ARG, "the cache's codes must be 16-byte and its scales 4-byte aligned");
    v->k = c->k_codes;
    v->v = c->v_codes;
    v->ks = c->k_scales;
    v->vs = c->v_scales;
    v->n_pages = c->n_pages;
    v->page = c->page_size;
    v->heads = c->kv_heads;
    v->dim = c->head_dim;
    v->nb = (c->head_dim + MPQ_MX_BLOCK - 1) / MPQ_MX_BLOCK;
    v->fmt = c->format;
    return MPQ_OK;
}

int check_stride(int64_t v, const char *name)
{
    if (v >= 0 && v <= kMaxStride) return MPQ_OK;
    return fail(MPQ_ERR_INVALID_ARG, "%s must be in [0, 2^40] (got %lld)", name, (long long)v);
}

// Output rows of d values: one of several does not overlap the next.
int check_apart(int64_t rows, int64_t stride, int64_t d, const char *name)
{
    if (rows <= 1 || stride >= d) return MPQ_OK;
    return fail(MPQ_ERR_INVALID_ARG, "%s must be at least head_dim (got %lld)", name, (long long)stride);
}

// The K, V and slots of a write or read.
int check_rows(const mpq::MxCacheView &c, const mpq::MxRows &r, int64_t n, const int64_t *slots)
{
    if (n < 0 || n > (int64_t)0x7fffffff)
        return fail(MPQ_ERR_INVALID_ARG, "n must be in [0, 2^31) (got %lld)", (long long)n);
    int rc = check_dtype(r.dtype, "dtype");
    if (rc == MPQ_OK) rc = check_stride(r.k_tok, "k_stride");
    if (rc == MPQ_OK) rc = check_stride(r.k_head, "k_head_stride");
    if (rc == MPQ_OK) rc = check_stride(r.v_tok, "v_stride");
    if (rc == MPQ_OK) rc = check_stride(r.v_head, "v_head_stride");
    if (rc != MPQ_OK) return rc;
    if (n > 0 && (!r.K || !r.V || !slots)) return fail(MPQ_ERR_INVALID_ARG, "K, V and slots must not be NULL");
    const int e = dtype_bytes(r.dtype);
    if (!aligned(r.K, e) || !aligned(r.V, e) || !aligned(slots, 8))
        return fail(MPQ_ERR_INVALID_ARG, "K, V and slots must be aligned to their elements");
    if (n > 0 && n * c.heads > kMaxRows / 4)
        return fail(MPQ_ERR_INVALID_ARG, "n * kv_heads is too large (%lld * %d)", (long long)n, c.heads);
    return MPQ_OK;
}

// The shape of an attention call (not its pointers).
int shape_attend(const mpq_mx_cache *cache, int64_t batch, int64_t q_heads, int64_t max_pages, mpq::MxAttend *a)
{
    int rc = view_cache(cache, &a->c);
    if (rc != MPQ_OK) return rc;
    if (batch < 0 || batch > 65535)
        return fail(MPQ_ERR_INVALID_ARG, "batch must be in [0, 65535] (got %lld)", (long long)batch);
    if (q_heads < 1 || q_heads > 65535 || q_heads % a->c.heads != 0)
        return fail(MPQ_ERR_INVALID_ARG, "q_heads must be a multiple of kv_heads in [1, 65535] (got %lld)",
                    (long long)q_heads);
    if (max_pages < 0 || max_pages > MPQ_MX_MAX_TOKENS / a->c.page)
        return fail(MPQ_ERR_INVALID_ARG, "max_pages must be in [0, %d] for pages of %d (got %lld)",
                    MPQ_MX_MAX_TOKENS / a->c.page, a->c.page, (long long)max_pages);
    a->batch = batch;
    a->q_heads = (int)q_heads;
    a->group = (int)(q_heads / a->c.heads);
    a->most = (int)(max_pages * a->c.page);
    return MPQ_OK;
}

}  // namespace

extern "C" {

int mpq_mx_quantize(const void *X, int dtype, int64_t rows, int64_t d, int64_t ld, uint8_t *codes, uint8_t *scales,
                    void *stream)
{
    int rc = check_dtype(dtype, "dtype");
    if (rc == MPQ_OK) rc = check_fp4_rows(codes, scales, rows, d, "rows");
    if (rc == MPQ_OK) rc = check_matrix(X, dtype, rows, d, ld, "X");
    if (rc != MPQ_OK || rows == 0) return rc;
    return done(mpq::launch_mx_quantize(X, dtype, rows, d, ld, codes, scales, (hipStream_t)stream), hipSuccess,
                "mx quantize launch");
}

int mpq_mx_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t d, void *Y, int dtype,
                      int64_t ld, void *stream)
{
    int rc = check_dtype(dtype, "dtype");
    if (rc == MPQ_OK) rc = check_fp4_rows(codes, scales, rows, d, "rows");
    if (rc == MPQ_OK) rc = check_matrix(Y, dtype, rows, d, ld, "Y");
    if (rc != MPQ_OK || rows == 0) return rc;
    return done(mpq::launch_mx_dequantize(codes, scales, rows, d, Y, dtype, ld, (hipStream_t)stream), hipSuccess,
                "mx dequantize launch");
}

int mpq_mx_product(const uint8_t *x_codes, const uint8_t *x_scales, int64_t n, const uint8_t *w_codes,
                   const uint8_t *w_scales, int64_t c_out, int64_t d, const float *bias_opt, void *Y, int dtype,
                   int64_t ld, void *stream)
{
    int rc = check_product(n, w_codes, w_scales, c_out, d, bias_opt, Y, dtype, ld);
    if (rc == MPQ_OK) rc = check_fp4_rows(x_codes, x_scales, n, d, "tokens");
    if (rc != MPQ_OK || n == 0 || c_out == 0) return rc;
    return done(mpq::launch_mx_product(product(x_codes, x_scales, n, w_codes, w_scales, c_out, d, bias_opt, Y, dtype,
                                               ld), (hipStream_t)stream),
                hipSuccess, "mx product launch");
}

int64_t mpq_mx_linear_workspace(int64_t n, int64_t c_out, int64_t d)
{
    if (n < 0 || n > MPQ_MX_MAX_N || c_out < 0 || d < 1 || d > MPQ_MX_MAX_D)
        return fail(MPQ_ERR_INVALID_ARG, "n, c_out or d out of range (%lld, %lld, %lld)", (long long)n,
                    (long long)c_out, (long long)d);
    return (int64_t)linear_bytes(n, d);
}

int mpq_mx_linear(const void *X, int x_dtype, int64_t n, int64_t x_ld, const uint8_t *w_codes,
                  const uint8_t *w_scales, int64_t c_out, int64_t d, const float *bias_opt, void *Y, int dtype,
                  int64_t ld, void *workspace_opt, int64_t workspace_bytes, void *stream)
{
    int rc = check_product(n, w_codes, w_scales, c_out, d, bias_opt, Y, dtype, ld);
    if (rc == MPQ_OK) rc = check_dtype(x_dtype, "x_dtype");
    if (rc == MPQ_OK) rc = check_matrix(X, x_dtype, n, d, x_ld, "X");
    if (rc != MPQ_OK || n == 0 || c_out == 0) return rc;
    hipStream_t s = (hipStream_t)stream;
    Workspace ws;
    rc = ws.open(workspace_opt, workspace_bytes, linear_bytes(n, d), s);
    if (rc != MPQ_OK) return rc;
    if (mpq::mx_quantizes_inside(n))
        return done(mpq::launch_mx_token(product(nullptr, nullptr, n, w_codes, w_scales, c_out, d, bias_opt, Y, dtype, ld),
                                         X, x_dtype, x_ld, d, s),
                    hipSuccess, "mx token launch");
    uint8_t *xc = ws.get(), *xs = xc + n * (mpq::mx_row(d) / 2);
    hipError_t e = mpq::launch_mx_quantize(X, x_dtype, n, d, x_ld, xc, xs, s);
    if (e == hipSuccess)
        e = mpq::launch_mx_product(product(xc, xs, n, w_codes, w_scales, c_out, d, bias_opt, Y, dtype, ld), s);
    const hipError_t freed = ws.close();
    return done(e, freed, "mx linear launch");
}

int mpq_mx_cache_write(const mpq_mx_cache *cache, const void *K, int64_t k_stride, int64_t k_head_stride,
                       const void *V, int64_t v_stride, int64_t v_head_stride, int dtype, int64_t n,
                       const int64_t *slots, void *stream)
{
    mpq::MxCacheView c;
    const mpq::MxRows r = {(void *)K, (void *)V, k_stride, k_head_stride, v_stride, v_head_stride, dtype};
    int rc = view_cache(cache, &c);
    if (rc == MPQ_OK) rc = check_rows(c, r, n, slots);
    if (rc != MPQ_OK || n == 0) return rc;
    return done(mpq::launch_mx_cache_write(c, r, n, slots, (hipStream_t)stream), hipSuccess, "mx cache write launch");
}

int mpq_mx_cache_read(const mpq_mx_cache *cache, void *K, int64_t k_stride, int64_t k_head_stride, void *V,
                      int64_t v_stride, int64_t v_head_stride, int dtype, int64_t n, const int64_t *slots, void *stream)
{
    mpq::MxCacheView c;
    const mpq::MxRows r = {K, V, k_stride, k_head_stride, v_stride, v_head_stride, dtype};
    int rc = view_cache(cache, &c);
    if (rc == MPQ_OK) rc = check_rows(c, r, n, slots);
    if (rc == MPQ_OK) rc = check_apart(n, k_stride, c.dim, "k_stride");
    if (rc == MPQ_OK) rc = check_apart(c.heads, k_head_stride, c.dim, "k_head_stride");
    if (rc == MPQ_OK) rc = check_apart(n, v_stride, c.dim, "v_stride");
    if (rc == MPQ_OK) rc = check_apart(c.heads, v_head_stride, c.dim, "v_head_stride");
    if (rc != MPQ_OK || n == 0) return rc;
    return done(mpq::launch_mx_cache_read(c, r, n, slots, (hipStream_t)stream), hipSuccess, "mx cache read launch");
}

int64_t mpq_mx_attend_workspace(const mpq_mx_cache *cache, int64_t batch, int64_t q_heads, int64_t max_pages)
{
    mpq::MxAttend a = {};
    const int rc = shape_attend(cache, batch, q_heads, max_pages, &a);
    return rc != MPQ_OK ? rc : (int64_t)mpq::mx_attend_plan(a);
}

int mpq_mx_attend(const mpq_mx_cache *cache, const void *Q, int64_t q_stride, int64_t q_head_stride, int dtype,
                  int64_t batch, int64_t q_heads, const int32_t *page_table, int64_t table_ld, int64_t max_pages,
                  const int32_t *lengths, int64_t window, float scale, void *O, int64_t o_stride,
                  int64_t o_head_stride, float *lse_opt, void *workspace_opt, int64_t workspace_bytes, void *stream)
{
    mpq::MxAttend a = {};
    int rc = shape_attend(cache, batch, q_heads, max_pages, &a);
    if (rc == MPQ_OK) rc = check_dtype(dtype, "dtype");
    if (rc == MPQ_OK) rc = check_stride(q_stride, "q_stride");
    if (rc == MPQ_OK) rc = check_stride(q_head_stride, "q_head_stride");
    if (rc == MPQ_OK) rc = check_stride(o_stride, "o_stride");
    if (rc == MPQ_OK) rc = check_stride(o_head_stride, "o_head_stride");
    if (rc == MPQ_OK) rc = check_apart(batch, o_stride, a.c.dim, "o_stride");
    if (rc == MPQ_OK) rc = check_apart(q_heads, o_head_stride, a.c.dim, "o_head_stride");
    if (rc != MPQ_OK) return rc;
    if (table_ld < max_pages || table_ld > kMaxStride)
        return fail(MPQ_ERR_INVALID_ARG, "table_ld must be at least max_pages (got %lld, %lld)", (long long)table_ld,
                    (long long)max_pages);
    if (window < 0) return fail(MPQ_ERR_INVALID_ARG, "window must be >= 0 (got %lld)", (long long)window);
    if (!isfinite(scale)) return fail(MPQ_ERR_INVALID_ARG, "scale must be finite");
    if (batch > 0 && (!Q || !O || !lengths || (!page_table && max_pages > 0)))
        return fail(MPQ_ERR_INVALID_ARG, "Q, O, page_table and lengths must not be NULL");
    const int e = dtype_bytes(dtype);
    if (!aligned(Q, e) || !aligned(O, e) || !aligned(page_table, 4) || !aligned(lengths, 4) || !aligned(lse_opt, 4))
        return fail(MPQ_ERR_INVALID_ARG, "Q, O, page_table, lengths and lse must be aligned to their elements");
    if (batch == 0) return MPQ_OK;
    a.Q = Q;
    a.q_batch = q_stride;
    a.q_head = q_head_stride;
    a.O = O;
    a.o_batch = o_stride;
    a.o_head = o_head_stride;
    a.dtype = dtype;
    a.lse = lse_opt;
    a.table = page_table;
    a.table_ld = table_ld;
    a.lengths = lengths;
    a.window = (int)(window > MPQ_MX_MAX_TOKENS ? MPQ_MX_MAX_TOKENS : window);
    a.scale = scale;
    const size_t need = mpq::mx_attend_plan(a);
    hipStream_t s = (hipStream_t)stream;
    Workspace ws;
    rc = ws.open(workspace_opt, workspace_bytes, need, s);
    if (rc != MPQ_OK) return rc;
    a.part = (float *)ws.get();
    const hipError_t err = mpq::launch_mx_attend(a, s);
    const hipError_t freed = ws.close();
    return done(err, freed, "mx attend launch");
}

}  // extern "C"
