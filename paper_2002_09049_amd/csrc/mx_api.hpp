// What the C entries of the microscaled operators share: checks of their
// arguments, workspaces and errors.
#pragma once

#include "internal.hpp"
#include "mpq.h"

using mpq::fail;
using mpq::hip_fail;

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 40;       // rows, tokens and slots
constexpr int64_t kMaxStride = (int64_t)1 << 40;

inline bool known_dtype(int dtype) { return dtype == MPQ_F32 || dtype == MPQ_F16 || dtype == MPQ_BF16; }
inline int dtype_bytes(int dtype) { return dtype == MPQ_F32 ? 4 : 2; }
inline bool aligned(const void *p, int to) { return (uintptr_t)p % to == 0; }

inline int check_dtype(int dtype, const char *name)
{
    if (known_dtype(dtype)) return MPQ_OK;
    return fail(MPQ_ERR_INVALID_ARG, "%s must be MPQ_F32, MPQ_F16 or MPQ_BF16 (got %d)", name, dtype);
}

// A matrix of rows of d values, ld apart.
inline int check_matrix(const void *p, int dtype, int64_t rows, int64_t d, int64_t ld, const char *name)
{
    if (ld < d || ld > kMaxStride)
        return fail(MPQ_ERR_INVALID_ARG, "%s: ld must be in [%lld, 2^40] (got %lld)", name, (long long)d,
                    (long long)ld);
    if (rows > 0 && !p) return fail(MPQ_ERR_INVALID_ARG, "%s must not be NULL", name);
    if (!aligned(p, dtype_bytes(dtype)))
        return fail(MPQ_ERR_INVALID_ARG, "%s must be aligned to its element", name);
    return MPQ_OK;
}

inline int check_fp4_rows(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t d, const char *name)
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

inline int done(hipError_t e, hipError_t freed, const char *what)
{
    if (e != hipSuccess) return hip_fail(e, what);
    if (freed != hipSuccess) return hip_fail(freed, "hipFreeAsync");
    return MPQ_OK;
}

inline int view_cache(const mpq_mx_cache *c, mpq::MxCacheView *v)
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

inline int check_stride(int64_t v, const char *name)
{
    if (v >= 0 && v <= kMaxStride) return MPQ_OK;
    return fail(MPQ_ERR_INVALID_ARG, "%s must be in [0, 2^40] (got %lld)", name, (long long)v);
}

// Output rows of d values: one of several does not overlap the next.
inline int check_apart(int64_t rows, int64_t stride, int64_t d, const char *name)
{
    if (rows <= 1 || stride >= d) return MPQ_OK;
    return fail(MPQ_ERR_INVALID_ARG, "%s must be at least head_dim (got %lld)", name, (long long)stride);
}

}  // namespace
