// C ABI of a serving step's operators around the microscaled products and cache
// (declared in include/mpq.h): argument checks, workspaces and launches.  Checks
// run before any HIP call.
#include <math.h>

#include "mx_api.hpp"

namespace {

// A device array of `count` elements of `size` bytes; may be NULL if there are none.
int check_array(const void *p, int64_t count, int size, const char *name)
{
    if (count > 0 && !p) return fail(MPQ_ERR_INVALID_ARG, "%s must not be NULL", name);
    if (!aligned(p, size)) return fail(MPQ_ERR_INVALID_ARG, "%s must be aligned to its element", name);
    return MPQ_OK;
}

int check_range(int64_t v, int64_t lo, int64_t hi, const char *name)
{
    if (v >= lo && v <= hi) return MPQ_OK;
    return fail(MPQ_ERR_INVALID_ARG, "%s must be in [%lld, %lld] (got %lld)", name, (long long)lo, (long long)hi,
                (long long)v);
}

// Heads [n][heads][dim]; as an output, none overlaps the next.
int check_heads(const void *p, int dtype, int64_t n, int64_t heads, int64_t dim, int64_t tok, int64_t head, bool output,
                const char *name)
{
    int rc = check_stride(tok, name);
    if (rc == MPQ_OK) rc = check_stride(head, name);
    if (rc == MPQ_OK) rc = check_array(p, n * heads, dtype_bytes(dtype), name);
    if (rc == MPQ_OK && output) rc = check_apart(n, tok, dim, name);
    if (rc == MPQ_OK && output) rc = check_apart(heads, head, dim, name);
    return rc;
}

// What rotation and append share; r's Q, K and their outputs are set.
int check_rotate(mpq::MxRotate &r, int64_t n, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int dtype,
                 const int32_t *positions, const double *freqs, int64_t rot, int interleaved, const float *q_weight,
                 const float *k_weight, float eps)
{
    int rc = check_dtype(dtype, "dtype");
    if (rc == MPQ_OK) rc = check_range(n, 0, 0x7fffffff, "n");
    if (rc == MPQ_OK) rc = check_range(q_heads, 1, 65535, "q_heads");
    if (rc == MPQ_OK) rc = check_range(kv_heads, 1, 65535, "kv_heads");
    if (rc == MPQ_OK) rc = check_range(head_dim, 1, MPQ_MX_MAX_HEAD_DIM, "head_dim");
    if (rc == MPQ_OK) rc = check_range(rot, 0, head_dim, "rot");
    if (rc != MPQ_OK) return rc;
    if (rot % 2 != 0) return fail(MPQ_ERR_INVALID_ARG, "rot must be even (got %lld)", (long long)rot);
    if (interleaved != 0 && interleaved != 1)
        return fail(MPQ_ERR_INVALID_ARG, "interleaved must be 0 or 1 (got %d)", interleaved);
    if ((q_weight || k_weight) && !(isfinite(eps) && eps > 0.0f))
        return fail(MPQ_ERR_INVALID_ARG, "eps must be finite and positive");
    rc = check_array(positions, rot > 0 ? n : 0, 4, "positions");
    if (rc == MPQ_OK) rc = check_array(freqs, n > 0 ? rot : 0, 8, "freqs");
    if (rc == MPQ_OK) rc = check_array(q_weight, 0, 4, "q_weight");
    if (rc == MPQ_OK) rc = check_array(k_weight, 0, 4, "k_weight");
    if (rc != MPQ_OK) return rc;
    r.dtype = dtype;
    r.n = n;
    r.heads = (int)q_heads;
    r.kv = (int)kv_heads;
    r.dim = (int)head_dim;
    r.rot = (int)rot;
    r.qw = q_weight;
    r.kw = k_weight;
    r.eps = eps;
    r.interleaved = interleaved;
    r.positions = positions;
    r.freqs = freqs;
    return MPQ_OK;
}

// The shape of a product by experts (not its pointers).
int check_experts(int64_t n, int64_t m, int64_t experts, int64_t c_out, int64_t d)
{
    int rc = check_range(n, 0, MPQ_MX_MAX_N, "n");
    if (rc == MPQ_OK) rc = check_range(m, 0, MPQ_MX_MAX_ROWS, "m");
    if (rc == MPQ_OK) rc = check_range(experts, 1, MPQ_MX_MAX_EXPERTS, "experts");
    if (rc == MPQ_OK) rc = check_range(d, 1, MPQ_MX_MAX_D, "d");
    if (rc == MPQ_OK) rc = check_range(c_out, 0, ((int64_t)1 << 42) / (experts * mpq::mx_row(d)), "c_out");
    if (rc == MPQ_OK && (n + 1) * (mpq::mx_row(d) / 2) > 0x7fffffff)
        rc = fail(MPQ_ERR_INVALID_ARG, "X: (n + 1) * D must be below 2^32 (got %lld rows of %lld)", (long long)n, (long long)d);
    return rc;
}

int check_route(int64_t n, int64_t experts, int64_t k)
{
    int rc = check_range(n, 0, MPQ_MX_MAX_N, "n");
    if (rc == MPQ_OK) rc = check_range(experts, 1, MPQ_MX_MAX_EXPERTS, "experts");
    if (rc == MPQ_OK) rc = check_range(k, 1, experts < MPQ_MX_MAX_CHOICES ? experts : MPQ_MX_MAX_CHOICES, "k");
    return rc;
}

}  // namespace

extern "C" {

int mpq_mx_plan(const int32_t *cached, const int32_t *fresh, int64_t batch, int32_t *page_table, int64_t table_ld,
                int64_t max_pages, const int32_t *free_pages, int64_t n_free, const int32_t *taken, int64_t page_size,
                int64_t max_tokens, int64_t *slots, int32_t *positions, int32_t *starts, int32_t *lengths,
                int32_t *taken_out, void *stream)
{
    int rc = check_range(batch, 0, 65535, "batch");
    if (rc == MPQ_OK) rc = check_range(page_size, 16, MPQ_MX_MAX_PAGE, "page_size");
    if (rc == MPQ_OK && page_size % 16 != 0)
        rc = fail(MPQ_ERR_INVALID_ARG, "page_size must be a multiple of 16 (got %lld)", (long long)page_size);
    if (rc == MPQ_OK) rc = check_range(max_pages, 0, MPQ_MX_MAX_TOKENS / page_size, "max_pages");
    if (rc == MPQ_OK) rc = check_range(table_ld, max_pages, kMaxStride, "table_ld");
    if (rc == MPQ_OK) rc = check_range(n_free, 0, 0x7fffffff, "n_free");
    if (rc == MPQ_OK) rc = check_range(max_tokens, 0, MPQ_MX_MAX_TOKENS, "max_tokens");
    if (rc == MPQ_OK) rc = check_array(cached, batch, 4, "cached");
    if (rc == MPQ_OK) rc = check_array(fresh, batch, 4, "fresh");
    if (rc == MPQ_OK) rc = check_array(page_table, batch * max_pages, 4, "page_table");
    if (rc == MPQ_OK) rc = check_array(free_pages, n_free, 4, "free_pages");
    if (rc == MPQ_OK) rc = check_array(taken, 1, 4, "taken");
    if (rc == MPQ_OK) rc = check_array(slots, max_tokens, 8, "slots");
    if (rc == MPQ_OK) rc = check_array(positions, max_tokens, 4, "positions");
    if (rc == MPQ_OK) rc = check_array(starts, 1, 4, "starts");
    if (rc == MPQ_OK) rc = check_array(lengths, batch, 4, "lengths");
    if (rc == MPQ_OK) rc = check_array(taken_out, 1, 4, "taken_out");
    if (rc == MPQ_OK && taken == taken_out) rc = fail(MPQ_ERR_INVALID_ARG, "taken_out must not be taken");
    if (rc == MPQ_OK && batch > 0 && (lengths == cached || lengths == fresh || starts == cached || starts == fresh))
        rc = fail(MPQ_ERR_INVALID_ARG, "starts and lengths must not be cached or fresh");
    if (rc != MPQ_OK) return rc;
    mpq::MxPlan p = {};
    p.cached = cached;
    p.fresh = fresh;
    p.batch = batch;
    p.table = page_table;
    p.table_ld = table_ld;
    p.columns = max_pages;
    p.free = free_pages;
    p.n_free = n_free;
    p.taken = taken;
    p.page = (int)page_size;
    p.tokens = max_tokens;
    p.slots = slots;
    p.positions = positions;
    p.starts = starts;
    p.lengths = lengths;
    p.taken_out = taken_out;
    return done(mpq::launch_mx_plan(p, (hipStream_t)stream), hipSuccess, "mx plan launch");
}

int mpq_mx_rotate(const void *Q, int64_t q_stride, int64_t q_head_stride, const void *K, int64_t k_stride,
                  int64_t k_head_stride, int dtype, int64_t n, int64_t q_heads, int64_t kv_heads, int64_t head_dim,
                  const int32_t *positions, const double *freqs, int64_t rot, int interleaved, const float *q_weight_opt,
                  const float *k_weight_opt, float eps, void *QO, int64_t qo_stride, int64_t qo_head_stride, void *KO,
                  int64_t ko_stride, int64_t ko_head_stride, void *stream)
{
    mpq::MxRotate r = {};
    int rc = check_rotate(r, n, q_heads, kv_heads, head_dim, dtype, positions, freqs, rot, interleaved, q_weight_opt,
                          k_weight_opt, eps);
    if (rc == MPQ_OK) rc = check_heads(Q, dtype, n, q_heads, head_dim, q_stride, q_head_stride, false, "Q");
    if (rc == MPQ_OK) rc = check_heads(K, dtype, n, kv_heads, head_dim, k_stride, k_head_stride, false, "K");
    if (rc == MPQ_OK) rc = check_heads(QO, dtype, n, q_heads, head_dim, qo_stride, qo_head_stride, true, "QO");
    if (rc == MPQ_OK) rc = check_heads(KO, dtype, n, kv_heads, head_dim, ko_stride, ko_head_stride, true, "KO");
    if (rc != MPQ_OK || n == 0) return rc;
    r.Q = Q;
    r.K = K;
    r.q_tok = q_stride;
    r.q_head = q_head_stride;
    r.k_tok = k_stride;
    r.k_head = k_head_stride;
    r.QO = QO;
    r.KO = KO;
    r.qo_tok = qo_stride;
    r.qo_head = qo_head_stride;
    r.ko_tok = ko_stride;
    r.ko_head = ko_head_stride;
    return done(mpq::launch_mx_rotate(r, false, (hipStream_t)stream), hipSuccess, "mx rotate launch");
}

int mpq_mx_cache_append(const mpq_mx_cache *cache, const void *Q, int64_t q_stride, int64_t q_head_stride, const void *K,
                        int64_t k_stride, int64_t k_head_stride, const void *V, int64_t v_stride, int64_t v_head_stride,
                        int dtype, int64_t n, int64_t q_heads, const int32_t *positions, const int64_t *slots,
                        const double *freqs, int64_t rot, int interleaved, const float *q_weight_opt,
                        const float *k_weight_opt, float eps, void *QO, int64_t qo_stride, int64_t qo_head_stride,
                        void *stream)
{
    mpq::MxRotate r = {};
    int rc = view_cache(cache, &r.c);
    if (rc == MPQ_OK)
        rc = check_rotate(r, n, q_heads, r.c.heads, r.c.dim, dtype, positions, freqs, rot, interleaved, q_weight_opt,
                          k_weight_opt, eps);
    if (rc == MPQ_OK) rc = check_heads(Q, dtype, n, q_heads, r.c.dim, q_stride, q_head_stride, false, "Q");
    if (rc == MPQ_OK) rc = check_heads(K, dtype, n, r.c.heads, r.c.dim, k_stride, k_head_stride, false, "K");
    if (rc == MPQ_OK) rc = check_heads(V, dtype, n, r.c.heads, r.c.dim, v_stride, v_head_stride, false, "V");
    if (rc == MPQ_OK) rc = check_heads(QO, dtype, n, q_heads, r.c.dim, qo_stride, qo_head_stride, true, "QO");
    if (rc == MPQ_OK) rc = check_array(slots, n, 8, "slots");
    if (rc != MPQ_OK || n == 0) return rc;
    r.Q = Q;
    r.K = K;
    r.V = V;
    r.q_tok = q_stride;
    r.q_head = q_head_stride;
    r.k_tok = k_stride;
    r.k_head = k_head_stride;
    r.v_tok = v_stride;
    r.v_head = v_head_stride;
    r.QO = QO;
    r.qo_tok = qo_stride;
    r.qo_head = qo_head_stride;
    r.slots = slots;
    return done(mpq::launch_mx_rotate(r, true, (hipStream_t)stream), hipSuccess, "mx append launch");
}

int64_t mpq_mx_route_workspace(int64_t n, int64_t experts, int64_t k)
{
    const int rc = check_route(n, experts, k);
    return rc != MPQ_OK ? rc : (int64_t)mpq::mx_route_bytes(n, experts);
}

int mpq_mx_route(const void *logits, int dtype, int64_t n, int64_t experts, int64_t ld, int64_t k, int renorm,
                 int32_t *chosen, float *weights, int32_t *order, int32_t *place, int32_t *offsets, void *workspace_opt,
                 int64_t workspace_bytes, void *stream)
{
    int rc = check_route(n, experts, k);
    if (rc == MPQ_OK) rc = check_dtype(dtype, "dtype");
    if (rc == MPQ_OK) rc = check_matrix(logits, dtype, n, experts, ld, "logits");
    if (rc == MPQ_OK) rc = check_range(renorm, 0, 1, "renorm");
    if (rc == MPQ_OK) rc = check_array(chosen, n, 4, "chosen");
    if (rc == MPQ_OK) rc = check_array(weights, n, 4, "weights");
    if (rc == MPQ_OK) rc = check_array(order, n, 4, "order");
    if (rc == MPQ_OK) rc = check_array(place, n, 4, "place");
    if (rc == MPQ_OK) rc = check_array(offsets, 1, 4, "offsets");
    if (rc != MPQ_OK) return rc;
    hipStream_t s = (hipStream_t)stream;
    Workspace ws;
    rc = ws.open(workspace_opt, workspace_bytes, mpq::mx_route_bytes(n, experts), s);
    if (rc != MPQ_OK) return rc;
    mpq::MxRoute r = {};
    r.logits = logits;
    r.dtype = dtype;
    r.n = n;
    r.ld = ld;
    r.experts = (int)experts;
    r.k = (int)k;
    r.renorm = renorm;
    r.chosen = chosen;
    r.order = order;
    r.place = place;
    r.offsets = offsets;
    r.weights = weights;
    const hipError_t e = mpq::launch_mx_route(r, ws.get(), s);
    const hipError_t freed = ws.close();
    return done(e, freed, "mx route launch");
}

int64_t mpq_mx_experts_workspace(int64_t n, int64_t m, int64_t experts, int64_t c_out, int64_t d)
{
    const int rc = check_experts(n, m, experts, c_out, d);
    return rc != MPQ_OK ? rc : n == 0 || m == 0 || c_out == 0 ? 0 : (int64_t)mpq::mx_experts_bytes(n, m, experts, c_out, d);
}

int mpq_mx_experts(const void *X, int x_dtype, int64_t n, int64_t x_ld, const uint8_t *w_codes, const uint8_t *w_scales,
                   int64_t experts, int64_t c_out, int64_t d, const int32_t *offsets, const int32_t *order_opt, int64_t m,
                   int64_t k, const float *bias_opt, void *Y, int dtype, int64_t ld, void *workspace_opt,
                   int64_t workspace_bytes, void *stream)
{
    int rc = check_experts(n, m, experts, c_out, d);
    if (rc == MPQ_OK) rc = check_dtype(x_dtype, "x_dtype");
    if (rc == MPQ_OK) rc = check_dtype(dtype, "dtype");
    if (rc == MPQ_OK) rc = check_fp4_rows(w_codes, w_scales, experts * c_out, d, "weights");
    if (rc == MPQ_OK) rc = check_matrix(X, x_dtype, n, d, x_ld, "X");
    if (rc == MPQ_OK) rc = check_matrix(Y, dtype, c_out > 0 ? m : 0, c_out, ld, "Y");
    if (rc == MPQ_OK) rc = check_array(offsets, 1, 4, "offsets");
    if (rc == MPQ_OK) rc = check_array(order_opt, 0, 4, "order");
    if (rc == MPQ_OK) rc = check_array(bias_opt, 0, 4, "bias");
    if (rc == MPQ_OK) rc = check_range(k, 1, 0x7fffffff, "k");
    if (rc == MPQ_OK && !order_opt && (m != n || k != 1))
        rc = fail(MPQ_ERR_INVALID_ARG, "without order, m must be n and k 1 (got %lld, %lld, %lld)", (long long)m,
                  (long long)n, (long long)k);
    if (rc == MPQ_OK && n == 0 && m > 0) rc = fail(MPQ_ERR_INVALID_ARG, "m must be 0 where n is (got %lld)", (long long)m);
    if (rc != MPQ_OK || m == 0 || c_out == 0) return rc;
    hipStream_t s = (hipStream_t)stream;
    Workspace ws;
    rc = ws.open(workspace_opt, workspace_bytes, mpq::mx_experts_bytes(n, m, experts, c_out, d), s);
    if (rc != MPQ_OK) return rc;
    mpq::MxExperts g = {};
    g.p.wc = w_codes;
    g.p.ws = w_scales;
    g.p.bias = bias_opt;
    g.p.Y = Y;
    g.p.dtype = dtype;
    g.p.nb = (int)(mpq::mx_row(d) / MPQ_MX_BLOCK);
    g.p.n = n;
    g.p.c = c_out;
    g.p.ldy = ld;
    g.experts = (int)experts;
    g.choices = (int)k;
    g.m = m;
    g.offsets = offsets;
    g.order = order_opt;
    const hipError_t e = mpq::launch_mx_experts(g, X, x_dtype, x_ld, d, ws.get(), s);
    const hipError_t freed = ws.close();
    return done(e, freed, "mx experts launch");
}

int mpq_mx_combine(const void *Y, int y_dtype, int64_t m, int64_t c, int64_t y_ld, const int32_t *place,
                   const float *weights, int64_t n, int64_t k, const void *residual_opt, int64_t residual_ld, void *Z,
                   int dtype, int64_t ld, void *stream)
{
    int rc = check_range(n, 0, MPQ_MX_MAX_N, "n");
    if (rc == MPQ_OK) rc = check_range(m, 0, MPQ_MX_MAX_ROWS, "m");
    if (rc == MPQ_OK) rc = check_range(c, 0, MPQ_MX_MAX_D, "c");
    if (rc == MPQ_OK) rc = check_range(k, 0, MPQ_MX_MAX_CHOICES, "k");
    if (rc == MPQ_OK) rc = check_dtype(y_dtype, "y_dtype");
    if (rc == MPQ_OK) rc = check_dtype(dtype, "dtype");
    if (rc == MPQ_OK) rc = check_matrix(Y, y_dtype, c > 0 ? m : 0, c, y_ld, "Y");
    if (rc == MPQ_OK) rc = check_matrix(Z, dtype, c > 0 ? n : 0, c, ld, "Z");
    if (rc == MPQ_OK && residual_opt) rc = check_matrix(residual_opt, y_dtype, n, c, residual_ld, "residual");
    if (rc == MPQ_OK) rc = check_array(place, n * k, 4, "place");
    if (rc == MPQ_OK) rc = check_array(weights, n * k, 4, "weights");
    if (rc != MPQ_OK || n == 0 || c == 0) return rc;
    mpq::MxCombine q = {};
    q.Y = Y;
    q.dtype = y_dtype;
    q.m = m;
    q.c = c;
    q.ldy = y_ld;
    q.n = n;
    q.place = place;
    q.weights = weights;
    q.k = (int)k;
    q.R = residual_opt;
    q.ldr = residual_ld;
    q.Z = Z;
    q.z_dtype = dtype;
    q.ldz = ld;
    return done(mpq::launch_mx_combine(q, (hipStream_t)stream), hipSuccess, "mx combine launch");
}

}  // extern "C"
