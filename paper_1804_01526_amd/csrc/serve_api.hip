// Host side of the serving operators: geometry, argument validation, dispatch.  Every check runs before anything is queued.
#include <string.h>

#include "serve.h"

using namespace hbfp;

namespace {

bool known_type(int dtype) { return dtype == HBFP_F32 || dtype == HBFP_BF16 || dtype == HBFP_F16; }
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
bool overlap(const void *p, uint64_t np, const void *q, uint64_t nq) {
    return (uintptr_t)p < (uintptr_t)q + nq && (uintptr_t)q < (uintptr_t)p + np;
}

int check_cache(const hbfp_cache *c) {
    if (!c) return HBFP_ERR_ARG;
    hbfp_cache p;
    if (hbfp_cache_plan(c->batch, c->heads, c->capacity, c->dim, &p) != HBFP_OK) return HBFP_ERR_LAYOUT;
    if (p.slots != c->slots || p.nblk != c->nblk || p.code_bytes != c->code_bytes || p.exp_bytes != c->exp_bytes) return HBFP_ERR_LAYOUT;
    if (!c->k || !c->v || !c->k_exps || !c->v_exps) return HBFP_ERR_ARG;
    if (((uintptr_t)c->k | (uintptr_t)c->v | (uintptr_t)c->k_exps | (uintptr_t)c->v_exps) & 15) return HBFP_ERR_ARG;
    return HBFP_OK;
}

CacheView view_of(const hbfp_cache &c) {
    CacheView v;
    v.k = c.k;
    v.v = c.v;
    v.ke = c.k_exps;
    v.ve = c.v_exps;
    v.head_codes = c.slots * 16 * c.nblk;
    v.head_exps = c.slots * c.nblk;
    v.batch = (int32_t)c.batch;
    v.heads = (int32_t)c.heads;
    v.capacity = (int32_t)c.capacity;
    v.dim = (int32_t)c.dim;
    v.nblk = (int32_t)c.nblk;
    v.slots = (int32_t)c.slots;
    return v;
}

// a tensor [batch][tokens][heads][dim]; outputs may not place two elements at one address
int check_heads(const hbfp_heads *h, int64_t batch, int64_t tokens, int64_t heads, int64_t dim, bool is_output) {
    if (!h || !h->data || h->reserved != 0) return HBFP_ERR_ARG;
    if (!known_type(h->dtype)) return HBFP_ERR_FORMAT;
    if ((uintptr_t)h->data & (h->dtype == HBFP_F32 ? 3 : 1)) return HBFP_ERR_ARG;
    const int64_t lim = (int64_t)1 << 40;
    if (h->stride_batch < 0 || h->stride_token < 0 || h->stride_head < 0) return HBFP_ERR_ARG;
    if (h->stride_batch > lim || h->stride_token > lim || h->stride_head > lim) return HBFP_ERR_ARG;
    if (is_output) {
        // sorted by stride, each must pass over what the ones below it span
        int64_t ext[3] = {batch, tokens, heads}, st[3] = {h->stride_batch, h->stride_token, h->stride_head};
        for (int i = 0; i < 3; ++i)
            for (int j = i + 1; j < 3; ++j)
                if (st[j] < st[i]) {
                    const int64_t e = ext[i], x = st[i];
                    ext[i] = ext[j], st[i] = st[j];
                    ext[j] = e, st[j] = x;
                }
        int64_t span = dim;
        for (int i = 0; i < 3; ++i) {
            if (ext[i] == 1) continue;
            if (st[i] < span) return HBFP_ERR_ARG;
            span += (ext[i] - 1) * st[i];
        }
    }
    return HBFP_OK;
}
Heads heads_of(const hbfp_heads &h) { return {h.data, h.stride_batch, h.stride_token, h.stride_head}; }

// tokens and query heads of a call that reads the cache; the rows of a key head have to fit 31 bits
int check_queries(const hbfp_cache *c, int64_t tokens, int64_t heads) {
    if (tokens <= 0 || heads <= 0 || heads % c->heads != 0 || heads > (1 << 20)) return HBFP_ERR_ARG;
    if (tokens > (((int64_t)1 << 30) / (heads / c->heads))) return HBFP_ERR_ARG;
    return HBFP_OK;
}

int32_t longest_of(const hbfp_cache *c, int64_t longest) { return (int32_t)(longest == 0 || longest > c->capacity ? c->capacity : longest); }

int attend_args(const hbfp_cache *cache, int64_t tokens, int64_t heads, int64_t longest, AttendArgs *a) {
    const int rc = check_queries(cache, tokens, heads);
    if (rc != HBFP_OK) return rc;
    if (longest < 0) return HBFP_ERR_ARG;
    memset(a, 0, sizeof *a);
    a->c = view_of(*cache);
    a->tokens = (int32_t)tokens;
    a->heads = (int32_t)heads;
    a->group = (int32_t)(heads / cache->heads);
    a->longest = longest_of(cache, longest);
    return HBFP_OK;
}

}  // namespace

extern "C" {

int hbfp_cache_plan(int64_t batch, int64_t heads, int64_t capacity, int64_t dim, hbfp_cache *out) {
    if (!out || batch <= 0 || heads <= 0 || capacity <= 0 || dim <= 0) return HBFP_ERR_ARG;
    if (dim > 256) return HBFP_ERR_FORMAT;
    const int64_t nblk = ceil_div(dim, 32), most = (int64_t)1 << 31;
    if (batch >= most || heads > (1 << 20) || batch * heads >= most || capacity > most || round_up(capacity, 64) * 16 * nblk >= most) return HBFP_ERR_FORMAT;
    memset(out, 0, sizeof *out);
    out->batch = batch;
    out->heads = heads;
    out->capacity = capacity;
    out->dim = dim;
    out->slots = round_up(capacity, 64);
    out->nblk = nblk;
    out->code_bytes = (uint64_t)batch * (uint64_t)heads * (uint64_t)(out->slots * 16 * nblk);
    out->exp_bytes = (uint64_t)batch * (uint64_t)heads * (uint64_t)(out->slots * nblk);
    return HBFP_OK;
}

int hbfp_cache_append(const hbfp_cache *cache, const hbfp_heads *k, const hbfp_heads *v, int64_t tokens, const int32_t *lengths,
                      void *k_values, void *v_values, void *stream) {
    int rc = check_cache(cache);
    if (rc != HBFP_OK) return rc;
    if (tokens <= 0 || tokens > ((int64_t)1 << 30) || !lengths || ((uintptr_t)lengths & 3)) return HBFP_ERR_ARG;
    if ((rc = check_heads(k, cache->batch, tokens, cache->heads, cache->dim, false)) != HBFP_OK) return rc;
    if ((rc = check_heads(v, cache->batch, tokens, cache->heads, cache->dim, false)) != HBFP_OK) return rc;
    if (k->dtype != v->dtype) return HBFP_ERR_FORMAT;
    if (((uintptr_t)k_values | (uintptr_t)v_values) & 1) return HBFP_ERR_ARG;
    return launch_cache_append(view_of(*cache), heads_of(*k), heads_of(*v), k->dtype, tokens, lengths, k_values, v_values, (hipStream_t)stream);
}

int hbfp_cache_read(const hbfp_cache *cache, const int32_t *lengths, int dtype, void *k, void *v, void *stream) {
    const int rc = check_cache(cache);
    if (rc != HBFP_OK) return rc;
    if (dtype != HBFP_F32 && dtype != HBFP_BF16) return HBFP_ERR_FORMAT;
    if (!lengths || ((uintptr_t)lengths & 3) || (!k && !v)) return HBFP_ERR_ARG;
    if (((uintptr_t)k | (uintptr_t)v) & (dtype == HBFP_F32 ? 3 : 1)) return HBFP_ERR_ARG;
    return launch_cache_read(view_of(*cache), lengths, dtype, k, v, (hipStream_t)stream);
}

int hbfp_cache_attend_workspace(const hbfp_cache *cache, int64_t tokens, int64_t heads, int dtype, int64_t longest, size_t *bytes) {
    if (!cache || !bytes) return HBFP_ERR_ARG;
    hbfp_cache plan;
    if (hbfp_cache_plan(cache->batch, cache->heads, cache->capacity, cache->dim, &plan) != HBFP_OK) return HBFP_ERR_LAYOUT;
    if (!known_type(dtype)) return HBFP_ERR_FORMAT;
    AttendArgs a;
    const int rc = attend_args(&plan, tokens, heads, longest, &a);
    if (rc != HBFP_OK) return rc;
    *bytes = align256(cache_attend_workspace(a));
    return HBFP_OK;
}

int hbfp_cache_attend(const hbfp_cache *cache, const hbfp_heads *q, int64_t tokens, int64_t heads, const int32_t *lengths,
                      int64_t longest, float scale, int causal, const hbfp_heads *out, float *lse, void *workspace, size_t ws_bytes,
                      void *stream) {
    int rc = check_cache(cache);
    if (rc != HBFP_OK) return rc;
    AttendArgs a;
    if ((rc = attend_args(cache, tokens, heads, longest, &a)) != HBFP_OK) return rc;
    if ((rc = check_heads(q, cache->batch, tokens, heads, cache->dim, false)) != HBFP_OK) return rc;
    if ((rc = check_heads(out, cache->batch, tokens, heads, cache->dim, true)) != HBFP_OK) return rc;
    if (q->dtype != out->dtype) return HBFP_ERR_FORMAT;
    if (!lengths || !lse || (((uintptr_t)lengths | (uintptr_t)lse) & 3) || (causal != 0 && causal != 1)) return HBFP_ERR_ARG;
    a.q = heads_of(*q);
    a.out = heads_of(*out);
    a.lengths = lengths;
    a.lse = lse;
    a.causal = causal;
    a.scale = scale;
    const size_t need = align256(cache_attend_workspace(a));
    if (need && (!workspace || ws_bytes < need || ((uintptr_t)workspace & 255))) return HBFP_ERR_WORKSPACE;
    a.ws = need ? (float *)workspace : nullptr;
    return launch_cache_attend(a, q->dtype, (hipStream_t)stream);
}

int hbfp_cache_weigh_longest(const hbfp_cache *cache, const hbfp_heads *q, int64_t tokens, int64_t heads, const int32_t *lengths,
                             int64_t longest, float scale, int causal, const float *lse, float decay, const float *w_in, float *w_out,
                             int64_t ld, void *stream) {
    int rc = check_cache(cache);
    if (rc != HBFP_OK) return rc;
    if ((rc = check_queries(cache, tokens, heads)) != HBFP_OK) return rc;
    if (longest < 0) return HBFP_ERR_ARG;
    if ((rc = check_heads(q, cache->batch, tokens, heads, cache->dim, false)) != HBFP_OK) return rc;
    if (!lengths || !lse || !w_in || !w_out || ld < cache->capacity || (causal != 0 && causal != 1)) return HBFP_ERR_ARG;
    if (((uintptr_t)lengths | (uintptr_t)lse | (uintptr_t)w_in | (uintptr_t)w_out) & 3) return HBFP_ERR_ARG;
    // in place, or apart: anything between would read what it has written
    const uint64_t span = 4 * ((uint64_t)(cache->batch * cache->heads - 1) * (uint64_t)ld + (uint64_t)cache->capacity);
    if (w_in != w_out && overlap(w_in, span, w_out, span)) return HBFP_ERR_ARG;
    WeighArgs a = {view_of(*cache), heads_of(*q), lengths, lse, w_in, w_out, ld, (int32_t)tokens, (int32_t)heads, (int32_t)(heads / cache->heads),
                   causal, longest_of(cache, longest), scale, decay};
    return launch_cache_weigh(a, q->dtype, (hipStream_t)stream);
}

int hbfp_cache_weigh(const hbfp_cache *cache, const hbfp_heads *q, int64_t tokens, int64_t heads, const int32_t *lengths, float scale,
                     int causal, const float *lse, float decay, const float *w_in, float *w_out, int64_t ld, void *stream) {
    return hbfp_cache_weigh_longest(cache, q, tokens, heads, lengths, 0, scale, causal, lse, decay, w_in, w_out, ld, stream);
}

int hbfp_cache_evict(const hbfp_cache *src, const float *w, int64_t ld, const int32_t *lengths, int64_t keep, int64_t recent,
                     const hbfp_cache *dst, float *w_out, int64_t ld_out, int32_t *kept, int32_t *lengths_out, void *stream) {
    int rc = check_cache(src);
    if (rc != HBFP_OK) return rc;
    if ((rc = check_cache(dst)) != HBFP_OK) return rc;
    if (src->batch != dst->batch || src->heads != dst->heads || src->dim != dst->dim) return HBFP_ERR_LAYOUT;
    if (!w || !lengths || !w_out || !kept || !lengths_out || keep <= 0 || recent < 0) return HBFP_ERR_ARG;
    if (((uintptr_t)w | (uintptr_t)lengths | (uintptr_t)w_out | (uintptr_t)kept | (uintptr_t)lengths_out) & 3) return HBFP_ERR_ARG;
    if (keep > dst->capacity || ld < src->capacity || ld_out < dst->capacity) return HBFP_ERR_ARG;
    const int64_t heads = src->batch * src->heads;
    if (recent > keep) recent = keep;
    const void *in[6] = {src->k, src->v, src->k_exps, src->v_exps, w, lengths};
    const uint64_t in_bytes[6] = {src->code_bytes, src->code_bytes, src->exp_bytes, src->exp_bytes,
                                  4 * ((uint64_t)(heads - 1) * (uint64_t)ld + (uint64_t)src->capacity), 4 * (uint64_t)src->batch};
    const void *out[7] = {dst->k, dst->v, dst->k_exps, dst->v_exps, w_out, kept, lengths_out};
    const uint64_t out_bytes[7] = {dst->code_bytes, dst->code_bytes, dst->exp_bytes, dst->exp_bytes,
                                   4 * ((uint64_t)(heads - 1) * (uint64_t)ld_out + (uint64_t)dst->capacity), 4 * (uint64_t)heads * (uint64_t)keep,
                                   4 * (uint64_t)src->batch};
    for (int i = 0; i < 7; ++i)
        for (int j = 0; j < 6; ++j)
            if (overlap(out[i], out_bytes[i], in[j], in_bytes[j])) return HBFP_ERR_ARG;
    return launch_cache_evict(view_of(*src), w, ld, lengths, keep, recent, view_of(*dst), w_out, ld_out, kept, lengths_out, (hipStream_t)stream);
}

int hbfp_rows_plan(int64_t rows, int64_t cols, int64_t *kpad, size_t *code_bytes) {
    if (rows <= 0 || cols <= 0 || rows > 0x7fffffff || cols > 0x7fffff00) return HBFP_ERR_ARG;
    if (kpad) *kpad = round_up(cols, 128);
    if (code_bytes) *code_bytes = (size_t)rows * (size_t)round_up(cols, 128);
    return HBFP_OK;
}

static int check_matrix(const void *p, int dtype, int64_t rows, int64_t cols, int64_t ld) {
    if (!p || hbfp_rows_plan(rows, cols, nullptr, nullptr) != HBFP_OK || ld < cols) return HBFP_ERR_ARG;
    if (!known_type(dtype)) return HBFP_ERR_FORMAT;
    return (uintptr_t)p & (dtype == HBFP_F32 ? 3 : 1) ? HBFP_ERR_ARG : HBFP_OK;
}

int hbfp_quant_rows(const void *src, int dtype, int64_t rows, int64_t cols, int64_t ld, int8_t *codes, float *scales, void *stream) {
    const int rc = check_matrix(src, dtype, rows, cols, ld);
    if (rc != HBFP_OK) return rc;
    if (!codes || !scales || ((uintptr_t)codes & 15) || ((uintptr_t)scales & 3)) return HBFP_ERR_ARG;
    return launch_quant_rows(src, dtype, rows, cols, ld, codes, scales, (hipStream_t)stream);
}

static int check_product(int64_t M, int64_t N, int64_t K) {
    if (M <= 0 || N <= 0 || K <= 0 || M > 0x7fffffff || N > 0x7fffffff) return HBFP_ERR_ARG;
    return K > 133144 ? HBFP_ERR_RANGE : HBFP_OK;               // 133144 * 127^2 < 2^31
}

int hbfp_gemm_rows_workspace(int64_t M, int64_t N, int64_t K, size_t *bytes) {
    const int rc = check_product(M, N, K);
    if (rc != HBFP_OK || !bytes) return rc != HBFP_OK ? rc : HBFP_ERR_ARG;
    *bytes = align256(gemm_rows_workspace(M, N, round_up(K, 128)));
    return HBFP_OK;
}

int hbfp_gemm_rows(const int8_t *a, const float *a_scales, const int8_t *b, const float *b_scales, const float *bias, int64_t M,
                   int64_t N, int64_t K, void *y, int dtype, int64_t ldy, void *workspace, size_t ws_bytes, void *stream) {
    int rc = check_product(M, N, K);
    if (rc != HBFP_OK) return rc;
    if (!a || !b || !a_scales || !b_scales || (((uintptr_t)a | (uintptr_t)b) & 15)) return HBFP_ERR_ARG;
    if (((uintptr_t)a_scales | (uintptr_t)b_scales | (uintptr_t)bias) & 3) return HBFP_ERR_ARG;
    if ((rc = check_matrix(y, dtype, M, N, ldy)) != HBFP_OK) return rc;
    const size_t need = align256(gemm_rows_workspace(M, N, round_up(K, 128)));
    if (need && (!workspace || ws_bytes < need || ((uintptr_t)workspace & 255))) return HBFP_ERR_WORKSPACE;
    const RowsArgs r = {a, b, a_scales, b_scales, bias, y, M, N, K, round_up(K, 128), ldy, dtype};
    return launch_gemm_rows(r, workspace, (hipStream_t)stream);
}

int hbfp_linear_i8_workspace(int64_t M, int64_t N, int64_t K, size_t *bytes) {
    const int rc = check_product(M, N, K);
    if (rc != HBFP_OK || !bytes) return rc != HBFP_OK ? rc : HBFP_ERR_ARG;
    const int64_t kpad = round_up(K, 128);
    *bytes = linear_fused_ok(M, N, kpad) ? 0 : align256(gemm_rows_workspace(M, N, kpad)) + align256((size_t)M * kpad) + align256((size_t)M * 4);
    return HBFP_OK;
}

int hbfp_linear_i8(const void *x, int dtype, int64_t M, int64_t K, int64_t ldx, const int8_t *b, const float *b_scales,
                   const float *bias, int64_t N, void *y, int64_t ldy, void *workspace, size_t ws_bytes, void *stream) {
    size_t need = 0;
    int rc = hbfp_linear_i8_workspace(M, N, K, &need);
    if (rc != HBFP_OK) return rc;
    if ((rc = check_matrix(x, dtype, M, K, ldx)) != HBFP_OK) return rc;
    if ((rc = check_matrix(y, dtype, M, N, ldy)) != HBFP_OK) return rc;
    if (!b || !b_scales || ((uintptr_t)b & 15) || (((uintptr_t)b_scales | (uintptr_t)bias) & 3)) return HBFP_ERR_ARG;
    const int64_t kpad = round_up(K, 128);
    if (linear_fused_ok(M, N, kpad)) {
        // every workgroup reads all of x for itself, while others store their part of y
        const int64_t size = dtype == HBFP_F32 ? 4 : 2;
        for (int64_t i = 0; i < M; ++i)
            for (int64_t j = 0; j < M; ++j)
                if (overlap((const uint8_t *)y + i * ldy * size, N * size, (const uint8_t *)x + j * ldx * size, K * size)) return HBFP_ERR_ARG;
        const RowsArgs r = {nullptr, b, nullptr, b_scales, bias, y, M, N, K, kpad, ldy, dtype};
        return launch_linear_fused(r, x, ldx, (hipStream_t)stream);
    }
    if (!workspace || ws_bytes < need || ((uintptr_t)workspace & 255)) return HBFP_ERR_WORKSPACE;
    int8_t *const codes = (int8_t *)workspace;
    float *const scales = (float *)(codes + align256((size_t)M * kpad));
    void *const rest = (uint8_t *)scales + align256((size_t)M * 4);
    if ((rc = launch_quant_rows(x, dtype, M, K, ldx, codes, scales, (hipStream_t)stream)) != HBFP_OK) return rc;
    const RowsArgs r = {codes, b, scales, b_scales, bias, y, M, N, K, kpad, ldy, dtype};
    return launch_gemm_rows(r, rest, (hipStream_t)stream);
}

}  // extern "C"
