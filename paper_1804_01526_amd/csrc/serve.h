// Launchers of the serving operators (4-bit cache, products with row scales).  Nothing here is part of the public ABI.
#pragma once
#include "hbfp_internal.h"

namespace hbfp {

// One call's tensor [batch][tokens][heads][dim]
struct Heads {
    void *data;
    int64_t sb, st, sh;
};

struct CacheView {
    uint8_t *k, *v, *ke, *ve;
    int64_t head_codes, head_exps;   // bytes of one (batch, head)
    int32_t batch, heads, capacity, dim, nblk, slots;
};

struct AttendArgs {
    CacheView c;
    Heads q, out;
    const int32_t *lengths;
    float *lse;
    int32_t tokens, heads, group;    // group: query heads of one key head
    int32_t longest, causal;
    float scale;
    float *ws;
};

// An attention call as its kernels see it: query rows (token, head of the group) of every key head in tiles, keys in chunks
struct SplitParams {
    AttendArgs a;
    float *ml, *o;            // partial results, [batch * heads][chunks][rows]: (max, sum) and [32 nblk]
    int32_t rows, tile_rows, tiles, chunk, chunks;
    float scale2;             // scale * log2(e)
    uint32_t wgs;
};

// kv_store.hip
int launch_cache_append(const CacheView &c, const Heads &k, const Heads &v, int dtype, int64_t tokens, const int32_t *lengths,
                        void *k_values, void *v_values, hipStream_t s);
int launch_cache_read(const CacheView &c, const int32_t *lengths, int dtype, void *k, void *v, hipStream_t s);
int launch_cache_evict(const CacheView &src, const float *w, int64_t ld, const int32_t *lengths, int64_t keep, int64_t recent,
                       const CacheView &dst, float *w_out, int64_t ld_out, int32_t *kept, int32_t *lengths_out, hipStream_t s);
// kv_attend.hip
size_t cache_attend_workspace(const AttendArgs &a);
int launch_cache_attend(const AttendArgs &a, int dtype, hipStream_t s);
// kv_prompt.hip: many rows a key head
bool cache_prompt_ok(const AttendArgs &a);
int64_t cache_prompt_rows(const AttendArgs &a);
int launch_cache_prompt(const SplitParams &p, int dtype, hipStream_t s);
struct WeighArgs {
    CacheView c;
    Heads q;
    const int32_t *lengths;
    const float *lse, *w_in;
    float *w_out;
    int64_t ld;
    int32_t tokens, heads, group, causal, longest;
    float scale, decay;
};
int launch_cache_weigh(const WeighArgs &a, int dtype, hipStream_t s);

// gemm_rows.hip
struct RowsArgs {
    const int8_t *a, *b;
    const float *sa, *sb, *bias;
    void *y;
    int64_t M, N, K, kpad, ldy;
    int32_t dtype;
};
int launch_quant_rows(const void *src, int dtype, int64_t rows, int64_t cols, int64_t ld, int8_t *codes, float *scales, hipStream_t s);
size_t gemm_rows_workspace(int64_t M, int64_t N, int64_t kpad);
int launch_gemm_rows(const RowsArgs &a, void *workspace, hipStream_t s);
// x converted inside the product: one or two tokens whose codes fit into LDS; a.a and a.sa are not read
bool linear_fused_ok(int64_t M, int64_t N, int64_t kpad);
int launch_linear_fused(const RowsArgs &a, const void *x, int64_t ldx, hipStream_t s);

}  // namespace hbfp
