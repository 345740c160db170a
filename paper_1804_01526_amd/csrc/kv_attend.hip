// Softmax attention over the 4-bit cache for few queries per key head (single tokens, drafted tokens), and the accumulation of
// attention weights.
//
// A wave holds 16 queries of one key head (the tokens' queries of the heads that share it) and walks over keys 32 at a time:
// scores S^T = K Q^T, so that a lane has one query's scores of 16 keys, the running maximum and sum of the softmax, and
// O^T += V^T P^T, whose second operand is the scores' own register layout: nothing passes through LDS between the two
// products.  The contraction of the first runs over dimensions, and a key's exponents are applied when its nibbles become bf16
// numbers; the contraction of the second runs over keys, whose exponents differ, so they multiply the weights, block of 32
// dimensions by block, and the values enter as integers (n / 4).
#include "kv_cache.h"

namespace hbfp {
namespace {

constexpr int kWaves = 4, kStepKeys = 32;

// a wave's 16 queries as the second operand of S^T = K Q^T: lane c + 16 g has dimensions 32 blk + 8 g .. + 7 of query c
template <int NB, int DT>
__device__ __forceinline__ void load_queries(const Heads &q, int64_t b, int key_head, int group, int row, int rows, int dim, int g,
                                             bool negate, v8bf (&out)[Pieces<DT>::n][NB]) {
    const bool real = row < rows;
    const int t = real ? row / group : 0, h = real ? key_head * group + row % group : 0;
    const int64_t base = b * q.sb + t * q.st + h * q.sh;
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) {
        const int d0 = 32 * blk + 8 * g, n = real ? dim - d0 : 0;
        float x[8];
        load8<DT>(q.data, base + d0, n, x);
        if (negate)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = -x[i];
        uint32_t w[4][Pieces<DT>::n];
#pragma unroll
        for (int i = 0; i < 4; ++i) bf16_pieces2<Pieces<DT>::n>(x[2 * i], x[2 * i + 1], w[i]);
#pragma unroll
        for (int p = 0; p < Pieces<DT>::n; ++p) {
            const v4u r = {w[0][p], w[1][p], w[2][p], w[3][p]};
            out[p][blk] = __builtin_bit_cast(v8bf, r);
        }
    }
}

// scores of 16 keys (rows of the result: keys 4 g + i) from 16 g.. of the key layout
template <int NB, int NP>
__device__ __forceinline__ v4f scores16(const uint32_t (&w)[NB], const uint32_t (&e)[NB], int j, const v8bf (&q)[NP][NB]) {
    v4f s = {0, 0, 0, 0};
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) {
        const v8bf k = key_values(w[blk], conversion_scale(e[blk] >> (8 * j), 0));
#pragma unroll
        for (int p = NP - 1; p >= 0; --p) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[p][blk], s, 0, 0, 0);
    }
    return s;
}

// The words of KS keys and values that a lane needs
template <int NB, int KS>
struct StepWords {
    uint32_t kw[KS / 16][NB], kx[KS / 16][NB], vw[KS / 16][NB], vx[KS / 16][NB];
};
template <int NB, int KS>
__device__ __forceinline__ void request_step(const uint8_t *k, const uint8_t *ke, const uint8_t *v, const uint8_t *ve, int key0, int c, int g,
                                             StepWords<NB, KS> &r) {
#pragma unroll
    for (int t = 0; t < KS / 16; ++t) {
        const uint32_t key = key0 + 16 * t + c, group = (key0 + 16 * t) / 4;
        load_words<NB>(k + (key * 16 + g * 4) * NB, r.kw[t]);
        load_words<NB>(ke + (group + c / 4) * 4 * NB, r.kx[t]);
    }
#pragma unroll
    for (int t = 0; t < KS / 16; ++t) {
        const uint32_t group = (key0 + 16 * t) / 4 + g;
        load_words<NB>(v + (group * 64 + c * 4) * NB, r.vw[t]);
        load_words<NB>(ve + group * 4 * NB, r.vx[t]);
    }
}

// One step of KS keys from key0 on.  MASK: some of the wave's queries do not see all of them.
template <int NB, int NP, int NW, int KS, bool MASK>
__device__ __forceinline__ void attend_step(const StepWords<NB, KS> &r, int key0, int limit, float scale2, int c, int g,
                                            const v8bf (&q)[NP][NB], v4f (&o)[2 * NB], float &m, float &l) {
    constexpr int T = KS / 16;
    const auto &kw = r.kw, &kx = r.kx, &vw = r.vw, &vx = r.vx;
    float s[T][4];
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const v4f x = scores16<NB, NP>(kw[t], kx[t], c & 3, q);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[t][i] = MASK ? key0 + 16 * t + 4 * g + i < limit ? x[i] : -INFINITY : x[i];
            top = fmaxf(top, s[t][i]);
        }
    }
    // m is the largest score up to a factor of 2^kSlack in its exponential: new largest scores are frequent among 16 queries, such
    // that are that much larger are not after the first steps
    top = max_over_rows(top) * scale2;
    if (__any(top > m + kSlack)) {
        const float m_new = fmaxf(m, top), shrink = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
        l *= shrink;
#pragma unroll
        for (int i = 0; i < 2 * NB; ++i) o[i] *= shrink;
        m = m_new;
    }
    const float from = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], scale2, -from));
            l += s[t][i];
        }
#pragma unroll
    for (int u = 0; u < T; u += 2)
#pragma unroll
        for (int blk = 0; blk < NB; ++blk) {
            uint32_t w[4][NW];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; i += 2)             // (a weight of 0 stays 0 whatever the exponent byte)
                    bf16_pieces2<NW>(times_exponent(s[u + t][i], vx[u + t][blk], i), times_exponent(s[u + t][i + 1], vx[u + t][blk], i + 1),
                                     w[2 * t + i / 2]);
            const uint32_t lo0 = fp8_of_low(vw[u][blk]), lo1 = fp8_of_low(vw[u + 1][blk]);
            const uint32_t hi0 = fp8_of_high(vw[u][blk]), hi1 = fp8_of_high(vw[u + 1][blk]);
            const v4u lo = {bf16_pair<false>(lo0, 1.0f), bf16_pair<true>(lo0, 1.0f), bf16_pair<false>(lo1, 1.0f), bf16_pair<true>(lo1, 1.0f)};
            const v4u hi = {bf16_pair<false>(hi0, 1.0f), bf16_pair<true>(hi0, 1.0f), bf16_pair<false>(hi1, 1.0f), bf16_pair<true>(hi1, 1.0f)};
#pragma unroll
            for (int p = NW - 1; p >= 0; --p) {
                const v4u pw = {w[0][p], w[1][p], w[2][p], w[3][p]};
                const v8bf pb = __builtin_bit_cast(v8bf, pw);
                o[2 * blk] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, lo), pb, o[2 * blk], 0, 0, 0);
                o[2 * blk + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, hi), pb, o[2 * blk + 1], 0, 0, 0);
            }
        }
}

// Bound by the vector instructions that turn nibbles and weights into numbers, 70 to 80 % of a busy compute unit's cycles: with four
// queries a head only a quarter of every tile of 16 is real, and the conversion is the same as for all.  16 heads (4 of keys) of 128 over
// 200001 tokens, FP16: 109 MB in 37 us, 3.0 TB/s; 32 conversations of 128 to 8192 tokens, 32 heads (8 of keys), bf16: 62 MB in 34 us,
// 1.8 TB/s (weights as one piece: 30), the compute units busy half of the time because lengths differ.
// A workgroup's four waves take the steps of a chunk in turn and join their results in LDS; with several chunks the joined
// ones go to the workspace, and cache_join_kernel joins those.
template <int NB, int DT>
__global__ __launch_bounds__(64 * kWaves, NB <= 4 ? 2 : 1) void cache_attend_kernel(const SplitParams p) {
    constexpr int NP = Pieces<DT>::n, NW = Pieces<DT>::weights, KS = kStepKeys, DP = 32 * NB, PITCH = DP + 4;
    extern __shared__ __attribute__((aligned(16))) float lds[];          // [wave][16 queries][PITCH], then [wave][16] max, [wave][16] sum
    const CacheView &cache = p.a.c;
    uint32_t id = blockIdx.x;
    const int tile = (int)(id % p.tiles);
    id /= p.tiles;
    const uint32_t heads = cache.batch * cache.heads;
    const int64_t bh = id % heads;
    const int chunk = (int)(id / heads);
    const int64_t b = bh / cache.heads;
    const int key_head = (int)(bh % cache.heads);
    const int length = p.a.lengths[b];
    const int bound = p.a.longest;
    const int last_row = 16 * tile + 15 < p.rows ? 16 * tile + 15 : p.rows - 1;
    const int most = visible(length, p.a.tokens, p.a.group, last_row, p.a.causal, bound);
    const int least = visible(length, p.a.tokens, p.a.group, 16 * tile, p.a.causal, bound);
    const int begin = chunk * p.chunk, end = most < begin + p.chunk ? most : begin + p.chunk;
    if (begin >= end && p.chunks > 1) return;                 // the whole workgroup, before any barrier

    const int t = threadIdx.x, lane = t & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int row = 16 * tile + c;
    const int limit = row < p.rows ? visible(length, p.a.tokens, p.a.group, row, p.a.causal, bound) : 0;
    v8bf q[NP][NB];
    load_queries<NB, DT>(p.a.q, b, key_head, p.a.group, row, p.rows, cache.dim, g, p.a.scale < 0.0f, q);   // (scale2 is the magnitude)
    const uint8_t *k = cache.k + bh * cache.head_codes, *v = cache.v + bh * cache.head_codes;
    const uint8_t *ke = cache.ke + bh * cache.head_exps, *ve = cache.ve + bh * cache.head_exps;
    v4f o[2 * NB];
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) o[i] = v4f{0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f;
    // a step's words are on their way while the step before it is computed
    constexpr int STRIDE = kWaves * KS;
    StepWords<NB, KS> r0, r1;
    int key0 = begin + wave * KS;
    const auto request = [&](int at, StepWords<NB, KS> &r) {
        if (at < end) request_step<NB, KS>(k, ke, v, ve, at, c, g, r);
    };
    request(key0, r0);
    for (; key0 + STRIDE < end && key0 + STRIDE + KS <= least; key0 += 2 * STRIDE) {
        request(key0 + STRIDE, r1);
        attend_step<NB, NP, NW, KS, false>(r0, key0, limit, p.scale2, c, g, q, o, m, l);
        request(key0 + 2 * STRIDE, r0);
        attend_step<NB, NP, NW, KS, false>(r1, key0 + STRIDE, limit, p.scale2, c, g, q, o, m, l);
    }
    for (; key0 < end; key0 += STRIDE) {
        attend_step<NB, NP, NW, KS, true>(r0, key0, limit, p.scale2, c, g, q, o, m, l);
        request(key0 + STRIDE, r0);
    }
    l = sum_over_rows(l);
    float *const lds_m = lds + kWaves * 16 * PITCH, *const lds_l = lds_m + kWaves * 16;
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) *reinterpret_cast<v4f *>(lds + (wave * 16 + c) * PITCH + 16 * i + 4 * g) = o[i];
    if (g == 0) lds_m[wave * 16 + c] = m, lds_l[wave * 16 + c] = l;
    __syncthreads();
    const int rows_here = p.rows - 16 * tile < 16 ? p.rows - 16 * tile : 16;
    for (int i = t; i < rows_here * (DP / 4); i += 64 * kWaves) {
        const int r = i / (DP / 4), d = 4 * (i % (DP / 4));
        float top = lds_m[r];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, lds_m[w * 16 + r]);
        const float from = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f;
        v4f acc = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(lds_m[w * 16 + r] - from);
            sum += f * lds_l[w * 16 + r];
            acc += f * *reinterpret_cast<const v4f *>(lds + (w * 16 + r) * PITCH + d);
        }
        const int grow = 16 * tile + r;
        if (p.chunks > 1) {
            const int64_t slot = (bh * p.chunks + chunk) * p.rows + grow;
            *reinterpret_cast<v4f *>(p.o + slot * DP + d) = acc;
            if (d == 0) p.ml[2 * slot] = top, p.ml[2 * slot + 1] = sum;
        } else {
            const int tok = grow / p.a.group, h = key_head * p.a.group + grow % p.a.group;
            const float inv = sum == 0.0f ? 0.0f : kUp / sum;
            const float out4[4] = {acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
            store4<DT>(p.a.out.data, b * p.a.out.sb + tok * p.a.out.st + h * p.a.out.sh + d, cache.dim - d, out4);
            if (d == 0) p.a.lse[(b * p.a.tokens + tok) * p.a.heads + h] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
        }
    }
}

// Joins the chunks of the rows: `parts` groups of 8 nblk threads (four dimensions each) share a row's chunks, each in their order,
// and are joined in theirs.  The largest maximum first, so that no chunk waits for the one before it.  Bound by latency: 5 us for 8
// chunks of 1024 rows, 9.4 us for 224 of 16 rows (391 of them 10.7; chunk
// after chunk by 256 threads 20).
template <int DT, int THREADS>
__global__ __launch_bounds__(THREADS) void cache_join_kernel(const SplitParams p, int parts) {
    __shared__ v4f lds[THREADS];
    __shared__ float lds_l[THREADS];
    const CacheView &cache = p.a.c;
    const int quads = 8 * cache.nblk, per_row = quads * parts, rows_here = THREADS / per_row;
    const int t = threadIdx.x, sub = t / per_row, part = t % per_row / quads, d = 4 * (t % per_row % quads);
    const int64_t at = (int64_t)blockIdx.x * rows_here + sub;
    const bool real = sub < rows_here && at < (int64_t)cache.batch * cache.heads * p.rows;
    const int row = real ? (int)(at % p.rows) : 0;
    const int64_t bh = real ? at / p.rows : 0, b = bh / cache.heads;
    const int key_head = (int)(bh % cache.heads);
    const int end_row = (row / p.tile_rows + 1) * p.tile_rows, last_row = end_row < p.rows ? end_row - 1 : p.rows - 1;
    const int most = visible(p.a.lengths[b], p.a.tokens, p.a.group, last_row, p.a.causal, p.a.longest);
    const int n = real ? (most + p.chunk - 1) / p.chunk : 0;  // chunks that wrote
    const int64_t first = bh * p.chunks * p.rows + row;
    float top = -INFINITY;
#pragma unroll 4
    for (int i = part; i < n; i += parts) top = fmaxf(top, p.ml[2 * (first + (int64_t)i * p.rows)]);
    if (parts > 1) {
        lds_l[t] = top;
        __syncthreads();
        if (sub < rows_here)
            for (int i = 0; i < parts; ++i) top = fmaxf(top, lds_l[sub * per_row + i * quads + d / 4]);
        __syncthreads();
    }
    const float from = top == -INFINITY ? 0.0f : top;
    float l = 0.0f;
    v4f acc = {0, 0, 0, 0};
#pragma unroll 4
    for (int i = part; i < n; i += parts) {
        const int64_t slot = first + (int64_t)i * p.rows;
        const float f = __builtin_amdgcn_exp2f(p.ml[2 * slot] - from);
        l += f * p.ml[2 * slot + 1];
        acc += f * *reinterpret_cast<const v4f *>(p.o + slot * 4 * quads + d);
    }
    if (parts > 1) {
        lds[t] = acc;
        lds_l[t] = l;
        __syncthreads();
        if (part != 0) return;
        for (int i = 1; i < parts; ++i) {
            if (sub < rows_here) {
                acc += lds[t + i * quads];
                l += lds_l[t + i * quads];
            }
        }
    }
    if (!real) return;
    const int tok = row / p.a.group, h = key_head * p.a.group + row % p.a.group;
    const float inv = l == 0.0f ? 0.0f : kUp / l;
    const float r[4] = {acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
    store4<DT>(p.a.out.data, b * p.a.out.sb + tok * p.a.out.st + h * p.a.out.sh + d, cache.dim - d, r);
    if (d == 0) p.a.lse[(b * p.a.tokens + tok) * p.a.heads + h] = l == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kLn2;
}
template <int DT>
int launch_join(const SplitParams &p, hipStream_t s) {
    const int quads = 8 * p.a.c.nblk, threads = p.chunks > 64 ? 1024 : 256, most = threads / quads;
    const int parts = p.chunks <= 4 ? 1 : (int)ceil_div(p.chunks, 4) < most ? (int)ceil_div(p.chunks, 4) : most;
    const int64_t wgs = ceil_div((int64_t)p.a.c.batch * p.a.c.heads * p.rows, threads / (quads * parts));
    if (wgs > 0x7fffffff) return HBFP_ERR_ARG;
    if (threads == 1024) hipLaunchKernelGGL((cache_join_kernel<DT, 1024>), dim3((unsigned)wgs), dim3(1024), 0, s, p, parts);
    else hipLaunchKernelGGL((cache_join_kernel<DT, 256>), dim3((unsigned)wgs), dim3(256), 0, s, p, parts);
    return launch_status();
}

// Chunks of keys: enough workgroups to fill the chip several times over, none shorter than a step of its four waves.  Several
// conversations may differ in length, which the host does not know: they get twice as many, so that the longest does not hold the last
// workgroups alone, and equal ones pay for that.  us, joining included, with 1024, 1536, 2048 and 4096 of them, 128 dimensions.  One of 200001
// tokens, 16 heads (4 of keys) 43.4, 42.3, 45.8, 53.7, 32 heads (8 of keys) over 8192 12.2, 12.3, 12.3, 12.3.  Different lengths, 32 heads: 16
// of 128 to 8192 31.6, 27.1, 31.9, 33.3, 32 of them 52.2, 40.1, 40.1, 41.9, another 32 (a whole step from cold caches) 1536 46.4, 2048
// 43.0.  Equal ones: 2 of 100000, 16 heads 40.2, 40.1, 43.0, 48.4; 32 heads, 8 of 8192 26.5, 29.9, 30.0, 40.0, 32 of 4096 40.4, 40.8,
// 42.9, 51.2
SplitParams split_of(const AttendArgs &a) {
    SplitParams p = {};
    p.a = a;
    p.rows = a.tokens * a.group;
    const bool prompt = cache_prompt_ok(a);
    p.tile_rows = prompt ? (int32_t)cache_prompt_rows(a) : 16;
    p.tiles = (int32_t)ceil_div(p.rows, p.tile_rows);
    p.scale2 = a.scale * kLog2e;
    p.scale2 = p.scale2 == 0.0f ? 1.2e-38f : p.scale2 < 0.0f ? -p.scale2 : p.scale2;     // (0 times a masked -infinity is no number)
    const int64_t heads = (int64_t)a.c.batch * a.c.heads * p.tiles;
    const int64_t step = prompt ? 512 : kWaves * kStepKeys;
    const int64_t want = ceil_div(prompt ? 512 : a.c.batch == 1 ? 1024 : 2048, heads);
    p.chunk = (int32_t)round_up(ceil_div(a.longest, want), step);
    p.chunks = (int32_t)ceil_div(a.longest, p.chunk);
    return p;
}
size_t split_floats(const SplitParams &p) {
    return p.chunks > 1 ? (size_t)p.a.c.batch * p.a.c.heads * p.chunks * p.rows * (size_t)(2 + 32 * p.a.c.nblk) : 0;
}

template <int NB, int DT>
int launch_split(const SplitParams &p, hipStream_t s) {
    static std::atomic<bool> configured;
    constexpr int bytes = (kWaves * 16 * (32 * NB + 4) + 2 * kWaves * 16) * 4;
    void (*const kernel)(SplitParams) = &cache_attend_kernel<NB, DT>;
    if (allow_dynamic_lds(configured, reinterpret_cast<const void *>(kernel), bytes) != HBFP_OK) return HBFP_ERR_LAUNCH;
    hipLaunchKernelGGL(kernel, dim3(p.wgs), dim3(64 * kWaves), bytes, s, p);
    return launch_status();
}
template <int DT>
int launch_split_of(const SplitParams &p, hipStream_t s) {
    switch (p.a.c.nblk) {
        case 1: return launch_split<1, DT>(p, s);
        case 2: return launch_split<2, DT>(p, s);
        case 3: return launch_split<3, DT>(p, s);
        case 4: return launch_split<4, DT>(p, s);
        case 5: return launch_split<5, DT>(p, s);
        case 6: return launch_split<6, DT>(p, s);
        case 7: return launch_split<7, DT>(p, s);
        default: return launch_split<8, DT>(p, s);
    }
}

// ---- accumulated weights.  A wave turns 64 keys into bf16 numbers once and meets every query of the key head with them; a
// lane's sums over its query columns are exchanged over the 16 lanes at the end.  A wave walks over kWeighGroups such groups, the
// words of the next on their way; queries that fit one tile stay in registers.  Bound by latency (half of the waves' time waits for memory): 16
// conversations of 128 to 8192 tokens, 32 heads (8 of keys) of 128, 45 MB in 26 us, 1.8 TB/s (a group a wave: 48 us).
constexpr int kWeighGroups = 4;
struct WeighParams {
    WeighArgs a;
    int32_t rows, tiles;
    float scale2;
    int64_t units;               // batch * heads * walks
};

// of 2 HALF values the lanes c with that bit keep the upper half and the others the lower, joined with those of lane c ^ HALF (a function
// of its own: as a loop over the halves it kept the array in registers only by comparing every index, 50 us instead of 14)
template <int HALF>
__device__ __forceinline__ void halve(float (&sum)[16], int c) {
    const bool upper = (c & HALF) != 0;
#pragma unroll
    for (int i = 0; i < HALF; ++i) {
        const float mine = upper ? sum[i + HALF] : sum[i], give = upper ? sum[i] : sum[i + HALF];
        sum[i] = mine + __shfl_xor(give, HALF);
    }
}

template <int NB, int DT>
__global__ __launch_bounds__(256) void cache_weigh_kernel(const WeighParams p) {
    constexpr int NP = Pieces<DT>::n;
    const CacheView &cache = p.a.c;
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (unit >= p.units) return;
    const int64_t heads = (int64_t)cache.batch * cache.heads, bh = unit % heads;
    const int begin = (int)(unit / heads) * 64 * kWeighGroups, bound = cache.capacity;
    const int end = begin + 64 * kWeighGroups < bound ? begin + 64 * kWeighGroups : bound;
    const int64_t b = bh / cache.heads;
    const int key_head = (int)(bh % cache.heads);
    const int length = p.a.lengths[b];
    const int held = visible(length, p.a.tokens, p.a.group, 0, 0, bound);
    // this lane's result of a group: value index c of its 16, key 16 (c / 4) + 4 g + c % 4
    const int own = 16 * (c >> 2) + 4 * g + (c & 3);
    float *const w_out = p.a.w_out + bh * p.a.ld;
    const float *const w_in = p.a.w_in + bh * p.a.ld;
    const uint8_t *k = cache.k + bh * cache.head_codes, *ke = cache.ke + bh * cache.head_exps;
    v8bf q[NP][NB];
    int limit = 0;
    float lse2 = 0.0f;
    const auto load_tile = [&](int tile) {
        const int row = 16 * tile + c;
        limit = 0;
        if (row < p.rows) {
            limit = visible(length, p.a.tokens, p.a.group, row, p.a.causal, p.a.longest);
            lse2 = p.a.lse[(b * p.a.tokens + row / p.a.group) * p.a.heads + key_head * p.a.group + row % p.a.group] * kLog2e;
        }
        load_queries<NB, DT>(p.a.q, b, key_head, p.a.group, row, p.rows, cache.dim, g, false, q);
    };
    uint32_t w[4][NB], e[4][NB];
    float before = 0.0f;
    const auto request = [&](int key0) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            load_words<NB>(k + (uint32_t)((key0 + 16 * t + c) * 16 + g * 4) * NB, w[t]);
            load_words<NB>(ke + (uint32_t)((key0 + 16 * t) / 4 + c / 4) * 4 * NB, e[t]);
        }
        before = key0 + own < held ? w_in[key0 + own] : 0.0f;
    };
    int key0 = begin;
    if (key0 < held) {
        request(key0);
        if (p.tiles == 1) load_tile(0);
    }
    for (; key0 < end && key0 < held; key0 += 64) {
        v8bf kf[4][NB];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int blk = 0; blk < NB; ++blk) kf[t][blk] = key_values(w[t][blk], conversion_scale(e[t][blk] >> (8 * (c & 3)), 0));
        const float old = before;
        if (key0 + 64 < end && key0 + 64 < held) request(key0 + 64);
        float sum[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[i] = 0.0f;
        for (int tile = 0; tile < p.tiles; ++tile) {
            const int last_row = 16 * tile + 15 < p.rows ? 16 * tile + 15 : p.rows - 1;
            if (visible(length, p.a.tokens, p.a.group, last_row, p.a.causal, p.a.longest) <= key0) continue;
            if (p.tiles > 1) load_tile(tile);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                v4f s = {0, 0, 0, 0};
#pragma unroll
                for (int blk = 0; blk < NB; ++blk)
#pragma unroll
                    for (int i = NP - 1; i >= 0; --i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t][blk], q[i][blk], s, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = __builtin_amdgcn_exp2f(s[i] * p.scale2 - lse2);
                    sum[4 * t + i] += key0 + 16 * t + 4 * g + i < limit ? x : 0.0f;
                }
            }
        }
        // over the 16 lanes of a row: each exchange halves the values a lane carries
        halve<8>(sum, c);
        halve<4>(sum, c);
        halve<2>(sum, c);
        halve<1>(sum, c);
        if (key0 + own < bound) w_out[key0 + own] = key0 + own < held ? p.a.decay * old + sum[0] : 0.0f;
    }
    for (; key0 < end; key0 += 64)
        if (key0 + lane < bound) w_out[key0 + lane] = 0.0f;
}

template <int DT>
int launch_weigh_of(const WeighParams &p, hipStream_t s) {
    static void (*const kernels[8])(WeighParams) = {&cache_weigh_kernel<1, DT>, &cache_weigh_kernel<2, DT>, &cache_weigh_kernel<3, DT>,
                                                    &cache_weigh_kernel<4, DT>, &cache_weigh_kernel<5, DT>, &cache_weigh_kernel<6, DT>,
                                                    &cache_weigh_kernel<7, DT>, &cache_weigh_kernel<8, DT>};
    const int64_t wgs = ceil_div(p.units, 4);
    if (wgs > 0x7fffffff) return HBFP_ERR_ARG;
    hipLaunchKernelGGL(kernels[p.a.c.nblk - 1], dim3((unsigned)wgs), dim3(256), 0, s, p);
    return launch_status();
}

}  // namespace

size_t cache_attend_workspace(const AttendArgs &a) {
    return split_floats(split_of(a)) * 4;
}

int launch_cache_attend(const AttendArgs &a, int dtype, hipStream_t s) {
    SplitParams p = split_of(a);
    const int64_t heads = (int64_t)a.c.batch * a.c.heads;
    const int64_t wgs = heads * p.tiles * p.chunks, rows = heads * p.rows;
    if (wgs > 0x7fffffff || rows > 0x7fffffff) return HBFP_ERR_ARG;
    p.wgs = (uint32_t)wgs;
    p.o = a.ws;
    p.ml = a.ws ? a.ws + heads * p.chunks * p.rows * 32 * a.c.nblk : nullptr;
    int rc = cache_prompt_ok(a) ? launch_cache_prompt(p, dtype, s)
             : dtype == HBFP_F32 ? launch_split_of<HBFP_F32>(p, s) : dtype == HBFP_BF16 ? launch_split_of<HBFP_BF16>(p, s) : launch_split_of<HBFP_F16>(p, s);
    if (rc != HBFP_OK || p.chunks == 1) return rc;
    return dtype == HBFP_F32 ? launch_join<HBFP_F32>(p, s) : dtype == HBFP_BF16 ? launch_join<HBFP_BF16>(p, s) : launch_join<HBFP_F16>(p, s);
}

int launch_cache_weigh(const WeighArgs &a, int dtype, hipStream_t s) {
    WeighParams p = {};
    p.a = a;
    p.rows = a.tokens * a.group;
    p.tiles = (int32_t)ceil_div(p.rows, 16);
    p.scale2 = a.scale * kLog2e;
    p.units = (int64_t)a.c.batch * a.c.heads * ceil_div(a.c.capacity, 64 * kWeighGroups);
    return dtype == HBFP_F32 ? launch_weigh_of<HBFP_F32>(p, s) : dtype == HBFP_BF16 ? launch_weigh_of<HBFP_BF16>(p, s) : launch_weigh_of<HBFP_F16>(p, s);
}

}  // namespace hbfp
