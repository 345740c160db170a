// Softmax attention over the 4-bit cache for many queries per key head (prompts, chunks of prompts).
//
// A workgroup of W waves holds 32 W query rows of one key head, 32 a wave, and walks over tiles of 64 keys.  A tile's keys and
// values are turned into bf16 numbers once, exactly, by all its waves together, into LDS: keys as they are, values transposed,
// in the order in which the scores' register layout presents keys.  Then S^T = K Q^T and O^T += V^T P^T as in the kernel for
// few queries, on the 32 x 32 x 16 matrix instruction: a lane holds one query, and its softmax needs one exchange with the lane
// 32 away.  Weights enter the second product as two pieces (bf16, FP16), so it costs twice its operations, and the matrix core
// bounds large prompts.  Two of 2048 tokens over 4096, 32 heads (8 of keys) of 128, causal, bf16: 206 Gflop, 309 on the matrix core, in
// 287 to 300 us (one piece: 225 to 240), 1.03 to 1.08 PFLOP/s of the 1.2 that a large bf16 product reaches; three of 501 tokens, 6 heads
// (2 of keys) of 96, FP16: 22 us, that of the longest of few workgroups, and 4.8 for joining the chunks.
#include "kv_cache.h"

namespace hbfp {
namespace {

struct No { static constexpr bool value = false; };
struct Yes { static constexpr bool value = true; };
constexpr int kTile = 64;                  // keys
constexpr int kValuePitch = kTile * 2 + 16;  // bytes of a row of transposed values: 16 more than its keys, so that rows differ in banks
template <int NB> struct PromptLds {
    static constexpr int kKeyPitch = 64 * NB + 16, kKeys = kTile * kKeyPitch, kValues = 32 * NB * kValuePitch;
    static constexpr int kBytes = 2 * (kKeys + kValues);     // two buffers of keys, two of values
};

// one thread's share of a tile: NB words of a key's row, or NB words of a group of four values, and their exponents
template <int NB>
struct RawItem {
    uint32_t w[NB], e[NB];
};
// two numbers with a scale each: both conversions of the pair, one half of each
template <bool HIGH>
__device__ __forceinline__ uint32_t bf16_pair2(uint32_t fp8, float s0, float s1) {
    return __builtin_amdgcn_perm(bf16_pair<HIGH>(fp8, s1), bf16_pair<HIGH>(fp8, s0), 0x07060100u);
}

// Whether a wave brings keys, values or both of every tile: with eight waves the first four bring the keys (an item of 64 threads
// each) and the others the values, with fewer every wave brings both.
enum { kBringKeys = 1, kBringValues = 2 };

// The walk of one wave over the tiles of its workgroup.  It is pipelined by one tile: while the scores of a tile become weights
// on the vector unit, the matrix core computes the scores of the next, and while it multiplies the weights with the values, the
// vector unit converts what is to come.  So iteration i reads keys i + 1 and values i, and writes keys i + 2 and values i + 1,
// each to the buffer of its parity: one barrier an iteration.
template <int NB, int DT, int W, int BRINGS>
__device__ __forceinline__ void prompt_walk(const SplitParams &p, uint8_t *lds, const uint8_t *k, const uint8_t *ke, const uint8_t *v,
                                            const uint8_t *ve, const v8bf (&q)[Pieces<DT>::n][2 * NB], int wave, int lane, int begin, int end,
                                            int wave_least, int wave_most, int limit, int stored_end, v16f (&o)[NB], float &m, float &l) {
    typedef PromptLds<NB> L;
    constexpr int NP = Pieces<DT>::n, NW = Pieces<DT>::weights;
    constexpr int KI = BRINGS & kBringKeys ? (W == 8 ? 1 : 4 / W) : 0, VI = BRINGS & kBringValues ? (W == 8 ? 1 : 4 / W) : 0;
    const int l32 = lane & 31, h = lane >> 5;
    RawItem<NB> rk[KI ? KI : 1], rv[VI ? VI : 1];
    // thread e of 256: words 4 g of key e / 4, g = e % 4; words of column e % 16 of value group e / 16
    const auto thread_of = [&](int i) { return 64 * ((wave + W * i) & 3) + lane; };
    const auto request_keys = [&](int key0) {
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            const int e = thread_of(i);
            const uint32_t key = key0 + (e >> 2);
            load_words<NB>(k + (key * 16 + (e & 3) * 4) * NB, rk[i].w);
            load_words<NB>(ke + (key >> 2) * 4 * NB, rk[i].e);
        }
    };
    const auto request_values = [&](int key0) {
#pragma unroll
        for (int i = 0; i < VI; ++i) {
            const int e = thread_of(i);
            const uint32_t group = key0 / 4 + (e >> 4);
            load_words<NB>(v + (group * 64 + (e & 15) * 4) * NB, rv[i].w);
            load_words<NB>(ve + group * 4 * NB, rv[i].e);
        }
    };
    const auto deliver_keys = [&](int buffer) {
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            const int e = thread_of(i), down = 8 * ((e >> 2) & 3);
            uint8_t *const dst = lds + buffer * L::kKeys + (e >> 2) * L::kKeyPitch + (e & 3) * 16;
#pragma unroll
            for (int blk = 0; blk < NB; ++blk)
                *reinterpret_cast<v8bf *>(dst + blk * 64) = key_values(rk[i].w[blk], conversion_scale(rk[i].e[blk] >> down, 0));
        }
    };
    const auto deliver_values = [&](int key0, int buffer) {
#pragma unroll
        for (int i = 0; i < VI; ++i) {
            const int e = thread_of(i), j4 = e >> 4, c = e & 15;
            // nothing past the stored tokens may be infinite: a weight of 0 has to silence it
            const int stored = stored_end - (key0 + 4 * j4);
            const uint32_t mask = stored >= 4 ? 0xffffffffu : stored <= 0 ? 0u : (1u << (8 * stored)) - 1u;
            uint8_t *const dst = lds + 2 * L::kKeys + buffer * L::kValues + c * kValuePitch + (16 * (j4 >> 2) + 8 * (j4 & 1) + 2 * (j4 & 2)) * 2;
#pragma unroll
            for (int blk = 0; blk < NB; ++blk) {
                const uint32_t x = rv[i].e[blk] & mask, lo = fp8_of_low(rv[i].w[blk]), hi = fp8_of_high(rv[i].w[blk]);
                const float s0 = value_scale(x, 0), s1 = value_scale(x, 1), s2 = value_scale(x, 2), s3 = value_scale(x, 3);
                const v2u a = {bf16_pair2<false>(lo, s0, s1), bf16_pair2<true>(lo, s2, s3)};
                const v2u z = {bf16_pair2<false>(hi, s0, s1), bf16_pair2<true>(hi, s2, s3)};
                *reinterpret_cast<v2u *>(dst + 32 * blk * kValuePitch) = a;
                *reinterpret_cast<v2u *>(dst + (32 * blk + 16) * kValuePitch) = z;
            }
        }
    };
    const auto scores = [&](int buffer, v16f (&s)[2]) {
        const uint8_t *const kb = lds + buffer * L::kKeys + l32 * L::kKeyPitch + h * 16;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int x = 0; x < 16; ++x) s[kt][x] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < 2 * NB; ++ks)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const v8bf a = *reinterpret_cast<const v8bf *>(kb + kt * 32 * L::kKeyPitch + ks * 32);
#pragma unroll
                for (int n = NP - 1; n >= 0; --n) s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[n][ks], s[kt], 0, 0, 0);
            }
    };
    // the largest of a lane's scores of the tile at key0, those it may not see made -infinity
    const auto largest = [&](int key0, v16f (&s)[2], auto masked) {
        float top = -INFINITY;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                if (decltype(masked)::value) s[kt][x] = key0 + 32 * kt + 8 * (x >> 2) + 4 * h + (x & 3) < limit ? s[kt][x] : -INFINITY;
                top = fmaxf(top, s[kt][x]);
            }
        const v2u sw = __builtin_bit_cast(v2u, __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false));
        return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * p.scale2;
    };
    // m is the largest score up to a factor of 2^kSlack in its exponential: among 32 queries a new largest score turns up in most
    // tiles, one that much larger hardly ever after the first
    const auto rescale = [&](float top) {
        if (__any(top > m + kSlack)) {
            const float m_new = fmaxf(m, top), shrink = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
            l *= shrink;
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int x = 0; x < 16; ++x) o[i][x] *= shrink;
            m = m_new;
        }
    };
    // the weights of a tile's scores
    const auto weights = [&](v16f (&s)[2]) {
        const float from = m == -INFINITY ? 0.0f : m;
        float sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int x = 0; x < 16; x += 2) {
                s[kt][x] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][x], p.scale2, -from));
                s[kt][x + 1] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][x + 1], p.scale2, -from));
                sum[0] += s[kt][x];
                sum[1] += s[kt][x + 1];
            }
        l += sum[0] + sum[1];
    };
    const auto accumulate = [&](int buffer, const v16f (&s)[2]) {
        const uint8_t *const vb = lds + 2 * L::kKeys + buffer * L::kValues + l32 * kValuePitch + h * 16;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                uint32_t w[4][NW];
#pragma unroll
                for (int i = 0; i < 4; ++i) bf16_pieces2<NW>(s[kt][8 * ks + 2 * i], s[kt][8 * ks + 2 * i + 1], w[i]);
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    const v8bf a = *reinterpret_cast<const v8bf *>(vb + 32 * i * kValuePitch + (32 * kt + 16 * ks) * 2);
#pragma unroll
                    for (int n = NW - 1; n >= 0; --n) {
                        const v4u pw = {w[0][n], w[1][n], w[2][n], w[3][n]};
                        o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(v8bf, pw), o[i], 0, 0, 0);
                    }
                }
            }
    };
    const int count = (end - begin + kTile - 1) / kTile;                          // tiles of the workgroup
    const int own_end = wave_most < end ? wave_most : end, free_end = wave_least < end ? wave_least : end;
    const int own = own_end > begin ? (own_end - begin + kTile - 1) / kTile : 0;   // that some of the wave's queries see
    const int open = free_end > begin ? (free_end - begin) / kTile : 0;            // that all of them see whole
    const auto key_of = [&](int i) { return begin + i * kTile; };
    // keys 0, keys 1 and values 0 into the buffers, the next ones on their way
    request_keys(begin);
    request_values(begin);
    deliver_keys(0);
    deliver_values(begin, 0);
    if (count > 1) {
        request_keys(key_of(1));
        request_values(key_of(1));
        deliver_keys(1);
    }
    if (count > 2) request_keys(key_of(2));
    // (without branches: past the last tile the same words are converted again, into buffers that nobody reads any more)
    const auto bring = [&](int i) {
        deliver_keys(i & 1);
        deliver_values(key_of(i + 1), (i + 1) & 1);
        request_keys(key_of(i + 3 < count ? i + 3 : count - 1));
        request_values(key_of(i + 2 < count ? i + 2 : count - 1));
    };
    __syncthreads();
    v16f s[2];
    float top = -INFINITY;
    if (own > 0) {
        scores(0, s);
        top = open > 0 ? largest(begin, s, No()) : largest(begin, s, Yes());
    }
    __syncthreads();                                                              // (iteration 0 writes keys 2 where keys 0 were)
    int i = 0;
    v16f other[2];
    const auto iteration = [&](v16f (&now)[2], v16f (&ahead)[2], auto masked) {
        rescale(top);
        scores((i + 1) & 1, ahead);
        weights(now);
        accumulate(i & 1, now);
        bring(i);
        top = largest(key_of(i + 1), ahead, masked);
        __syncthreads();
        ++i;
    };
    const auto settle = [&]() { s[0] = other[0], s[1] = other[1]; };
    while (i + 2 < open) {
        iteration(s, other, No());
        iteration(other, s, No());
    }
    if (i + 1 < open) iteration(s, other, No()), settle();
    while (i + 1 < own) iteration(s, other, Yes()), settle();
    if (own > 0) {
        rescale(top);
        weights(s);
        accumulate(i & 1, s);
    }
    for (; i < count; ++i) {
        bring(i);
        __syncthreads();
    }
}

template <int NB, int DT, int W>
__global__ __launch_bounds__(64 * W, 2) void cache_prompt_kernel(const SplitParams p) {
    constexpr int NP = Pieces<DT>::n, DP = 32 * NB;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const CacheView &cache = p.a.c;
    // heads innermost: consecutive workgroups are dealt to different XCDs, and those of one head meet in one; the tiles with the
    // most keys (the last rows) first
    uint32_t id = blockIdx.x;
    const uint32_t heads = cache.batch * cache.heads;
    const int64_t bh = id % heads;
    id /= heads;
    const int chunk = (int)(id % p.chunks), tile = p.tiles - 1 - (int)(id / p.chunks);
    const int64_t b = bh / cache.heads;
    const int key_head = (int)(bh % cache.heads);
    const int length = p.a.lengths[b], bound = p.a.longest;
    const int t = threadIdx.x, lane = t & 63, l32 = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int row0 = 32 * W * tile, end_row = row0 + 32 * W < p.rows ? row0 + 32 * W : p.rows;
    const int most = visible(length, p.a.tokens, p.a.group, end_row - 1, p.a.causal, bound);
    const int begin = chunk * p.chunk, end = most < begin + p.chunk ? most : begin + p.chunk;
    if (begin >= end && p.chunks > 1) return;                 // the whole workgroup, before any barrier

    // this wave's rows, this lane's row
    const int wrow0 = row0 + 32 * wave, wend = wrow0 + 32 < p.rows ? wrow0 + 32 : p.rows, row = wrow0 + l32;
    int wave_most = 0, wave_least = 0, limit = 0;
    if (wrow0 < p.rows) {
        wave_most = visible(length, p.a.tokens, p.a.group, wend - 1, p.a.causal, bound);
        wave_least = visible(length, p.a.tokens, p.a.group, wrow0, p.a.causal, bound);
    }
    int64_t q_at = 0;
    if (row < p.rows) {
        limit = visible(length, p.a.tokens, p.a.group, row, p.a.causal, bound);
        q_at = b * p.a.q.sb + (row / p.a.group) * p.a.q.st + (key_head * p.a.group + row % p.a.group) * p.a.q.sh;
    }
    v8bf q[NP][2 * NB];
#pragma unroll
    for (int ks = 0; ks < 2 * NB; ++ks) {
        const int d0 = 16 * ks + 8 * h;
        float x[8];
        load8<DT>(p.a.q.data, q_at + d0, row < p.rows ? cache.dim - d0 : 0, x);
        if (p.a.scale < 0.0f)                               // scale2 is the magnitude
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = -x[i];
        uint32_t w[4][NP];
#pragma unroll
        for (int i = 0; i < 4; ++i) bf16_pieces2<NP>(x[2 * i], x[2 * i + 1], w[i]);
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            const v4u r = {w[0][n], w[1][n], w[2][n], w[3][n]};
            q[n][ks] = __builtin_bit_cast(v8bf, r);
        }
    }

    const uint8_t *k = cache.k + bh * cache.head_codes, *v = cache.v + bh * cache.head_codes;
    const uint8_t *ke = cache.ke + bh * cache.head_exps, *ve = cache.ve + bh * cache.head_exps;
    v16f o[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[i][x] = 0.0f;
    float m = -INFINITY, l = 0.0f;
    if (begin < end) {
        const int stored_end = length < bound ? length : bound;
        if constexpr (W == 8) {
            if (wave < 4) prompt_walk<NB, DT, W, kBringKeys>(p, lds, k, ke, v, ve, q, wave, lane, begin, end, wave_least, wave_most, limit, stored_end, o, m, l);
            else prompt_walk<NB, DT, W, kBringValues>(p, lds, k, ke, v, ve, q, wave, lane, begin, end, wave_least, wave_most, limit, stored_end, o, m, l);
        } else {
            prompt_walk<NB, DT, W, kBringKeys | kBringValues>(p, lds, k, ke, v, ve, q, wave, lane, begin, end, wave_least, wave_most, limit, stored_end, o, m, l);
        }
    }
    {
        const v2u sw = __builtin_bit_cast(v2u, __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false));
        l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    }
    if (row >= p.rows) return;
    if (p.chunks > 1) {
        const int64_t slot = (bh * p.chunks + chunk) * p.rows + row;
        float *const dst = p.o + slot * DP + 4 * h;
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int x = 0; x < 16; x += 4) {
                const v4f r = {o[i][x], o[i][x + 1], o[i][x + 2], o[i][x + 3]};
                *reinterpret_cast<v4f *>(dst + 32 * i + 2 * x) = r;
            }
        if (h == 0) p.ml[2 * slot] = m, p.ml[2 * slot + 1] = l;
        return;
    }
    const int tok = row / p.a.group, head = key_head * p.a.group + row % p.a.group;
    const float inv = l == 0.0f ? 0.0f : kUp / l;
    const int64_t dst = b * p.a.out.sb + tok * p.a.out.st + head * p.a.out.sh;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int x = 0; x < 16; x += 4) {
            const int d = 32 * i + 2 * x + 4 * h;
            const float r[4] = {o[i][x] * inv, o[i][x + 1] * inv, o[i][x + 2] * inv, o[i][x + 3] * inv};
            store4<DT>(p.a.out.data, dst + d, cache.dim - d, r);
        }
    if (h == 0) p.a.lse[(b * p.a.tokens + tok) * p.a.heads + head] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int NB, int DT, int W>
int launch_prompt(const SplitParams &p, hipStream_t s) {
    static std::atomic<bool> configured;
    void (*const kernel)(SplitParams) = &cache_prompt_kernel<NB, DT, W>;
    if (allow_dynamic_lds(configured, reinterpret_cast<const void *>(kernel), PromptLds<NB>::kBytes) != HBFP_OK) return HBFP_ERR_LAUNCH;
    hipLaunchKernelGGL(kernel, dim3(p.wgs), dim3(64 * W), PromptLds<NB>::kBytes, s, p);
    return launch_status();
}
template <int NB, int DT>
int launch_prompt_rows(const SplitParams &p, hipStream_t s) {
    return p.tile_rows == 256 ? launch_prompt<NB, DT, 8>(p, s) : p.tile_rows == 128 ? launch_prompt<NB, DT, 4>(p, s) : launch_prompt<NB, DT, 2>(p, s);
}
template <int DT>
int launch_prompt_of(const SplitParams &p, hipStream_t s) {
    switch (p.a.c.nblk) {
        case 1: return launch_prompt_rows<1, DT>(p, s);
        case 2: return launch_prompt_rows<2, DT>(p, s);
        case 3: return launch_prompt_rows<3, DT>(p, s);
        default: return launch_prompt_rows<4, DT>(p, s);
    }
}

}  // namespace

// Rows from which the tiles of this kernel are ahead of tiles of 16 (below, most of a tile of 64 would be empty), and their height:
// tall where the chip is full either way, because a tile of keys is converted once for all rows of a workgroup
bool cache_prompt_ok(const AttendArgs &a) {
    return a.c.nblk <= 4 && (int64_t)a.tokens * a.group > 48;
}
int64_t cache_prompt_rows(const AttendArgs &a) {
    const int64_t rows = (int64_t)a.tokens * a.group, heads = (int64_t)a.c.batch * a.c.heads;
    const int64_t chunks = ceil_div(a.longest, 512);
    if (rows > 128 && heads * ceil_div(rows, 256) * chunks >= 256) return 256;
    return rows > 64 && heads * ceil_div(rows, 128) * chunks >= 256 ? 128 : 64;
}

int launch_cache_prompt(const SplitParams &p, int dtype, hipStream_t s) {
    return dtype == HBFP_F32 ? launch_prompt_of<HBFP_F32>(p, s) : dtype == HBFP_BF16 ? launch_prompt_of<HBFP_BF16>(p, s) : launch_prompt_of<HBFP_F16>(p, s);
}

}  // namespace hbfp
