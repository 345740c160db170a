// Softmax attention over the 4-bit cache for many queries per key head (prompts, chunks of prompts).
//
// A workgroup of W waves holds 32 W query rows of one key head, 32 a wave, and walks over tiles of 64 keys.  A tile's keys and
// values are turned into bf16 numbers once, exactly, by all its waves together, into LDS: keys as they are, values transposed,
// in the order in which the scores' register layout presents keys.  Then S^T = K Q^T and O^T += V^T P^T as in the kernel for
// few queries, on the 32 x 32 x 16 matrix instruction: a lane holds one query, and its softmax needs one exchange with the lane
// 32 away.  The raw nibbles of the tile after next are on their way from memory, and the next tile is written to the other
// buffer, while a tile is multiplied: one barrier a tile.
#include "kv_cache.h"

namespace hbfp {
namespace {

struct No { static constexpr bool value = false; };
struct Yes { static constexpr bool value = true; };
constexpr int kTile = 64;                  // keys
constexpr float kSlack = 6.0f;
constexpr int kValuePitch = kTile * 2 + 16;  // bytes of a row of transposed values: 16 more than its keys, so that rows differ in banks
template <int NB> struct PromptLds {
    static constexpr int kKeyPitch = 64 * NB + 16, kKeys = kTile * kKeyPitch, kValues = 32 * NB * kValuePitch;
    static constexpr int kBuffer = kKeys + kValues, kBytes = 2 * kBuffer;
};

// one thread's share of a tile: NB words of a key's row, or NB words of a group of four values, and their exponents
template <int NB>
struct RawItem {
    uint32_t w[NB], e[NB];
};
template <int NB>
__device__ __forceinline__ void load_item(const uint8_t *codes, const uint8_t *exps, uint32_t at, uint32_t exp_at, RawItem<NB> &r) {
    load_words<NB>(codes + at, r.w);
    load_words<NB>(exps + exp_at, r.e);
}
// two numbers with a scale each: both conversions of the pair, one half of each
template <bool HIGH>
__device__ __forceinline__ uint32_t bf16_pair2(uint32_t fp8, float s0, float s1) {
    return __builtin_amdgcn_perm(bf16_pair<HIGH>(fp8, s1), bf16_pair<HIGH>(fp8, s0), 0x07060100u);
}

template <int NB, int DT, int W>
__global__ __launch_bounds__(64 * W, 2) void cache_prompt_kernel(const SplitParams p) {
    typedef PromptLds<NB> L;
    constexpr int NP = Pieces<DT>::n, DP = 32 * NB, ITEMS = 8 / W;
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
    RawItem<NB> raw[ITEMS];
    // items 0..3 are keys (a quarter of the tile each: thread e has words 4 g of key e / 4, g = e % 4), 4..7 values (group e / 16,
    // column e % 16)
    const auto request = [&](int key0) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int item = wave + W * i, e = 64 * (item & 3) + lane;
            if (item < 4) {
                const uint32_t key = key0 + (e >> 2);
                load_item<NB>(k, ke, (key * 16 + (e & 3) * 4) * NB, (key >> 2) * 4 * NB, raw[i]);
            } else {
                const uint32_t group = key0 / 4 + (e >> 4);
                load_item<NB>(v, ve, (group * 64 + (e & 15) * 4) * NB, group * 4 * NB, raw[i]);
            }
        }
    };
    const auto deliver = [&](int key0, int buffer) {
        uint8_t *const kb = lds + buffer * L::kBuffer, *const vb = kb + L::kKeys;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int item = wave + W * i, e = 64 * (item & 3) + lane;
            if (item < 4) {
                uint8_t *const dst = kb + (e >> 2) * L::kKeyPitch + (e & 3) * 16;
                const int down = 8 * ((e >> 2) & 3);
#pragma unroll
                for (int blk = 0; blk < NB; ++blk)
                    *reinterpret_cast<v8bf *>(dst + blk * 64) = key_values(raw[i].w[blk], conversion_scale(raw[i].e[blk] >> down, 0));
            } else {
                const int j4 = e >> 4, c = e & 15;
                // nothing past the stored tokens may be infinite: a weight of 0 has to silence it
                const int stored = (length < bound ? length : bound) - (key0 + 4 * j4);
                const uint32_t mask = stored >= 4 ? 0xffffffffu : stored <= 0 ? 0u : (1u << (8 * stored)) - 1u;
                uint8_t *const dst = vb + c * kValuePitch + (16 * (j4 >> 2) + 8 * (j4 & 1) + 2 * (j4 & 2)) * 2;
#pragma unroll
                for (int blk = 0; blk < NB; ++blk) {
                    const uint32_t x = raw[i].e[blk] & mask, lo = fp8_of_low(raw[i].w[blk]), hi = fp8_of_high(raw[i].w[blk]);
                    const float s0 = conversion_scale(x, 0), s1 = conversion_scale(x, 1), s2 = conversion_scale(x, 2), s3 = conversion_scale(x, 3);
                    const v2u a = {bf16_pair2<false>(lo, s0, s1), bf16_pair2<true>(lo, s2, s3)};
                    const v2u z = {bf16_pair2<false>(hi, s0, s1), bf16_pair2<true>(hi, s2, s3)};
                    *reinterpret_cast<v2u *>(dst + 32 * blk * kValuePitch) = a;
                    *reinterpret_cast<v2u *>(dst + (32 * blk + 16) * kValuePitch) = z;
                }
            }
        }
    };

    v16f o[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[i][x] = 0.0f;
    float m = -INFINITY, l = 0.0f;

    const auto multiply = [&](int key0, int buffer, auto masked) {
        constexpr bool MASK = decltype(masked)::value;
        const uint8_t *const kb = lds + buffer * L::kBuffer + l32 * L::kKeyPitch + h * 16;
        const uint8_t *const vb = lds + buffer * L::kBuffer + L::kKeys + l32 * kValuePitch + h * 16;
        v16f s[2];
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
        float top = -INFINITY;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                if (MASK) s[kt][x] = key0 + 32 * kt + 8 * (x >> 2) + 4 * h + (x & 3) < limit ? s[kt][x] : -INFINITY;
                top = fmaxf(top, s[kt][x]);
            }
        const v2u sw = __builtin_bit_cast(v2u, __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false));
        top = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * p.scale2;
        // m is the largest score up to a factor of 2^kSlack in its exponential: among 32 queries a new largest score turns up in most
        // tiles, one that much larger hardly ever after the first
        if (__any(top > m + kSlack)) {
            const float m_new = fmaxf(m, top), shrink = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
            l *= shrink;
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int x = 0; x < 16; ++x) o[i][x] *= shrink;
            m = m_new;
        }
        const float from = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                uint32_t w[4][NP];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][8 * ks + 2 * i], p.scale2, -from));
                    const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][8 * ks + 2 * i + 1], p.scale2, -from));
                    l += x + y;
                    bf16_pieces2<NP>(x, y, w[i]);
                }
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    const v8bf a = *reinterpret_cast<const v8bf *>(vb + 32 * i * kValuePitch + (32 * kt + 16 * ks) * 2);
#pragma unroll
                    for (int n = NP - 1; n >= 0; --n) {
                        const v4u pw = {w[0][n], w[1][n], w[2][n], w[3][n]};
                        o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(v8bf, pw), o[i], 0, 0, 0);
                    }
                }
            }
    };

    if (begin < end) {
        request(begin);
        deliver(begin, 0);
        if (begin + kTile < end) request(begin + kTile);
        __syncthreads();
        // the tiles that all of the wave's queries see, those that some see, those that are for the other waves: a loop each, so that
        // the accumulators stay where they are; every wave passes the same number of barriers
        int key0 = begin, buffer = 0;
        const auto prepare = [&]() {
            if (key0 + kTile < end) {
                deliver(key0 + kTile, buffer ^ 1);
                if (key0 + 2 * kTile < end) request(key0 + 2 * kTile);
            }
        };
        const auto next = [&]() {
            __syncthreads();
            key0 += kTile;
            buffer ^= 1;
        };
        while (key0 < end && key0 + kTile <= wave_least) {
            prepare();
            multiply(key0, buffer, No());
            next();
        }
        while (key0 < end && key0 < wave_most) {
            prepare();
            multiply(key0, buffer, Yes());
            next();
        }
        while (key0 < end) {
            prepare();
            next();
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
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
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

bool cache_prompt_ok(const AttendArgs &a, int dtype) {
    (void)dtype;
    return a.c.nblk <= 4 && (int64_t)a.tokens * a.group > 48;
}
int64_t cache_prompt_rows(const AttendArgs &a) {
    const int64_t rows = (int64_t)a.tokens * a.group;
    return rows <= 64 ? 64 : rows <= 128 ? 128 : 256;
}

int launch_cache_prompt(const SplitParams &p, int dtype, hipStream_t s) {
    return dtype == HBFP_F32 ? launch_prompt_of<HBFP_F32>(p, s) : dtype == HBFP_BF16 ? launch_prompt_of<HBFP_BF16>(p, s) : launch_prompt_of<HBFP_F16>(p, s);
}

}  // namespace hbfp
