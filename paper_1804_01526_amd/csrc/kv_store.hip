// The 4-bit cache: converting and storing new tokens, reading values back, and eviction by accumulated attention weight.
#include "bfp_device.h"
#include "kv_cache.h"

namespace hbfp {
namespace {

__device__ __forceinline__ int clamp_length(int n, int capacity) { return n < 0 ? 0 : n > capacity ? capacity : n; }

// ---- append.  Sixteen lanes hold the 32 dimensions of one block for the four slots of a group: lane 4 j + g has dimensions
// 8 g .. 8 g + 7 of slot 4 group + j, so a block's largest magnitude is the largest of four neighbouring lanes.  Bound by the
// reads of the inputs (prompts) or by the launch (single tokens): 4 to 5 us for one token of up to 32 conversations, 25 us for 2 x 2048
// tokens of 8 key heads of 128 in bf16 with the held values returned (34 MB, 1.4 TB/s).
struct AppendParams {
    CacheView c;
    Heads k, v;
    const int32_t *lengths;
    uint16_t *k_values, *v_values;
    int64_t units;               // batch * heads * groups * nblk
    int32_t tokens, groups;
};

// eight mantissas as nibbles (low: 0..3, high: 4..7, one byte each pair) and the exponent byte of the block
__device__ __forceinline__ uint32_t convert8(const float *x, uint32_t &Eb) {
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = __float_as_uint(x[i]) & 0x7fffffffu;
        amax = a > amax ? a : amax;
    }
    uint32_t o = __shfl_xor(amax, 1);
    amax = o > amax ? o : amax;
    o = __shfl_xor(amax, 2);
    amax = o > amax ? o : amax;
    Eb = block_exponent<HBFP_RNE>(amax, 4);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int q = quant_rne(x[i], 129 - (int)Eb);
        const uint32_t mag = (uint32_t)(q < 0 ? -q : q) & 7u;      // (& 7: values that are not finite, whose mantissas are unspecified)
        w |= (mag | (q < 0 ? 8u : 0u)) << (8 * (i & 3) + 4 * (i >> 2));
    }
    return w;
}
__device__ __forceinline__ float nibble_value(uint32_t nib, uint32_t Eb) {
    const float m = (float)(nib & 7u);
    return __builtin_amdgcn_ldexpf(nib & 8u ? -m : m, (int)Eb - 129);
}

template <int DT>
__global__ __launch_bounds__(256) void cache_append_kernel(const AppendParams p) {
    const int64_t unit = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (unit >= p.units) return;                              // sixteen lanes leave together
    const int lane = threadIdx.x & 15, g = lane & 3, j = lane >> 2;
    const int nblk = p.c.nblk;
    const int blk = (int)(unit % nblk);
    const int64_t gi = unit / nblk;
    const int64_t bh = gi / p.groups;
    const int h = (int)(bh % p.c.heads);
    const int64_t b = bh / p.c.heads;
    const int length = p.lengths[b];
    const int64_t first = (int64_t)(length < 0 ? 0 : length) - p.tokens;   // slot of token 0
    const int64_t group = (first >> 2) + gi % p.groups, slot = 4 * group + j;
    const int64_t t = slot - first;
    const bool mine = t >= 0 && t < p.tokens, held = mine && slot >= 0 && slot < p.c.capacity;
    const int d0 = 32 * blk + 8 * g, n = mine ? p.c.dim - d0 : 0;
    float xk[8], xv[8];
    load8<DT>(p.k.data, b * p.k.sb + t * p.k.st + h * p.k.sh + d0, n, xk);
    load8<DT>(p.v.data, b * p.v.sb + t * p.v.st + h * p.v.sh + d0, n, xv);
    uint32_t ek, ev;
    const uint32_t wk = convert8(xk, ek), wv = convert8(xv, ev);
    // an Inf or a NaN in a value is marked in the key's exponent, which makes the score of whoever sees the token NaN: the kernels
    // then never meet a value that is not finite, and a weight of 0 silences any value
    ek = ev == 255u ? 255u : ek;
    ev = ev == 255u ? 254u : ev;
    const uint32_t partner = __shfl_xor(wv, 2);               // dimensions 16 higher (g 0, 1) of the same block and slot
    if (held) {
        uint8_t *kc = p.c.k + bh * p.c.head_codes, *vc = p.c.v + bh * p.c.head_codes;
        *reinterpret_cast<uint32_t *>(kc + (slot * 16 + g * 4) * nblk + blk * 4) = wk;
        if (g < 2) {
            // this lane's dimensions are columns c = 8 g + i of the value group, low nibbles; the partner's the high ones
            uint8_t *dst = vc + (group * 64 + 8 * g * 4) * nblk + blk * 4 + j;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int sh = 8 * (i & 3) + 4 * (i >> 2);
                dst[i * 4 * nblk] = (uint8_t)(((wv >> sh) & 15u) | (((partner >> sh) & 15u) << 4));
            }
        }
        if (g == 0) {
            const int64_t e = bh * p.c.head_exps + (group * nblk + blk) * 4 + j;
            p.c.ke[e] = (uint8_t)ek;
            p.c.ve[e] = (uint8_t)ev;
        }
    }
    if (mine && d0 < p.c.dim) {
        const int64_t o = ((b * p.tokens + t) * p.c.heads + h) * p.c.dim + d0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int sh = 8 * (i & 3) + 4 * (i >> 2);
            if (d0 + i < p.c.dim) {
                if (p.k_values) store_float<HBFP_BF16>(p.k_values, o + i, held ? nibble_value((wk >> sh) & 15u, ek) : 0.0f);
                if (p.v_values) store_float<HBFP_BF16>(p.v_values, o + i, held ? nibble_value((wv >> sh) & 15u, ev) : 0.0f);
            }
        }
    }
}

// ---- read.  A thread has eight dimensions of one slot of a head; slots from the length on are 0.  Bound by its stores: 128
// heads of 4096 slots of 128 in bf16, 268 MB written in 57 us, 4.7 TB/s.
struct ReadParams {
    CacheView c;
    const int32_t *lengths;
    void *k, *v;
    int64_t units;               // batch * heads * capacity * 4 nblk
};

template <int DT>
__device__ __forceinline__ void store8(void *p, int64_t i, int n, bool whole, const float *x) {
    if (whole) {
        if (DT == HBFP_F32) {
            const v4f a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
            *reinterpret_cast<v4f *>(reinterpret_cast<float *>(p) + i) = a;
            *reinterpret_cast<v4f *>(reinterpret_cast<float *>(p) + i + 4) = b;
        } else {
            const v4u a = {bf16_bits2(x[0], x[1]), bf16_bits2(x[2], x[3]), bf16_bits2(x[4], x[5]), bf16_bits2(x[6], x[7])};
            *reinterpret_cast<v4u *>(reinterpret_cast<uint16_t *>(p) + i) = a;
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) store_float<DT>(p, i + j, x[j]);
}

template <int DT>
__global__ __launch_bounds__(256) void cache_read_kernel(const ReadParams p) {
    const int64_t unit = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (unit >= p.units) return;
    const int nblk = p.c.nblk, pieces = 4 * nblk;
    const int piece = (int)(unit % pieces), blk = piece >> 2, g = piece & 3;
    const int64_t row = unit / pieces, bh = row / p.c.capacity;
    const int slot = (int)(row % p.c.capacity), j = slot & 3, group = slot >> 2;
    const bool held = slot < clamp_length(p.lengths[bh / p.c.heads], p.c.capacity);
    const int d0 = 32 * blk + 8 * g, n = p.c.dim - d0;
    if (n <= 0) return;
    const bool whole = n >= 8 && p.c.dim % 8 == 0;
    const int64_t e = bh * p.c.head_exps + ((int64_t)group * nblk + blk) * 4 + j, o = row * p.c.dim + d0;
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (p.k) {
        if (held) {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(p.c.k + bh * p.c.head_codes + ((int64_t)slot * 16 + g * 4) * nblk + blk * 4);
            const uint32_t Eb = p.c.ke[e];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = nibble_value(w >> (8 * (i & 3) + 4 * (i >> 2)), Eb);
        }
        store8<DT>(p.k, o, n, whole && ((uintptr_t)p.k & 15) == 0, x);
    }
    if (p.v) {
        if (held) {
            const uint8_t *src = p.c.v + bh * p.c.head_codes + ((int64_t)group * 64 + 8 * (g & 1) * 4) * nblk + blk * 4 + j;
            const uint32_t Eb = p.c.ve[e];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = nibble_value((uint32_t)src[i * 4 * nblk] >> (g & 2 ? 4 : 0), Eb);
        }
        store8<DT>(p.v, o, n, whole && ((uintptr_t)p.v & 15) == 0, x);
    }
}

// ---- eviction.  One workgroup per head finds the keep - r largest of its first n - r weights: the smallest weight that stays is
// found 11, 11 and 10 bits at a time from counts of the values that share the bits above (integers in the order of the weights;
// eleven bits, because a histogram of exponents alone has all lanes at the same few counters), then one ordered walk writes the
// slots that stay.  A thread has 16 consecutive weights of a segment, in registers when one segment is all.  Bound by the latency of
// LDS counters and barriers: 128 heads of up to 16384 weights 22 us, 2 heads of 600 11 us.
struct EvictParams {
    CacheView src, dst;
    const float *w;
    float *w_out;
    const int32_t *lengths;
    int32_t *kept, *lengths_out;
    int64_t ld, ld_out;
    int32_t keep, recent;
    int64_t units;
};
// unsigned integers in the order of the weights; -0 equals 0, a NaN comes below everything
__device__ __forceinline__ uint32_t ordered(float x) {
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr int kOwn = 16, kBins = 2048;

// exclusive sums over the workgroup's threads, and the total; `sums`: one word per wave
template <int THREADS>
__device__ __forceinline__ uint32_t block_before(uint32_t x, uint32_t *sums, uint32_t &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t upto = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(upto, o);
        if (lane >= o) upto += y;
    }
    __syncthreads();                                         // (the words of the call before have been read)
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    uint32_t before = upto - x;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        const uint32_t s = sums[w];
        before += w < wave ? s : 0u;
        total += s;
    }
    return before;
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(const EvictParams p) {
    constexpr int kSegment = THREADS * kOwn, PER = kBins / THREADS;
    __shared__ uint32_t count[kBins];
    __shared__ uint32_t sums[THREADS / 64];
    __shared__ uint32_t found[2];
    const int64_t bh = blockIdx.x;
    const int b = (int)(bh / p.src.heads), t = threadIdx.x;
    const int n = clamp_length(p.lengths[b], p.src.capacity);
    const int m = n < p.keep ? n : p.keep;
    const float *w = p.w + bh * p.ld;
    float *w_out = p.w_out + bh * p.ld_out;
    int32_t *kept = p.kept + bh * p.keep;
    if (t == 0 && bh % p.src.heads == 0) p.lengths_out[b] = m;
    for (int i = m + t; i < p.keep; i += THREADS) kept[i] = -1;
    for (int i = m + t; i < p.dst.capacity; i += THREADS) w_out[i] = 0.0f;
    if (n <= p.keep) {
        for (int i = t; i < n; i += THREADS) kept[i] = i, w_out[i] = w[i];
        return;
    }
    const int r = p.recent < p.keep ? p.recent : p.keep, others = n - r, top = p.keep - r;
    float own[kOwn];
    const auto load = [&](int segment) {
        const int i0 = segment * kSegment + t * kOwn;
#pragma unroll
        for (int i = 0; i < kOwn; i += 4) {
            if (i0 + i + 4 <= n) {
                const v4f_at x = *reinterpret_cast<const v4f_at *>(w + i0 + i);
#pragma unroll
                for (int k = 0; k < 4; ++k) own[i + k] = x[k];
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) own[i + k] = i0 + i + k < n ? w[i0 + i + k] : 0.0f;
            }
        }
    };
    const int segments = (n + kSegment - 1) / kSegment;
    if (segments == 1) load(0);
    // the top-th largest of w[0 .. others): its bits in `prefix`, how many equal ones stay in `ties`
    uint32_t prefix = 0, ties = (uint32_t)top;
    if (top > 0) {
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            const uint32_t digit = pass == 2 ? 1023u : 2047u, above = pass == 0 ? 0u : pass == 1 ? ~0u << 21 : ~0u << 10;
            for (int i = t; i < kBins; i += THREADS) count[i] = 0;
            __syncthreads();
            for (int segment = 0; segment < segments; ++segment) {
                if (segments > 1) load(segment);
                const int i0 = segment * kSegment + t * kOwn;
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    const uint32_t key = ordered(own[i]);
                    if (i0 + i < others && (key & above) == prefix) atomicAdd(&count[(key >> shift) & digit], 1u);
                }
            }
            __syncthreads();
            // thread t: PER digits from the largest, 2047, down; how many keys have larger ones
            uint32_t c[PER], mine = 0, all;
#pragma unroll
            for (int i = 0; i < PER; ++i) mine += c[i] = count[kBins - 1 - PER * t - i];
            uint32_t before = block_before<THREADS>(mine, sums, all);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (before < ties && ties <= before + c[i]) found[0] = kBins - 1 - PER * t - i, found[1] = ties - before;
                before += c[i];
            }
            __syncthreads();
            prefix |= found[0] << shift;
            ties = found[1];
        }
    }
    // ordered walk: slot i stays if it is recent, above the bound, or one of the first `ties` at it
    uint32_t out = 0, equal_before = 0;
    for (int segment = 0; segment < segments; ++segment) {
        if (segments > 1) load(segment);
        const int i0 = segment * kSegment + t * kOwn;
        uint32_t stays = 0, equal = 0;                        // a bit for each own weight
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const uint32_t key = ordered(own[i]);
            const bool here = i0 + i < n, late = i0 + i >= others;
            if (here && (late || (top > 0 && key > prefix))) stays |= 1u << i;
            else if (here && top > 0 && key == prefix) equal |= 1u << i;
        }
        uint32_t all;
        uint32_t rank = equal_before + block_before<THREADS>((uint32_t)__popc(equal), sums, all);
        equal_before += all;
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
            if (equal >> i & 1u) {
                if (rank < ties) stays |= 1u << i;
                ++rank;
            }
        uint32_t pos = out + block_before<THREADS>((uint32_t)__popc(stays), sums, all);
        out += all;
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
            if (stays >> i & 1u) {
                kept[pos] = i0 + i;
                w_out[pos] = own[i];
                ++pos;
            }
    }
}

// Copies the kept slots.  Sixteen lanes have a group of four: lane c copies a quarter of one of its key rows (c / 4, c % 4) and
// joins column c of its values from the columns of the four slots' groups, whole words of which one byte is theirs.  Bound by those
// words, of which slots that are not neighbours use a quarter: 4096 slots of 128 heads of 128 in 39 us (byte by byte 103).
template <int NB>
__global__ __launch_bounds__(256) void evict_copy_kernel(const EvictParams p) {
    const int64_t gi = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (gi >= p.units) return;
    const int groups = (p.keep + 3) >> 2, c = threadIdx.x & 15;
    const int64_t bh = gi / groups;
    const int group = (int)(gi % groups);
    const int32_t *kept = p.kept + bh * p.keep;
    int from[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) from[j] = 4 * group + j < p.keep ? kept[4 * group + j] : -1;
    if (from[0] < 0) return;
    const uint8_t *sk = p.src.k + bh * p.src.head_codes, *sv = p.src.v + bh * p.src.head_codes;
    const uint8_t *ske = p.src.ke + bh * p.src.head_exps, *sve = p.src.ve + bh * p.src.head_exps;
    uint32_t kw[NB], vw[4][NB];
    const int j = c >> 2;
    int f = from[0];
#pragma unroll
    for (int i = 1; i < 4; ++i) f = j == i ? from[i] : f;
    if (f >= 0) load_words<NB>(sk + ((int64_t)f * 16 + (c & 3) * 4) * NB, kw);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int slot = from[i] < 0 ? from[0] : from[i];       // (no such slot: any that exists, nothing reads the result)
        load_words<NB>(sv + ((int64_t)(slot >> 2) * 64 + c * 4) * NB, vw[i]);
    }
    if (f >= 0) {
        uint32_t *const dst = reinterpret_cast<uint32_t *>(p.dst.k + bh * p.dst.head_codes + ((int64_t)(4 * group + j) * 16 + (c & 3) * 4) * NB);
#pragma unroll
        for (int i = 0; i < NB; ++i) dst[i] = kw[i];
    }
    uint32_t *const dst = reinterpret_cast<uint32_t *>(p.dst.v + bh * p.dst.head_codes + ((int64_t)group * 64 + c * 4) * NB);
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) {
        uint32_t r = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) r |= ((vw[i][blk] >> (8 * (from[i] & 3))) & 0xffu) << (8 * i);
        dst[blk] = r;
    }
    if (c < NB) {
        uint32_t rk = 0, rv = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (from[i] >= 0) {
                const int64_t e = ((int64_t)(from[i] >> 2) * NB + c) * 4 + (from[i] & 3);
                rk |= (uint32_t)ske[e] << (8 * i);
                rv |= (uint32_t)sve[e] << (8 * i);
            }
        const int64_t e = bh * p.dst.head_exps + ((int64_t)group * NB + c) * 4;
        *reinterpret_cast<uint32_t *>(p.dst.ke + e) = rk;
        *reinterpret_cast<uint32_t *>(p.dst.ve + e) = rv;
    }
}

}  // namespace

int launch_cache_append(const CacheView &c, const Heads &k, const Heads &v, int dtype, int64_t tokens, const int32_t *lengths,
                        void *k_values, void *v_values, hipStream_t s) {
    AppendParams p = {};
    p.c = c;
    p.k = k;
    p.v = v;
    p.lengths = lengths;
    p.k_values = (uint16_t *)k_values;
    p.v_values = (uint16_t *)v_values;
    p.tokens = (int32_t)tokens;
    p.groups = (int32_t)((tokens + 6) / 4);                     // groups of four slots that the tokens can touch
    p.units = (int64_t)c.batch * c.heads * p.groups * c.nblk;
    const int64_t wgs = ceil_div(p.units, 16);
    if (wgs > 0x7fffffff) return HBFP_ERR_ARG;
    void (*const kernel)(AppendParams) = dtype == HBFP_F32    ? &cache_append_kernel<HBFP_F32>
                                         : dtype == HBFP_BF16 ? &cache_append_kernel<HBFP_BF16>
                                                              : &cache_append_kernel<HBFP_F16>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(256), 0, s, p);
    return launch_status();
}

int launch_cache_read(const CacheView &c, const int32_t *lengths, int dtype, void *k, void *v, hipStream_t s) {
    ReadParams p = {c, lengths, k, v, (int64_t)c.batch * c.heads * c.capacity * 4 * c.nblk};
    const int64_t wgs = ceil_div(p.units, 256);
    if (wgs > 0x7fffffff) return HBFP_ERR_ARG;
    void (*const kernel)(ReadParams) = dtype == HBFP_F32 ? &cache_read_kernel<HBFP_F32> : &cache_read_kernel<HBFP_BF16>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(256), 0, s, p);
    return launch_status();
}

int launch_cache_evict(const CacheView &src, const float *w, int64_t ld, const int32_t *lengths, int64_t keep, int64_t recent,
                       const CacheView &dst, float *w_out, int64_t ld_out, int32_t *kept, int32_t *lengths_out, hipStream_t s) {
    EvictParams p = {src, dst, w, w_out, lengths, kept, lengths_out, ld, ld_out, (int32_t)keep, (int32_t)recent, 0};
    p.units = (int64_t)src.batch * src.heads * ceil_div(keep, 4);
    const int64_t wgs = ceil_div(p.units, 16);
    static void (*const copies[8])(EvictParams) = {&evict_copy_kernel<1>, &evict_copy_kernel<2>, &evict_copy_kernel<3>, &evict_copy_kernel<4>,
                                                   &evict_copy_kernel<5>, &evict_copy_kernel<6>, &evict_copy_kernel<7>, &evict_copy_kernel<8>};
    if (wgs > 0x7fffffff) return HBFP_ERR_ARG;
    // a segment that holds the whole cache, if one does: four waves for small caches (barriers among 16 cost 600 slots 15 us)
    if (src.capacity <= 256 * kOwn) hipLaunchKernelGGL(evict_select_kernel<256>, dim3((unsigned)(src.batch * src.heads)), dim3(256), 0, s, p);
    else hipLaunchKernelGGL(evict_select_kernel<1024>, dim3((unsigned)(src.batch * src.heads)), dim3(1024), 0, s, p);
    hipLaunchKernelGGL(copies[src.nblk - 1], dim3((unsigned)wgs), dim3(256), 0, s, p);
    return launch_status();
}

}  // namespace hbfp
