// Device side of the 4-bit cache: its layout (stated in the public header), the way from nibbles to bf16 and loads and
// stores of the three tensor types.
#pragma once
#include "hbfp_internal.h"
#include "serve.h"

namespace hbfp {
namespace {

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr float kSlack = 6.0f;             // of a running maximum, in powers of two
// Values enter the sums 2^-kDown times as large: weights of up to 2^kSlack times values below 2^127, over as many tokens as a head's buffer
// can hold (2^27), stay below 2^128, and the division by the sum of the weights takes the factor back
constexpr int kDown = 34;
constexpr float kUp = 0x1p34f;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// keys that row `row` (token row / group) of batch entry b may see
__device__ __forceinline__ int visible(int length, int tokens, int group, int row, int causal, int bound) {
    const int len = length < 0 ? 0 : length;
    const int64_t n = causal ? (int64_t)len - tokens + row / group + 1 : (int64_t)len;
    return n < 0 ? 0 : n > bound ? bound : (int)n;
}

// ---- nibbles -> numbers.  A nibble is sign and magnitude, so that one byte permute looks four magnitudes up in a table of
// eight FP8 (E4M3) numbers, n / 4, and the sign is the fourth bit moved to the eighth: four instructions for the four low or
// the four high nibbles of a word.  The conversion FP8 -> bf16 multiplies by a power of two, whose FP32 exponent field is
// the block's exponent byte itself: n / 4 * 2^(Eb - 127) = n * 2^(Eb - 129).  Exact for every Eb up to 254, subnormal results
// included; Eb = 255 gives NaN.
__device__ __forceinline__ uint32_t fp8_of_low(uint32_t w) {
    return __builtin_amdgcn_perm(0x3E3C3A38u, 0x34302800u, w & 0x07070707u) | ((w << 4) & 0x80808080u);
}
__device__ __forceinline__ uint32_t fp8_of_high(uint32_t w) {
    return __builtin_amdgcn_perm(0x3E3C3A38u, 0x34302800u, (w >> 4) & 0x07070707u) | (w & 0x80808080u);
}
// bytes 0 and 1 (HIGH: 2 and 3) as two bf16 numbers times scale, a power of two
template <bool HIGH>
__device__ __forceinline__ uint32_t bf16_pair(uint32_t fp8, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(fp8, scale, HIGH));
}
// the same scale for the FP8 conversion, which looks at nothing but the exponent field: the byte `j` of a word moved there
__device__ __forceinline__ float conversion_scale(uint32_t word, int j) { return __uint_as_float(j < 3 ? word << (23 - 8 * j) : word >> 1); }
// ... of a block of values, 2^-kDown times as large (units below 2^-95 count as that: exponents end at 0)
__device__ __forceinline__ float value_scale(uint32_t word, int j) {
    return conversion_scale(word, j) * (1.0f / kUp);
}
// x times the 2^(Eb - 127 - kDown) of the exponent byte `j` of a word; 0 stays 0 for every byte
__device__ __forceinline__ float times_exponent(float x, uint32_t word, int j) {
    return __builtin_amdgcn_ldexpf(x, (int)((word >> (8 * j)) & 0xffu) - (127 + kDown));
}

// eight values in the order low nibbles, high nibbles (for the key layout: dimensions 8 g .. 8 g + 7)
__device__ __forceinline__ v8bf key_values(uint32_t w, float scale) {
    const uint32_t lo = fp8_of_low(w), hi = fp8_of_high(w);
    const v4u r = {bf16_pair<false>(lo, scale), bf16_pair<true>(lo, scale), bf16_pair<false>(hi, scale), bf16_pair<true>(hi, scale)};
    return __builtin_bit_cast(v8bf, r);
}

// ---- the three tensor types
template <int DT>
__device__ __forceinline__ float load_as_float(const void *p, int64_t i) {
    if (DT == HBFP_F32) return reinterpret_cast<const float *>(p)[i];
    if (DT == HBFP_BF16) return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(p)[i] << 16);
    return (float)reinterpret_cast<const _Float16 *>(p)[i];
}
template <int DT>
__device__ __forceinline__ void store_float(void *p, int64_t i, float x) {
    if (DT == HBFP_F32) reinterpret_cast<float *>(p)[i] = x;
    else if (DT == HBFP_BF16) reinterpret_cast<__bf16 *>(p)[i] = (__bf16)x;
    else reinterpret_cast<_Float16 *>(p)[i] = (_Float16)x;
}
// eight consecutive elements from i on, of which n (may be <= 0) exist, the others 0.  Wide loads need no more than the elements' own
// alignment here.
typedef float v4f_at __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t v4u_at __attribute__((ext_vector_type(4), aligned(2)));
template <int DT>
__device__ __forceinline__ void load8(const void *p, int64_t i, int n, float *x) {
    if (n >= 8) {
        if (DT == HBFP_F32) {
            const v4f_at a = *reinterpret_cast<const v4f_at *>(reinterpret_cast<const float *>(p) + i);
            const v4f_at b = *reinterpret_cast<const v4f_at *>(reinterpret_cast<const float *>(p) + i + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = a[j], x[4 + j] = b[j];
        } else {
            const v4u_at a = *reinterpret_cast<const v4u_at *>(reinterpret_cast<const uint16_t *>(p) + i);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t h = j & 1 ? a[j / 2] >> 16 : a[j / 2] & 0xffffu;
                x[j] = DT == HBFP_BF16 ? __uint_as_float(h << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)h);
            }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < n ? load_as_float<DT>(p, i + j) : 0.0f;
}

template <int N>
__device__ __forceinline__ void load_words(const uint8_t *p, uint32_t (&w)[N]) {
    if (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const v4u x = reinterpret_cast<const v4u *>(p)[i];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[4 * i + k] = x[k];
        }
    } else if (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const v2u x = reinterpret_cast<const v2u *>(p)[i];
            w[2 * i] = x[0];
            w[2 * i + 1] = x[1];
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = reinterpret_cast<const uint32_t *>(p)[i];
    }
}

__device__ __forceinline__ uint32_t bf16_bits2(float a, float b) {
    const v2bf r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}
// four consecutive elements from i on, of which n (may be <= 0) exist
template <int DT>
__device__ __forceinline__ void store4(void *p, int64_t i, int n, const float *x) {
    typedef uint32_t v2u_at __attribute__((ext_vector_type(2), aligned(2)));
    if (n >= 4) {
        if (DT == HBFP_F32) {
            *reinterpret_cast<v4f_at *>(reinterpret_cast<float *>(p) + i) = v4f_at{x[0], x[1], x[2], x[3]};
        } else if (DT == HBFP_BF16) {
            *reinterpret_cast<v2u_at *>(reinterpret_cast<uint16_t *>(p) + i) = v2u_at{bf16_bits2(x[0], x[1]), bf16_bits2(x[2], x[3])};
        } else {
            typedef _Float16 v4h_at __attribute__((ext_vector_type(4), aligned(2)));
            *reinterpret_cast<v4h_at *>(reinterpret_cast<_Float16 *>(p) + i) = v4h_at{(_Float16)x[0], (_Float16)x[1], (_Float16)x[2], (_Float16)x[3]};
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < n) store_float<DT>(p, i + j, x[j]);
}
// x as a sum of N bf16 numbers, the first N * 8 bits of it: piece p of two values
template <int N>
__device__ __forceinline__ void bf16_pieces2(float a, float b, uint32_t *out) {
#pragma unroll
    for (int p = 0; p < N; ++p) {
        out[p] = bf16_bits2(a, b);
        a -= __uint_as_float(out[p] << 16);
        b -= __uint_as_float(out[p] & 0xffff0000u);
    }
}

// bf16 numbers a type's values are cut into (bf16 8 bits, FP16 11 bits, FP32 24 bits), and the softmax weights of its calls: 16 bits
// for bf16 and FP16, far below the one rounding of the output.  Weights of 8 bits put bf16 outputs 0.0017 to 0.0018 from 64 bits in the
// RMS, these 0.0016, which is the rounding alone; the second product costs twice as much (prompts 222 -> 289 us, one token for 32
// conversations 39 -> 43)
template <int DT> struct Pieces {
    static constexpr int n = DT == HBFP_F32 ? 3 : DT == HBFP_F16 ? 2 : 1, weights = DT == HBFP_F32 ? 3 : 2;
};

// largest of the lanes l, l ^ 16, l ^ 32, l ^ 48, and the sum: two exchanges of rows of lanes on the vector unit
__device__ __forceinline__ float max_over_rows(float x) {
    const v2u a = __builtin_bit_cast(v2u, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const v2u b = __builtin_bit_cast(v2u, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_over_rows(float x) {
    const v2u a = __builtin_bit_cast(v2u, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const v2u b = __builtin_bit_cast(v2u, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

}  // namespace
}  // namespace hbfp
