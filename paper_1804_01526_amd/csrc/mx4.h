// Microscaled 4-bit operands (layout and arithmetic in the public header): launchers, and the device side of the conversion.
#pragma once
#include "bfp_device.h"
#include "kv_cache.h"

namespace hbfp {

struct Mx4View {
    uint8_t *codes, *scales;
    int64_t rows, kdim, groups, scale_rows;
};

// mx4_quant.hip
int launch_quant_mx4(const void *src, int dtype, int64_t rows, int64_t cols, int64_t ld, int rounding, uint64_t seed, const Mx4View *along,
                     const Mx4View *down, hipStream_t s);
int launch_read_mx4(const Mx4View &t, int dtype, void *dst, int64_t ld, hipStream_t s);

// gemm_mx4.hip
struct Mx4Product {
    Mx4View a, b;
    const float *bias;
    void *y;
    int64_t ldy;
    int32_t dtype;
};
// whether a launch can hold the product's tiles
bool gemm_mx4_fits(int64_t M, int64_t N, int64_t groups);
size_t gemm_mx4_workspace(int64_t M, int64_t N, int64_t groups);
int launch_gemm_mx4(const Mx4Product &p, void *workspace, hipStream_t s);
// x converted inside the product: few tokens whose codes fit into LDS; p.a's buffers are not read
bool linear_mx4_fused_ok(int64_t M, int64_t N, int64_t groups);
int launch_linear_mx4_fused(const Mx4Product &p, const void *x, int64_t ldx, hipStream_t s);

// norm.hip
struct NormArgs {
    hbfp_norm n;
    int8_t *codes;               // int8 rows of kpad bytes and a scale each, or
    float *scales;
    int64_t kpad;
    Mx4View mx4;                 // (codes NULL)
};
int launch_norm(const NormArgs &a, hipStream_t s);
struct NormGradArgs {
    const void *g, *sum, *g_sum;
    const float *rstd, *weight;
    void *dx;
    float *dweight, *partial;
    int64_t ldg, ld_sum, ld_g_sum, ldx, rows, cols;
    int32_t dtype;
};
size_t norm_grad_workspace(int64_t rows, int64_t cols);
int launch_norm_grad(const NormGradArgs &a, hipStream_t s);

namespace {

// One dimension of a launch has fewer than 2^32 threads: more than 2^21 workgroups go in rows of that many, and those behind the last find
// nothing to do.
constexpr int kGridBits = 21;
inline dim3 grid_of(int64_t wgs) {
    return wgs <= 1 << kGridBits ? dim3((unsigned)wgs) : dim3(1u << kGridBits, (unsigned)ceil_div(wgs, (int64_t)1 << kGridBits));
}
__device__ __forceinline__ uint32_t workgroup() { return (blockIdx.y << kGridBits) + blockIdx.x; }
// launches whose workgroups are counted otherwise have to fit into one row
inline bool one_row(int64_t wgs, int threads) { return wgs * threads <= 0xffffffffll; }

// the byte of a block from the bit pattern of its largest magnitude: adding what rounds up carries into the exponent field
template <int ROUND>
__device__ __forceinline__ uint32_t mx4_byte(uint32_t amax) {
    if (amax >= 0x7f800000u) return 255u;
    uint32_t e = (amax + (ROUND == HBFP_RNE ? 0x200000u : 0x3fffffu)) >> 23;
    e = e > 254u ? 254u : e;
    return e < 2u ? 0u : e - 2u;
}

// eight values -> a word of codes, four or two -> a half or a quarter of one, to nearest.  The instruction divides by a power of two of which it reads the exponent field alone
// (0: 2^-127), rounds to nearest even and cuts at 6; the builtin writes one byte of the word.
template <int C>
__device__ __forceinline__ uint32_t mx4_codes(const float *x, uint32_t byte) {
    const float unit = __uint_as_float(byte << 23);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], unit, 0);
    if constexpr (C >= 4) w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], unit, 1);
    if constexpr (C == 8) {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], unit, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], unit, 3);
    }
    return byte == 255u ? 0u : w;
}

// ... stochastically.  From two units up a step is the second bit of the significand, whatever the exponent, so that the code is the upper bits of
// the number itself after the word's top 22 bits are added below; exponent and bit count the codes from 4 on.  Below, a step is half a unit: the
// fraction of 2 |x| times 2^32, cut to an integer, decides as the exact one does, h being an integer.  (What |x| in units loses when it leaves
// FP32's range is far below 2^-32.)
__device__ __forceinline__ uint32_t mx4_code_sr(float x, uint32_t byte, uint32_t h) {
    const uint32_t bits = __float_as_uint(x) & 0x7fffffffu;
    const uint32_t high = ((bits + (h >> 10)) >> 22) + 2u - 2u * byte;
    const float a = __builtin_amdgcn_ldexpf(__builtin_fabsf(x), 128 - (int)byte);
    const uint32_t frac = (uint32_t)__builtin_amdgcn_ldexpf(__builtin_amdgcn_fractf(a), 32);
    const uint32_t low = (uint32_t)a + ((frac + h) < h ? 1u : 0u);
    uint32_t code = a >= 4.0f ? high : low;
    code = code > 7u ? 7u : code;
    return code | ((__float_as_uint(x) >> 28) & 8u);
}

// a word of eight codes -> the values, or pairs of bf16: exact, subnormal results included; the conversion reads the exponent field of its scale
// alone (0: 2^-127, 255: NaN)
__device__ __forceinline__ void mx4_values8(uint32_t w, uint32_t byte, float *x) {
    const float unit = __uint_as_float(byte << 23);
    const v2f a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 1);
    const v2f c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 3);
    x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1], x[4] = c[0], x[5] = c[1], x[6] = d[0], x[7] = d[1];
}
__device__ __forceinline__ v4u mx4_bf16_8(uint32_t w, uint32_t byte) {
    const float unit = __uint_as_float(byte << 23);
    return v4u{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 3))};
}

// largest magnitude of eight values, as bits (a NaN is larger than everything)
__device__ __forceinline__ uint32_t mx4_largest8(const float *x) {
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = __float_as_uint(x[i]) & 0x7fffffffu;
        amax = a > amax ? a : amax;
    }
    return amax;
}
// ... of four neighbouring lanes: a block of 32
__device__ __forceinline__ uint32_t largest_of_quad(uint32_t a) {
    uint32_t b = (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0xB1, 0xF, 0xF, true);      // lanes 1, 0, 3, 2
    a = b > a ? b : a;
    b = (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0x4E, 0xF, 0xF, true);               // lanes 2, 3, 0, 1
    return b > a ? b : a;
}

}  // namespace
}  // namespace hbfp
