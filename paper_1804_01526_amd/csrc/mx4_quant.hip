// Conversion of a matrix into microscaled 4-bit operands, along its rows, down its columns or both from one read, and back.
// Bound by memory: a value costs its bytes once and 17/32 byte for each operand.
#include "mx4.h"

namespace hbfp {
namespace {

struct QuantMx4Params {
    const void *src;
    int64_t rows, cols, ld;
    uint32_t s0, s1;
    Mx4View along, down;
    uint32_t tiles_c;            // tiles along the source's columns
};

template <int ROUND>
__device__ __forceinline__ uint32_t codes8(const float *x, uint32_t byte, int64_t idx, const QuantMx4Params &p) {
    if constexpr (ROUND == HBFP_RNE) {
        return mx4_codes8(x, byte);
    } else {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint64_t at = (uint64_t)idx + i;
            w |= mx4_code_sr(x[i], 127 - (int)byte, sr_hash((uint32_t)at, (uint32_t)(at >> 32), p.s0, p.s1)) << (4 * i);
        }
        return byte == 255u ? 0u : w;
    }
}

// ---- along the rows alone.  A workgroup has 32 rows of one group of 256: a thread converts 8 neighbours of 4 rows, all loads first;
// four lanes are a block, 32 lanes a line of codes.
template <int DT, int ROUND>
__global__ __launch_bounds__(256) void quant_mx4_along_kernel(const QuantMx4Params p) {
    const int t = threadIdx.x;
    const int64_t group = blockIdx.x % p.tiles_c, r0 = (int64_t)(blockIdx.x / p.tiles_c) * 32 + t / 32;
    const int64_t c = group * 256 + 8 * (t % 32);
    const int64_t left = p.cols - c;
    float x[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t r = r0 + 8 * i;
        load8<DT>(p.src, r * p.ld + c, r >= p.rows || left <= 0 ? 0 : left < 8 ? (int)left : 8, x[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t r = r0 + 8 * i;
        const uint32_t byte = mx4_byte<ROUND>(largest_of_quad(mx4_largest8(x[i])));
        const uint32_t w = codes8<ROUND>(x[i], byte, r * p.cols + c, p);
        if (r >= p.rows) continue;
        reinterpret_cast<uint32_t *>(p.along.codes + (group * p.rows + r) * 128)[t % 32] = w;
        if (t % 4 == 0) p.along.scales[(group * p.along.scale_rows + r) * 8 + (t % 32) / 4] = (uint8_t)byte;
    }
}

// ---- down the columns, or both.  A workgroup has a tile of 128 x 128: it converts along the rows from the registers that the values were
// loaded into, and down the columns from LDS, where a thread reads two neighbouring columns of 32 rows (a wave reads whole rows).
template <int DT>
struct Tile {
    static constexpr int kSize = DT == HBFP_F32 ? 4 : 2;
    static constexpr int kBytes = 128 * 128 * kSize;
};
template <int DT, int ROUND, bool ALONG>
__global__ __launch_bounds__(256) void quant_mx4_down_kernel(const QuantMx4Params p) {
    extern __shared__ __attribute__((aligned(16))) uint8_t tile[];
    const int t = threadIdx.x;
    const int64_t c0 = (int64_t)(blockIdx.x % p.tiles_c) * 128, r0 = (int64_t)(blockIdx.x / p.tiles_c) * 128;
    {
        const int64_t c = c0 + 8 * (t % 16), left = p.cols - c;
        float x[8][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t r = r0 + t / 16 + 16 * i;
            load8<DT>(p.src, r * p.ld + c, r >= p.rows || left <= 0 ? 0 : left < 8 ? (int)left : 8, x[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int at = (t / 16 + 16 * i) * 128 + 8 * (t % 16);
            if constexpr (DT == HBFP_F32) {
                v4f *to = reinterpret_cast<v4f *>(tile + 4 * at);
                to[0] = v4f{x[i][0], x[i][1], x[i][2], x[i][3]};
                to[1] = v4f{x[i][4], x[i][5], x[i][6], x[i][7]};
            } else {
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if constexpr (DT == HBFP_BF16) w[k] = __float_as_uint(x[i][2 * k]) >> 16 | (__float_as_uint(x[i][2 * k + 1]) & 0xffff0000u);
                    else
                        w[k] = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x[i][2 * k]) |
                               (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x[i][2 * k + 1]) << 16;
                }
                *reinterpret_cast<v4u *>(tile + 2 * at) = v4u{w[0], w[1], w[2], w[3]};
            }
        }
        if constexpr (ALONG) {
            const int64_t group = c0 >> 8;
            if (group < p.along.groups) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int64_t r = r0 + t / 16 + 16 * i;
                    const uint32_t byte = mx4_byte<ROUND>(largest_of_quad(mx4_largest8(x[i])));
                    const uint32_t w = codes8<ROUND>(x[i], byte, r * p.cols + c, p);
                    if (r >= p.rows) continue;
                    reinterpret_cast<uint32_t *>(p.along.codes + (group * p.rows + r) * 128 + ((c0 & 255) >> 1))[t % 16] = w;
                    if (t % 4 == 0) p.along.scales[(group * p.along.scale_rows + r) * 8 + ((c0 & 255) >> 5) + (t % 16) / 4] = (uint8_t)byte;
                }
            }
        }
    }
    __syncthreads();
    const int64_t k0 = r0 + 32 * (t / 64), group = k0 >> 8;          // (a wave has one block of 32 rows)
    if (group >= p.down.groups) return;
    const int cc = 2 * (t % 64);
    float x[2][32];
    const uint8_t *from = tile + ((t / 64) * 32 * 128 + cc) * Tile<DT>::kSize;
#pragma unroll
    for (int k = 0; k < 32; ++k) {
        if constexpr (DT == HBFP_F32) {
            const v2f two = *reinterpret_cast<const v2f *>(from + k * 512);
            x[0][k] = two[0];
            x[1][k] = two[1];
        } else {
            const uint32_t two = *reinterpret_cast<const uint32_t *>(from + k * 256);
            if constexpr (DT == HBFP_BF16) {
                x[0][k] = __uint_as_float(two << 16);
                x[1][k] = __uint_as_float(two & 0xffff0000u);
            } else {
                x[0][k] = (float)__builtin_bit_cast(_Float16, (uint16_t)two);
                x[1][k] = (float)__builtin_bit_cast(_Float16, (uint16_t)(two >> 16));
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t c = c0 + cc + j;
        if (c >= p.cols) continue;
        uint32_t amax = 0;
#pragma unroll
        for (int k = 0; k < 32; k += 8) {
            const uint32_t a = mx4_largest8(x[j] + k);
            amax = a > amax ? a : amax;
        }
        const uint32_t byte = mx4_byte<ROUND>(amax);
        v4u w;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (ROUND == HBFP_RNE) {
                w[k] = mx4_codes8(x[j] + 8 * k, byte);
            } else {
                w[k] = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint64_t at = (uint64_t)(k0 + 8 * k + i) * (uint64_t)p.cols + (uint64_t)c;
                    w[k] |= mx4_code_sr(x[j][8 * k + i], 127 - (int)byte, sr_hash((uint32_t)at, (uint32_t)(at >> 32), p.s0, p.s1)) << (4 * i);
                }
                if (byte == 255u) w[k] = 0;
            }
        }
        *reinterpret_cast<v4u *>(p.down.codes + (group * p.cols + c) * 128 + ((k0 & 255) >> 1)) = w;
        p.down.scales[(group * p.down.scale_rows + c) * 8 + ((k0 & 255) >> 5)] = (uint8_t)byte;
    }
}

template <int DT, int ROUND>
int launch_quant(QuantMx4Params p, bool along, bool down, hipStream_t s) {
    if (!down) {
        p.tiles_c = (uint32_t)p.along.groups;
        const int64_t wgs = p.along.groups * ceil_div(p.rows, 32);
        if (wgs > 0x7fffffff) return HBFP_ERR_ARG;
        hipLaunchKernelGGL((quant_mx4_along_kernel<DT, ROUND>), dim3((unsigned)wgs), dim3(256), 0, s, p);
        return launch_status();
    }
    // whole groups of whichever operands are wanted: what is past the source is stored as zeros
    const int64_t tiles_c = along ? 2 * p.along.groups : ceil_div(p.cols, 128), tiles_r = 2 * p.down.groups;
    const int64_t wgs = tiles_c * tiles_r;
    if (wgs > 0x7fffffff) return HBFP_ERR_ARG;
    p.tiles_c = (uint32_t)tiles_c;
    void (*const kernel)(QuantMx4Params) = along ? &quant_mx4_down_kernel<DT, ROUND, true> : &quant_mx4_down_kernel<DT, ROUND, false>;
    static std::atomic<bool> configured[2];
    if (allow_dynamic_lds(configured[along], reinterpret_cast<const void *>(kernel), Tile<DT>::kBytes) != HBFP_OK) return HBFP_ERR_LAUNCH;
    hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(256), Tile<DT>::kBytes, s, p);
    return launch_status();
}

// ---- back: a thread has a word of eight codes
template <int DT>
__global__ __launch_bounds__(256) void read_mx4_kernel(const Mx4View t, void *dst, int64_t ld, uint32_t words) {
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t r = e / words;
    const int64_t k = 8 * (e - r * words);
    if (r >= t.rows) return;
    const uint32_t w = *reinterpret_cast<const uint32_t *>(t.codes + ((k >> 8) * t.rows + r) * 128 + ((k & 255) >> 1));
    const int byte = t.scales[((k >> 8) * t.scale_rows + r) * 8 + ((k & 255) >> 5)];
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t c = (w >> (4 * i)) & 7u;
        const float half = (float)((0xC8643210u >> (4 * c)) & 15u);             // the magnitude in halves: 0 1 2 3 4 6 8 12
        const float v = byte == 255 ? __builtin_nanf("") : __builtin_amdgcn_ldexpf(half, byte - 128);
        x[i] = (w >> (4 * i)) & 8u ? -v : v;
    }
    const int64_t left = t.kdim - k;
    store4<DT>(dst, r * ld + k, left < 4 ? (int)left : 4, x);
    store4<DT>(dst, r * ld + k + 4, left < 8 ? (int)left - 4 : 4, x + 4);
}

template <int DT>
int launch_quant_of(const QuantMx4Params &p, int rounding, bool along, bool down, hipStream_t s) {
    return rounding == HBFP_RNE ? launch_quant<DT, HBFP_RNE>(p, along, down, s) : launch_quant<DT, HBFP_STOCHASTIC>(p, along, down, s);
}

}  // namespace

int launch_quant_mx4(const void *src, int dtype, int64_t rows, int64_t cols, int64_t ld, int rounding, uint64_t seed, const Mx4View *along,
                     const Mx4View *down, hipStream_t s) {
    QuantMx4Params p = {src, rows, cols, ld, (uint32_t)seed, (uint32_t)(seed >> 32), {}, {}, 0};
    if (along) p.along = *along;
    if (down) p.down = *down;
    return dtype == HBFP_F32    ? launch_quant_of<HBFP_F32>(p, rounding, along, down, s)
           : dtype == HBFP_BF16 ? launch_quant_of<HBFP_BF16>(p, rounding, along, down, s)
                                : launch_quant_of<HBFP_F16>(p, rounding, along, down, s);
}

int launch_read_mx4(const Mx4View &t, int dtype, void *dst, int64_t ld, hipStream_t s) {
    const int64_t words = ceil_div(t.kdim, 8), wgs = ceil_div(words * t.rows, 256);
    if (wgs > 0x7fffffff) return HBFP_ERR_ARG;
    if (dtype == HBFP_F32) hipLaunchKernelGGL(read_mx4_kernel<HBFP_F32>, dim3((unsigned)wgs), dim3(256), 0, s, t, dst, ld, (uint32_t)words);
    else hipLaunchKernelGGL(read_mx4_kernel<HBFP_BF16>, dim3((unsigned)wgs), dim3(256), 0, s, t, dst, ld, (uint32_t)words);
    return launch_status();
}

}  // namespace hbfp
