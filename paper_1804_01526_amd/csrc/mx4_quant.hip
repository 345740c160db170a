// Conversion of a matrix into microscaled 4-bit operands, along its rows, down its columns or both from one read, and back.
// Bound by memory: a value costs its bytes once and 17/32 byte for each operand.  4096 x 4096 along the rows: bf16 8.9 us (4.8 TB/s), FP32 12.9
// (5.9); down the columns 10.1 and 14.3; both 13.7 and 17.1 (3.8 and 5.0), where the two calls would take 19.0 and 27.2.  Stochastic rounding is bound
// by the vector unit, 54 instructions a value for both operands, two of them 32-bit multiplications at a quarter of the rate: bf16 along
// 18.7 us, both 31.
#include "mx4.h"

namespace hbfp {
namespace {

struct QuantMx4Params {
    const void *src;
    int64_t rows, cols, ld;
    uint32_t s0, s1;
    Mx4View along, down;
    uint32_t tiles_c, tiles;     // tiles along the source's columns, all tiles
    int32_t eights;              // rows of a multiple of eight values
};

// the random words of C neighbours from position `at` on.  Where rows are multiples of eight, `at` is one of C, and the hash's first steps, which are
// linear over bits, are taken once for all of them (4096 x 4096 bf16 along 21.8 -> 19.8 us, both 33.8 -> 31.7, with four rows a thread)
template <int C>
__device__ __forceinline__ void random_words(uint64_t at, const QuantMx4Params &p, uint32_t *h) {
    if (p.eights) {
        const uint32_t first = sr_triple((uint32_t)at ^ p.s0), high = (uint32_t)(at >> 32) ^ p.s1;
#pragma unroll
        for (int i = 0; i < C; ++i) h[i] = sr_hash_tail(first ^ sr_triple(i), high);
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i) h[i] = sr_hash((uint32_t)(at + i), (uint32_t)((at + i) >> 32), p.s0, p.s1);
    }
}

template <int ROUND>
__device__ __forceinline__ uint32_t codes8(const float *x, uint32_t byte, int64_t idx, const QuantMx4Params &p) {
    if constexpr (ROUND == HBFP_RNE) {
        return mx4_codes<8>(x, byte);
    } else {
        uint32_t w = 0, h[8];
        random_words<8>((uint64_t)idx, p, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) w |= mx4_code_sr(x[i], byte, h[i]) << (4 * i);
        return byte == 255u ? 0u : w;
    }
}

// ---- along the rows alone.  A workgroup has 8 N rows of one group of 256: a thread converts 8 neighbours of N rows, all loads first;
// four lanes are a block, 32 lanes a line of codes.
template <int DT, int ROUND, int N>
__global__ __launch_bounds__(256) void quant_mx4_along_kernel(const QuantMx4Params p) {
    const int t = threadIdx.x;
    const int64_t group = workgroup() % p.tiles_c, r0 = (int64_t)(workgroup() / p.tiles_c) * (8 * N) + t / 32;
    const int64_t c = group * 256 + 8 * (t % 32);
    const int64_t left = p.cols - c;
    float x[N][8];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int64_t r = r0 + 8 * i;
        load8<DT>(p.src, r * p.ld + c, r >= p.rows || left <= 0 ? 0 : left < 8 ? (int)left : 8, x[i]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int64_t r = r0 + 8 * i;
        const uint32_t byte = mx4_byte<ROUND>(largest_of_quad(mx4_largest8(x[i])));
        const uint32_t w = codes8<ROUND>(x[i], byte, r * p.cols + c, p);
        if (r >= p.rows) continue;
        reinterpret_cast<uint32_t *>(p.along.codes + (group * p.rows + r) * 128)[t % 32] = w;
        if (t % 4 == 0) p.along.scales[(group * p.along.scale_rows + r) * 8 + (t % 32) / 4] = (uint8_t)byte;
    }
}

// ---- down the columns, or both.  A workgroup has a tile of 128 rows and 16 C columns, a thread 8 rows and C columns of it: 32 / C neighbouring lanes
// share the blocks along its rows, and the four lanes 16 apart of a wave those down its columns, so that both maxima are found between lanes and a random
// word serves both codes of its value (with values that meet in LDS and are rounded by each side for itself, stochastic 4096 x 4096 took 44 us, 1001 x 777
// 31 instead of 13).  The words of the columns meet in LDS, from where four threads store 64 bytes of a column's codes.  The writes there are free of
// conflicts; of the reads, 16 bytes a lane, every fourth row's end meets the banks of the first: 0.57 cycles of conflict for each cycle of an access.

// largest of the lanes l, l ^ 16, l ^ 32, l ^ 48: two exchanges of rows of lanes on the vector unit
__device__ __forceinline__ uint32_t largest_of_column(uint32_t x) {
    const v2u a = __builtin_bit_cast(v2u, __builtin_amdgcn_permlane32_swap(x, x, false, false));
    x = a[0] > a[1] ? a[0] : a[1];
    const v2u b = __builtin_bit_cast(v2u, __builtin_amdgcn_permlane16_swap(x, x, false, false));
    return b[0] > b[1] ? b[0] : b[1];
}
// ... of the 32 / C neighbouring lanes of a block
template <int C>
__device__ __forceinline__ uint32_t largest_of_block(uint32_t x) {
    x = largest_of_quad(x);
    if constexpr (C <= 4) {
        const uint32_t y = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xF, 0xF, true);      // lanes 7, 6, ... 0
        x = y > x ? y : x;
    }
    if constexpr (C == 2) {
        const uint32_t y = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x140, 0xF, 0xF, true);      // lanes 15, 14, ... 0
        x = y > x ? y : x;
    }
    return x;
}

// C neighbours from element i on, of which n (may be <= 0) exist
template <int DT, int C>
__device__ __forceinline__ void load_some(const void *p, int64_t i, int64_t n, float *x) {
    if constexpr (C == 8) {
        load8<DT>(p, i, n < 0 ? 0 : n < 8 ? (int)n : 8, x);
    } else if (n < C) {
#pragma unroll
        for (int j = 0; j < C; ++j) x[j] = j < n ? load_as_float<DT>(p, i + j) : 0.0f;
    } else if constexpr (DT == HBFP_F32) {
        typedef float floats_at __attribute__((ext_vector_type(C), aligned(4)));
        const floats_at a = *reinterpret_cast<const floats_at *>(reinterpret_cast<const float *>(p) + i);
#pragma unroll
        for (int j = 0; j < C; ++j) x[j] = a[j];
    } else {
        typedef uint16_t halves_at __attribute__((ext_vector_type(C), aligned(2)));
        const halves_at a = *reinterpret_cast<const halves_at *>(reinterpret_cast<const uint16_t *>(p) + i);
#pragma unroll
        for (int j = 0; j < C; ++j) x[j] = DT == HBFP_BF16 ? __uint_as_float((uint32_t)a[j] << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)a[j]);
    }
}
template <int C>
__device__ __forceinline__ uint32_t largest_of(const float *x) {
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const uint32_t a = __float_as_uint(x[i]) & 0x7fffffffu;
        amax = a > amax ? a : amax;
    }
    return amax;
}

template <int DT, int ROUND, bool ALONG, int C>
__global__ __launch_bounds__(256, ALONG && ROUND == HBFP_STOCHASTIC && C == 8 ? 3 : 4) void quant_mx4_down_kernel(const QuantMx4Params p) {
    constexpr int kWide = 16 * C;
    __shared__ __attribute__((aligned(16))) uint32_t words[kWide][20];   // 16 of column C a + b in row 16 b + a: a wave's writes cover all banks
    const int t = threadIdx.x, lane = t & 63, tr = t / 16;
    // workgroups are dealt to the 8 XCDs in turn: each gets a run of tiles, two rows of them side by side, so that the halves of a line of codes
    // of either operand meet in one L2 (16384 x 16384 bf16, both: 219 us by rows of tiles over all XCDs, 190 so; 4096 x 4096 13.4 and 13.7)
    const uint32_t tile = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
    if (tile >= p.tiles) return;
    const uint32_t band = tile / (2 * p.tiles_c), in_band = tile - band * 2 * p.tiles_c;
    const int64_t c0 = (int64_t)(in_band >> 1) * kWide, r0 = ((int64_t)band * 2 + (in_band & 1)) * 128;
    const int64_t c = c0 + C * (t % 16), r = r0 + 8 * tr, left = p.cols - c;
    float x[8][C];
#pragma unroll
    for (int i = 0; i < 8; ++i) load_some<DT, C>(p.src, (r + i) * p.ld + c, r + i >= p.rows ? 0 : left, x[i]);
    uint32_t down[C];                                       // bytes of the columns' blocks
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const float y[8] = {x[0][j], x[1][j], x[2][j], x[3][j], x[4][j], x[5][j], x[6][j], x[7][j]};
        down[j] = mx4_byte<ROUND>(largest_of_column(mx4_largest8(y)));
    }
    uint32_t column[C];
#pragma unroll
    for (int j = 0; j < C; ++j) column[j] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        // one row after the other: side by side they would take 256 registers
        __builtin_amdgcn_sched_barrier(0);
        uint64_t at = (uint64_t)(r + i) * (uint64_t)p.cols + (uint64_t)c;
        asm volatile("" : "+v"(at));
#pragma unroll
        for (int j = 0; j < C; ++j) asm volatile("" : "+v"(x[i][j]));
        uint32_t byte = 0, w = 0;
        if constexpr (ALONG) byte = mx4_byte<ROUND>(largest_of_block<C>(largest_of<C>(x[i])));
        if constexpr (ROUND == HBFP_RNE) {
            if constexpr (ALONG) w = mx4_codes<C>(x[i], byte);
        } else {
            uint32_t h[C];
            random_words<C>(at, p, h);
#pragma unroll
            for (int j = 0; j < C; ++j) {
                if constexpr (ALONG) w |= mx4_code_sr(x[i][j], byte, h[j]) << (4 * j);
                column[j] |= mx4_code_sr(x[i][j], down[j], h[j]) << (4 * i);
            }
            if (byte == 255u) w = 0;
#pragma unroll
            for (int j = 0; j < C; ++j) asm volatile("" : "+v"(column[j]));
            asm volatile("" : "+v"(w));
        }
        if constexpr (ALONG) {
            if (r + i < p.rows) {
                uint8_t *const line = p.along.codes + ((c0 >> 8) * p.rows + r + i) * 128 + ((c0 & 255) >> 1);
                if constexpr (C == 8) reinterpret_cast<uint32_t *>(line)[t % 16] = w;
                else if constexpr (C == 4) reinterpret_cast<uint16_t *>(line)[t % 16] = (uint16_t)w;
                else line[t % 16] = (uint8_t)w;
                if (t % (32 / C) == 0)
                    p.along.scales[((c0 >> 8) * p.along.scale_rows + r + i) * 8 + ((c0 & 255) >> 5) + (t % 16) / (32 / C)] = (uint8_t)byte;
            }
        }
    }
    const int64_t group = r0 >> 8;
#pragma unroll
    for (int j = 0; j < C; ++j) {
        if constexpr (ROUND == HBFP_RNE) {
            const float y[8] = {x[0][j], x[1][j], x[2][j], x[3][j], x[4][j], x[5][j], x[6][j], x[7][j]};
            column[j] = mx4_codes<8>(y, down[j]);
        } else {
            if (down[j] == 255u) column[j] = 0;
        }
        words[16 * j + t % 16][tr] = column[j];
        if (lane < 16 && c + j < p.cols) p.down.scales[(group * p.down.scale_rows + c + j) * 8 + ((r0 & 255) >> 5) + t / 64] = (uint8_t)down[j];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < (C + 2) / 4; ++i) {
        const int col = C * (lane / 4) + t / 64 + 4 * i;     // (columns C apart: neighbouring rows of words, 20 banks from one to the next)
        if ((C > 2 || t < 128) && c0 + col < p.cols)
            *reinterpret_cast<v4u *>(p.down.codes + (group * p.cols + c0 + col) * 128 + ((r0 & 255) >> 1) + 16 * (t % 4)) =
                *reinterpret_cast<const v4u *>(&words[16 * (col % C) + col / C][4 * (t % 4)]);
    }
}

template <int DT, int ROUND, int C>
int launch_down(QuantMx4Params p, bool along, hipStream_t s) {
    // whole groups of whichever operands are wanted: what is past the source is stored as zeros
    const int64_t tiles_c = along ? 16 / C * p.along.groups : ceil_div(p.cols, 16 * C), wgs = tiles_c * 2 * p.down.groups;
    if (!one_row(round_up(wgs, 8), 256)) return HBFP_ERR_ARG;
    p.tiles_c = (uint32_t)tiles_c;
    p.tiles = (uint32_t)wgs;
    void (*const kernel)(QuantMx4Params) = along ? &quant_mx4_down_kernel<DT, ROUND, true, C> : &quant_mx4_down_kernel<DT, ROUND, false, C>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)round_up(wgs, 8)), dim3(256), 0, s, p);
    return launch_status();
}

// Rows of a thread, of the kernels that go along the rows: one where they are few, else two, a compromise between the conversions and reading back: four are
// ahead to nearest at 4096 x 4096, two at 8192 x 8192 and for reading back from 8192 x 8192 on.  us with 1, 2 and 4, conversion to nearest and stochastically and
// reading back, of bf16: 64 x 4096 3.1, 3.3, 3.6; 3.4, 3.9, 5.2; 2.9, 3.0, 3.2; 1024 x 1024 (512 workgroups of one row a thread) 3.0, 3.2, 3.7; 4.0, 4.1, 5.3; 3.1,
// 3.2, 3.5; 512 x 8192 3.9, 3.9, 4.1; 7.9, 6.6, 7.1; 4.3, 4.4, 4.5; 4096 x 4096 9.5, 8.9, 8.2; 23.3, 18.7, 19.5; 8.5, 8.5, 8.4; 8192 x 8192 -, 26.2, 32.0;
// -, 59.0, 62.2; 26.5, 26.5, 29.0; 16384 x 16384 -, 112, 115; -, 225, 223; 168, 129, 135
bool few_lines(const Mx4View &t) { return t.groups * ceil_div(t.rows, 8) <= 512; }

template <int DT, int ROUND, int N>
int launch_along(QuantMx4Params p, hipStream_t s) {
    p.tiles_c = (uint32_t)p.along.groups;
    const int64_t wgs = p.along.groups * ceil_div(p.rows, 8 * N);
    if (wgs > 0x7fffffff) return HBFP_ERR_ARG;
    hipLaunchKernelGGL((quant_mx4_along_kernel<DT, ROUND, N>), grid_of(wgs), dim3(256), 0, s, p);
    return launch_status();
}

// Columns of a thread: fewer where the matrix has too few tiles to keep the chip's vector units busy.  us with 8, 4 and 2 of both operands, stochastic (bf16):
// 501 x 730 13.8, 9.1, 6.9; 1024 x 1024 (64 tiles) 11.0, 7.8, 6.7; 1024 x 2048 11.2, 8.1, 8.1; 2048 x 2048 12.0, 11.1, 11.7; 2048 x 4096 17.3, 17.1;
// 4096 x 4096 30.4, 30.9; to nearest 6.1, 5.3, 5.1 of 1024 x 1024, 8.1, 8.1 of 2048 x 4096, 13.1, 14.0 of 4096 x 4096
int down_columns(const QuantMx4Params &p, bool along) {
    const int64_t tiles = (along ? 2 * p.along.groups : ceil_div(p.cols, 128)) * 2 * p.down.groups;
    return tiles <= 64 ? 2 : tiles <= 512 ? 4 : 8;
}
template <int DT, int ROUND>
int launch_quant(QuantMx4Params p, bool along, bool down, hipStream_t s) {
    if (!down) {
        return few_lines(p.along) ? launch_along<DT, ROUND, 1>(p, s) : launch_along<DT, ROUND, 2>(p, s);
    }
    const int wide = down_columns(p, along);
    return wide == 2 ? launch_down<DT, ROUND, 2>(p, along, s) : wide == 4 ? launch_down<DT, ROUND, 4>(p, along, s) : launch_down<DT, ROUND, 8>(p, along, s);
}

// ---- back.  A workgroup has 8 N rows of one group; a thread a word of eight codes in N of them, all loads first.  8192 x 4096 as bf16: 14.5 us, 5.9 TB/s.
template <int DT, int N>
__global__ __launch_bounds__(256) void read_mx4_kernel(const Mx4View t, void *dst, int64_t ld) {
    const int64_t group = workgroup() % (uint32_t)t.groups, r0 = (int64_t)(workgroup() / (uint32_t)t.groups) * (8 * N) + threadIdx.x / 32;
    const int at = threadIdx.x % 32;
    const int64_t k = group * 256 + 8 * at, left = t.kdim - k;
    if (left <= 0) return;
    uint32_t w[N], byte[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int64_t r = r0 + 8 * i < t.rows ? r0 + 8 * i : t.rows - 1;
        w[i] = reinterpret_cast<const uint32_t *>(t.codes + (group * t.rows + r) * 128)[at];
        byte[i] = t.scales[(group * t.scale_rows + r) * 8 + at / 4];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int64_t r = r0 + 8 * i;
        if (r >= t.rows) return;
        if (DT == HBFP_BF16 && left >= 8) {
            *reinterpret_cast<v4u_at *>(reinterpret_cast<uint16_t *>(dst) + r * ld + k) = mx4_bf16_8(w[i], byte[i]);
            continue;
        }
        float x[8];
        mx4_values8(w[i], byte[i], x);
        store4<DT>(dst, r * ld + k, left < 4 ? (int)left : 4, x);
        store4<DT>(dst, r * ld + k + 4, left < 8 ? (int)left - 4 : 4, x + 4);
    }
}

template <int DT, int N>
int launch_read(const Mx4View &t, void *dst, int64_t ld, hipStream_t s) {
    const int64_t wgs = t.groups * ceil_div(t.rows, 8 * N);
    if (wgs > 0x7fffffff) return HBFP_ERR_ARG;
    hipLaunchKernelGGL((read_mx4_kernel<DT, N>), grid_of(wgs), dim3(256), 0, s, t, dst, ld);
    return launch_status();
}
template <int DT>
int launch_read_of(const Mx4View &t, void *dst, int64_t ld, hipStream_t s) {
    return few_lines(t) ? launch_read<DT, 1>(t, dst, ld, s) : launch_read<DT, 2>(t, dst, ld, s);
}

template <int DT>
int launch_quant_of(const QuantMx4Params &p, int rounding, bool along, bool down, hipStream_t s) {
    return rounding == HBFP_RNE ? launch_quant<DT, HBFP_RNE>(p, along, down, s) : launch_quant<DT, HBFP_STOCHASTIC>(p, along, down, s);
}

}  // namespace

int launch_quant_mx4(const void *src, int dtype, int64_t rows, int64_t cols, int64_t ld, int rounding, uint64_t seed, const Mx4View *along,
                     const Mx4View *down, hipStream_t s) {
    QuantMx4Params p = {src, rows, cols, ld, (uint32_t)seed, (uint32_t)(seed >> 32), {}, {}, 0, 0, cols % 8 == 0};
    if (along) p.along = *along;
    if (down) p.down = *down;
    return dtype == HBFP_F32    ? launch_quant_of<HBFP_F32>(p, rounding, along, down, s)
           : dtype == HBFP_BF16 ? launch_quant_of<HBFP_BF16>(p, rounding, along, down, s)
                                : launch_quant_of<HBFP_F16>(p, rounding, along, down, s);
}

int launch_read_mx4(const Mx4View &t, int dtype, void *dst, int64_t ld, hipStream_t s) {
    return dtype == HBFP_F32 ? launch_read_of<HBFP_F32>(t, dst, ld, s) : launch_read_of<HBFP_BF16>(t, dst, ld, s);
}

}  // namespace hbfp
