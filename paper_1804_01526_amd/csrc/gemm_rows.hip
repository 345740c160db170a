// Products in 8-bit integers with an FP32 scale per row of each operand:
//     y[m][n] = (sum_k a[m][k] b[n][k]) * sa[m] * sb[n] + bias[n]
// The sum is an exact int32 whatever its order; scales and bias are FP32 and y is rounded once.
#include "gemm_wide.h"
#include "kv_cache.h"

namespace hbfp {
namespace {

// ---- rows -> codes.  A workgroup has one row; it reads the row twice, the second time from the caches.
struct QuantParams {
    const void *src;
    int8_t *codes;
    float *scales;
    int64_t cols, ld, kpad;
    int32_t wide;
};

__device__ __forceinline__ float row_scale(uint32_t amax) { return __uint_as_float(amax) * (1.0f / 127.0f); }
__device__ __forceinline__ uint32_t code_of(float x, float scale) {
    const float q = __builtin_rintf(x / scale);
    return (uint32_t)(int)fminf(fmaxf(q, -127.0f), 127.0f) & 0xffu;
}

template <int DT>
__global__ __launch_bounds__(256) void quant_rows_kernel(const QuantParams p) {
    __shared__ uint32_t top[4];
    const int64_t row = blockIdx.x, base = row * p.ld;
    const int t = threadIdx.x;
    uint32_t amax = 0;
    for (int64_t c = 8 * t; c < p.cols; c += 2048) {
        float x[8];
        const int64_t left = p.cols - c;
        load8<DT>(p.src, base + c, left < 8 ? (int)left : 8, left >= 8 && p.wide, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t a = __float_as_uint(x[i]) & 0x7fffffffu;
            amax = a > amax ? a : amax;
        }
    }
    for (int o = 32; o >= 1; o >>= 1) {
        const uint32_t a = __shfl_xor(amax, o);
        amax = a > amax ? a : amax;
    }
    if ((t & 63) == 0) top[t >> 6] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) amax = top[w] > amax ? top[w] : amax;
    const float scale = row_scale(amax);
    if (t == 0) p.scales[row] = scale;
    const float by = scale == 0.0f ? 1.0f : scale;
    for (int64_t c = 8 * t; c < p.kpad; c += 2048) {
        float x[8];
        const int64_t left = p.cols - c;
        load8<DT>(p.src, base + c, left < 8 ? (int)left : 8, left >= 8 && p.wide, x);
        v2u w = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i >> 2] |= code_of(x[i], by) << (8 * (i & 3));
        *reinterpret_cast<v2u *>(p.codes + row * p.kpad + c) = w;
    }
}

// ---- few tokens: the product is one pass over b.  A wave has 16 channels and MT x 16 tokens and a quarter of the contraction;
// the four waves' int32 sums meet in LDS.  Lane c + 16 g of a fragment has 32 consecutive bytes of its row, 32 g .. of a stretch
// of 128, for two matrix instructions: which of the contraction's elements meet in one instruction does not matter as long as
// both operands agree, and a row is read in whole cache lines.
struct FewParams {
    RowsArgs r;
    int32_t stretches, tiles_n;
};

template <int MT, int DT>
__global__ __launch_bounds__(256) void gemm_rows_few_kernel(const FewParams p) {
    __shared__ v4i sums[4][MT][64];
    const RowsArgs &r = p.r;
    const int t = threadIdx.x, lane = t & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t n0 = (int64_t)(blockIdx.x % p.tiles_n) * 16, m0 = (int64_t)(blockIdx.x / p.tiles_n) * 16 * MT;
    const int64_t nr = n0 + c < r.N ? n0 + c : r.N - 1;
    const int8_t *b = r.b + nr * r.kpad + 32 * g;
    const int8_t *a[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t mr = m0 + 16 * i + c < r.M ? m0 + 16 * i + c : r.M - 1;
        a[i] = r.a + mr * r.kpad + 32 * g;
    }
    v4i acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = v4i{0, 0, 0, 0};
    for (int s = wave; s < p.stretches; s += 4) {
        const v4i b0 = *reinterpret_cast<const v4i *>(b + (int64_t)s * 128), b1 = *reinterpret_cast<const v4i *>(b + (int64_t)s * 128 + 16);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const v4i a0 = *reinterpret_cast<const v4i *>(a[i] + (int64_t)s * 128), a1 = *reinterpret_cast<const v4i *>(a[i] + (int64_t)s * 128 + 16);
            acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b0, a0, acc[i], 0, 0, 0);
            acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b1, a1, acc[i], 0, 0, 0);
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) sums[wave][i][lane] = acc[i];
    __syncthreads();
    // lane: token c, channels 4 g + v; wave w finishes the token tiles w, w + 4, ...
    for (int i = wave; i < MT; i += 4) {
        const v4i all = sums[0][i][lane] + sums[1][i][lane] + sums[2][i][lane] + sums[3][i][lane];
        const int64_t m = m0 + 16 * i + c;
        if (m >= r.M) continue;
        const float sa = r.sa[m];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int64_t n = n0 + 4 * g + v;
            if (n >= r.N) continue;
            store_float<DT>(r.y, m * r.ldy + n, scaled_sum(all[v], sa, r.sb[n], r.bias ? r.bias[n] : 0.0f, r.bias != nullptr));
        }
    }
}

template <int DT>
int launch_few(const RowsArgs &r, hipStream_t s) {
    FewParams p = {r, (int32_t)(r.kpad / 128), (int32_t)ceil_div(r.N, 16)};
    const int mt = r.M <= 16 ? 1 : r.M <= 32 ? 2 : 4;
    const int64_t wgs = p.tiles_n * ceil_div(r.M, 16 * mt);
    if (wgs > 0x7fffffff) return HBFP_ERR_ARG;
    void (*const kernel)(FewParams) = mt == 1 ? &gemm_rows_few_kernel<1, DT> : mt == 2 ? &gemm_rows_few_kernel<2, DT> : &gemm_rows_few_kernel<4, DT>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(256), 0, s, p);
    return launch_status();
}

}  // namespace

int launch_quant_rows(const void *src, int dtype, int64_t rows, int64_t cols, int64_t ld, int8_t *codes, float *scales, hipStream_t s) {
    const int size = dtype == HBFP_F32 ? 4 : 2;
    if (rows > 0x7fffffff) return HBFP_ERR_ARG;
    QuantParams p = {src, codes, scales, cols, ld, round_up(cols, 128), (((uintptr_t)src | (uint64_t)ld * size) & 15) == 0};
    void (*const kernel)(QuantParams) = dtype == HBFP_F32    ? &quant_rows_kernel<HBFP_F32>
                                        : dtype == HBFP_BF16 ? &quant_rows_kernel<HBFP_BF16>
                                                             : &quant_rows_kernel<HBFP_F16>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(256), 0, s, p);
    return launch_status();
}

// Few tokens are a pass over b, the others tiles on the matrix core.
static bool few_rows(int64_t M) { return M <= 64; }

size_t gemm_rows_workspace(int64_t M, int64_t N, int64_t kpad) {
    if (few_rows(M)) return 0;
    const WidePlan plan = wide_plan(M, N, kpad / 64, true);
    return plan.splits > 1 ? (size_t)plan.splits * (size_t)M * (size_t)N * 4 : 0;
}

int launch_gemm_rows(const RowsArgs &a, void *workspace, hipStream_t s) {
    if (few_rows(a.M)) return a.dtype == HBFP_F32 ? launch_few<HBFP_F32>(a, s) : a.dtype == HBFP_BF16 ? launch_few<HBFP_BF16>(a, s) : launch_few<HBFP_F16>(a, s);
    if (ceil_div(a.M, 128) * ceil_div(a.N, 128) > 0x7ffffff0) return HBFP_ERR_ARG;
    const WidePlan plan = wide_plan(a.M, a.N, a.kpad / 64, true);
    WideParams p = {};
    p.A = (const uint8_t *)a.a;
    p.B = (const uint8_t *)a.b;
    p.C = (float *)a.y;
    p.partial = (int32_t *)workspace;
    p.M = a.M;
    p.N = a.N;
    p.kpad = a.kpad;
    p.ldc = a.ldy;
    p.sa = a.sa;
    p.sb = a.sb;
    p.bias = a.bias;
    GemmArgs g = {};
    g.M = a.M;
    g.N = a.N;
    g.C = (float *)a.y;
    g.ldc = a.ldy;
    const bool stream = a.kpad > 1024 || stores_stream(&g);
    return a.dtype == HBFP_F32    ? launch_wide_planned<kWideF32>(p, plan, stream, s)
           : a.dtype == HBFP_BF16 ? launch_wide_planned<kWideBf16>(p, plan, stream, s)
                                  : launch_wide_planned<kWideF16>(p, plan, stream, s);
}

}  // namespace hbfp
