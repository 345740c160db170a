// Products in 8-bit integers with an FP32 scale per row of each operand:
//     y[m][n] = (sum_k a[m][k] b[n][k]) * sa[m] * sb[n] + bias[n]
// The sum is an exact int32 whatever its order; scales and bias are FP32 and y is rounded once.
#include "gemm_wide.h"
#include "kv_cache.h"

namespace hbfp {
namespace {

// ---- rows -> codes.  A workgroup has one row: its largest magnitude, then its codes.  Bound by memory: 4096 x 4096 bf16 in 16.4 us, 3.1 TB/s.
struct QuantParams {
    const void *src;
    int8_t *codes;
    float *scales;
    int64_t cols, ld, kpad;
};

__device__ __forceinline__ float row_scale(uint32_t amax) { return __uint_as_float(amax) * (1.0f / 127.0f); }
__device__ __forceinline__ uint32_t code_of(float x, float scale) {
    const float q = __builtin_rintf(x / scale);
    return (uint32_t)(int)fminf(fmaxf(q, -127.0f), 127.0f) & 0xffu;
}

__device__ __forceinline__ uint32_t largest8(uint32_t amax, const float *x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = __float_as_uint(x[i]) & 0x7fffffffu;
        amax = a > amax ? a : amax;
    }
    return amax;
}
__device__ __forceinline__ uint32_t largest_of_wave(uint32_t amax) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        const uint32_t a = __shfl_xor(amax, o);
        amax = a > amax ? a : amax;
    }
    return amax;
}
__device__ __forceinline__ v2u codes8(const float *x, float scale) {
    const float by = scale == 0.0f ? 1.0f : scale;
    v2u w = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i >> 2] |= code_of(x[i], by) << (8 * (i & 3));
    return w;
}

template <int DT>
__global__ __launch_bounds__(256) void quant_rows_kernel(const QuantParams p) {
    __shared__ uint32_t top[4];
    const int64_t row = blockIdx.x, base = row * p.ld;
    const int t = threadIdx.x;
    // up to KEEP x 2048 columns stay in registers between the two walks
    constexpr int KEEP = 4;
    float kept[KEEP][8];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int64_t c = 8 * t + 2048 * i, left = p.cols - c;
        load8<DT>(p.src, base + c, left < 8 ? (int)(left < 0 ? 0 : left) : 8, kept[i]);
        amax = largest8(amax, kept[i]);
    }
    for (int64_t c = 8 * t + 2048 * KEEP; c < p.cols; c += 2048) {
        float x[8];
        const int64_t left = p.cols - c;
        load8<DT>(p.src, base + c, left < 8 ? (int)left : 8, x);
        amax = largest8(amax, x);
    }
    amax = largest_of_wave(amax);
    if ((t & 63) == 0) top[t >> 6] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) amax = top[w] > amax ? top[w] : amax;
    const float scale = row_scale(amax);
    if (t == 0) p.scales[row] = scale;
    int8_t *const codes = p.codes + row * p.kpad;
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
        if (8 * t + 2048 * i < p.kpad) *reinterpret_cast<v2u *>(codes + 8 * t + 2048 * i) = codes8(kept[i], scale);
    for (int64_t c = 8 * t + 2048 * KEEP; c < p.kpad; c += 2048) {
        float x[8];
        const int64_t left = p.cols - c;
        load8<DT>(p.src, base + c, left < 8 ? (int)left : 8, x);
        *reinterpret_cast<v2u *>(codes + c) = codes8(x, scale);
    }
}

// ---- few tokens: the product is one pass over b.  A wave has 16 channels and MT x 16 tokens and a share of the contraction; the
// waves' int32 sums meet in LDS.  Lane c + 16 g of a fragment has 32 consecutive bytes of its row, 32 g .. of a stretch of 128,
// for two matrix instructions: which of the contraction's elements meet in one instruction does not matter as long as both
// operands agree, and a row is read in whole cache lines.  U stretches are on their way at once.
// FUSED (one or two tokens): x is converted by every workgroup for itself, into LDS, while the first of b are on their way.
struct FewParams {
    RowsArgs r;
    const void *x;
    int64_t ldx;
    int32_t stretches, tiles_n;
};
constexpr int kFusedRows = 2, kFusedBytes = 32768;

template <int MT, int U, int W, int DT, bool FUSED>
__global__ __launch_bounds__(64 * W) void gemm_rows_few_kernel(const FewParams p) {
    __shared__ v4i sums[W][MT][64];
    __shared__ __attribute__((aligned(16))) uint8_t own[FUSED ? kFusedBytes : 16];
    __shared__ uint32_t top[kFusedRows][W];
    const RowsArgs &r = p.r;
    const int t = threadIdx.x, lane = t & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t n0 = (int64_t)(blockIdx.x % p.tiles_n) * 16, m0 = (int64_t)(blockIdx.x / p.tiles_n) * 16 * MT;
    const int64_t nr = n0 + c < r.N ? n0 + c : r.N - 1;
    const int8_t *b = r.b + nr * r.kpad + 32 * g;
    const int8_t *a[MT];
    if constexpr (!FUSED) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int64_t mr = m0 + 16 * i + c < r.M ? m0 + 16 * i + c : r.M - 1;
            a[i] = r.a + mr * r.kpad + 32 * g;
        }
    }
    v4i bw[U][2], aw[U][MT][2];
    const auto request = [&](int s0) {                      // stretches s0, s0 + W, ...; past the end the last one again
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = (int64_t)(s0 + u * W < p.stretches ? s0 + u * W : p.stretches - 1) * 128;
            bw[u][0] = *reinterpret_cast<const v4i *>(b + at);
            bw[u][1] = *reinterpret_cast<const v4i *>(b + at + 16);
            if constexpr (!FUSED) {
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    aw[u][i][0] = *reinterpret_cast<const v4i *>(a[i] + at);
                    aw[u][i][1] = *reinterpret_cast<const v4i *>(a[i] + at + 16);
                }
            }
        }
    };
    request(wave);
    float scale[kFusedRows];
    if constexpr (FUSED) {
        for (int m = 0; m < r.M; ++m) {
            uint32_t amax = 0;
            for (int64_t k = 8 * t; k < r.K; k += 512 * W) {
                float x[8];
                const int64_t left = r.K - k;
                load8<DT>(p.x, m * p.ldx + k, left < 8 ? (int)left : 8, x);
                amax = largest8(amax, x);
            }
            amax = largest_of_wave(amax);
            if (lane == 0) top[m][wave] = amax;
        }
        __syncthreads();
#pragma unroll
        for (int m = 0; m < kFusedRows; ++m) {
            if (m >= r.M) break;
            uint32_t amax = top[m][0];
#pragma unroll
            for (int w = 1; w < W; ++w) amax = top[m][w] > amax ? top[m][w] : amax;
            scale[m] = row_scale(amax);
            for (int64_t k = 8 * t; k < r.kpad; k += 512 * W) {
                float x[8];
                const int64_t left = r.K - k;
                load8<DT>(p.x, m * p.ldx + k, left < 8 ? (int)left : 8, x);
                *reinterpret_cast<v2u *>(own + m * r.kpad + k) = codes8(x, scale[m]);
            }
        }
        __syncthreads();
        a[0] = reinterpret_cast<const int8_t *>(own) + (c < r.M ? c : 0) * r.kpad + 32 * g;
    }
    v4i acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = v4i{0, 0, 0, 0};
    for (int s0 = wave; s0 < p.stretches; s0 += W * U) {
        if (s0 != wave) request(s0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + u * W;
            if (s < p.stretches) {
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    if constexpr (FUSED) {
                        aw[u][i][0] = *reinterpret_cast<const v4i *>(a[i] + (int64_t)s * 128);
                        aw[u][i][1] = *reinterpret_cast<const v4i *>(a[i] + (int64_t)s * 128 + 16);
                    }
                    acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bw[u][0], aw[u][i][0], acc[i], 0, 0, 0);
                    acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bw[u][1], aw[u][i][1], acc[i], 0, 0, 0);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) sums[wave][i][lane] = acc[i];
    __syncthreads();
    // lane: token c, channels 4 g + v; wave w finishes the token tiles w, w + W, ...
    for (int i = wave; i < MT; i += W) {
        v4i all = sums[0][i][lane];
#pragma unroll
        for (int w = 1; w < W; ++w) all += sums[w][i][lane];
        const int64_t m = m0 + 16 * i + c;
        if (m >= r.M) continue;
        const float sa = FUSED ? (c == 0 ? scale[0] : scale[1]) : r.sa[m];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int64_t n = n0 + 4 * g + v;
            if (n >= r.N) continue;
            store_float<DT>(r.y, m * r.ldy + n, scaled_sum(all[v], sa, r.sb[n], r.bias ? r.bias[n] : 0.0f, r.bias != nullptr));
        }
    }
}

template <int MT, int U, int W, int DT, bool FUSED>
int launch_few(FewParams p, hipStream_t s) {
    p.stretches = (int32_t)(p.r.kpad / 128);
    p.tiles_n = (int32_t)ceil_div(p.r.N, 16);
    const int64_t wgs = p.tiles_n * ceil_div(p.r.M, 16 * MT);
    if (wgs > 0x7fffffff) return HBFP_ERR_ARG;
    hipLaunchKernelGGL((gemm_rows_few_kernel<MT, U, W, DT, FUSED>), dim3((unsigned)wgs), dim3(64 * W), 0, s, p);
    return launch_status();
}
// Waves and stretches in flight of a workgroup (W x U = 32, or 16 with two token tiles: the same bytes on their way).  us with
// 4, 8 and 16 waves, bf16, conversion included: 16 tokens 4096 x 4096 10.8, 10.9, 11.3, 512 x 512 8.3, 6.6, 6.0, 28672 x 4096 36.7,
// 39.5, 43.3; one token converted inside 4096 x 4096 7.7, 7.1, 6.4, 8192 x 8192 18.8, 16.2, 16.9
template <int DT>
int launch_few_of(const FewParams &p, hipStream_t s) {
    if (p.r.M > 16) return launch_few<2, 1, 16, DT, false>(p, s);
    return p.r.N <= 8192 ? launch_few<1, 4, 8, DT, false>(p, s) : launch_few<1, 8, 4, DT, false>(p, s);
}
template <int DT>
int launch_fused_of(const FewParams &p, hipStream_t s) {
    return p.r.N <= 5120 ? launch_few<1, 2, 16, DT, true>(p, s) : launch_few<1, 4, 8, DT, true>(p, s);
}

}  // namespace

int launch_quant_rows(const void *src, int dtype, int64_t rows, int64_t cols, int64_t ld, int8_t *codes, float *scales, hipStream_t s) {
    if (rows > 0x7fffffff) return HBFP_ERR_ARG;
    QuantParams p = {src, codes, scales, cols, ld, round_up(cols, 128)};
    void (*const kernel)(QuantParams) = dtype == HBFP_F32    ? &quant_rows_kernel<HBFP_F32>
                                        : dtype == HBFP_BF16 ? &quant_rows_kernel<HBFP_BF16>
                                                             : &quant_rows_kernel<HBFP_F16>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(256), 0, s, p);
    return launch_status();
}

// Few tokens are a pass over b, more of them tiles on the matrix core.  Up to 16 tokens the pass is ahead at every size (16 x 28672 x
// 4096 36.7 us, tiles 36.8; 16 x 8192 x 8192 23.7 and 26.9; 16 x 512 x 512 6.6 and 8.6), with a second tile of tokens only where b is
// small (32 x 4096 x 4096 13.6 and 16.9, 32 x 5003 x 2730 15.2 and 16.8; 32 x 8192 x 8192 34.3 and 27.7, 32 x 1024 x 8192 17.6 and 15.8)
static bool few_rows(int64_t M, int64_t N, int64_t kpad) {
    return M <= 16 || (M <= 32 && kpad <= 4096 && N * kpad <= (int64_t)16 << 20);
}

size_t gemm_rows_workspace(int64_t M, int64_t N, int64_t kpad) {
    if (few_rows(M, N, kpad)) return 0;
    const WidePlan plan = wide_plan(M, N, kpad / 64, true);
    return plan.splits > 1 ? (size_t)plan.splits * (size_t)M * (size_t)N * 4 : 0;
}

int launch_gemm_rows(const RowsArgs &a, void *workspace, hipStream_t s) {
    if (few_rows(a.M, a.N, a.kpad)) {
        const FewParams p = {a, nullptr, 0, 0, 0};
        return a.dtype == HBFP_F32 ? launch_few_of<HBFP_F32>(p, s) : a.dtype == HBFP_BF16 ? launch_few_of<HBFP_BF16>(p, s) : launch_few_of<HBFP_F16>(p, s);
    }
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

// One token: 4096 x 4096 6.4 us against about 10 in two launches.  Two: 7.7 and 9.8, but 28672 x 4096 32 and 27: every workgroup
// converts both again
bool linear_fused_ok(int64_t M, int64_t N, int64_t kpad) { return (M == 1 || (M == 2 && N <= 16384)) && M * kpad <= kFusedBytes; }

int launch_linear_fused(const RowsArgs &a, const void *x, int64_t ldx, hipStream_t s) {
    const FewParams p = {a, x, ldx, 0, 0};
    return a.dtype == HBFP_F32 ? launch_fused_of<HBFP_F32>(p, s) : a.dtype == HBFP_BF16 ? launch_fused_of<HBFP_BF16>(p, s) : launch_fused_of<HBFP_F16>(p, s);
}

}  // namespace hbfp
