// Root-mean-square norm of rows with the residual's addition before it and the conversion of its rows after it, and its gradient.
// Bound by memory: every tensor is read or written once.  8192 x 4096 bf16 with residual, sum and values: 8-bit rows 64 us (4.7 TB/s), microscaled
// 59 (4.8); the gradient 44 us and 5 for its partial sums.  Walking a row twice instead of keeping it would read a third more.
#include "mx4.h"

namespace hbfp {
namespace {

// ---- sums and maxima over the W waves that share a row; `meet` is this row's room in LDS, used once for each of them
template <class V, class F>
__device__ __forceinline__ V over_wave(V x, const F &join) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) x = join(x, __shfl_xor(x, o));
    return x;
}
template <int W, class V, class F>
__device__ __forceinline__ V over_row(V x, V *meet, int wave, int lane, const F &join) {
    x = over_wave(x, join);
    if constexpr (W > 1) {
        if (lane == 0) meet[wave] = x;
        __syncthreads();
        x = meet[0];
#pragma unroll
        for (int w = 1; w < W; ++w) x = join(x, meet[w]);
    }
    return x;
}
struct Add {
    template <class V> __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};
struct Larger {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};

template <int DT>
__device__ __forceinline__ float rounded(float x) {
    if (DT == HBFP_BF16) return (float)(__bf16)x;
    if (DT == HBFP_F16) return (float)(_Float16)x;
    return x;
}

enum { kNormI8 = 0, kNormMx4 = 1 };

// the sum of x and the residual for eight columns of a row, as it is stored
template <int DT>
__device__ __forceinline__ void sum8(const hbfp_norm &n, int64_t row, int64_t c, int left, float *s) {
    load8<DT>(n.x, row * n.ldx + c, left, s);
    if (n.residual) {
        float r[8];
        load8<DT>(n.residual, row * n.ld_residual + c, left, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = rounded<DT>(s[i] + r[i]);
    }
}
template <int DT>
__device__ __forceinline__ void store8(void *p, int64_t i, int n, const float *x) {
    store4<DT>(p, i, n < 4 ? n : 4, x);
    store4<DT>(p, i + 4, n < 8 ? n - 4 : 4, x + 4);
}
// s -> n, in place
__device__ __forceinline__ void normalise8(float *s, double rstd, const float *weight, int64_t c, int left) {
    float w[8];
    if (weight) load8<HBFP_F32>(weight, c, left, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double u = (double)s[i] * rstd;
        s[i] = (float)(weight ? u * (double)w[i] : u);
    }
    if (left < 8) {                                          // past the row 0, whatever rstd is
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= left) s[i] = 0.0f;
    }
}
__device__ __forceinline__ double sum_of_squares8(const float *s) {
    double q = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) q = __builtin_fma((double)s[i], (double)s[i], q);
    return q;
}
// eight values of n, their codes and the values those stand for
template <int DT>
__device__ __forceinline__ void put_i8(const NormArgs &a, int64_t row, int64_t c, int left, const float *n, float scale) {
    const float by = scale == 0.0f ? 1.0f : scale;
    v2u w = {0, 0};
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = fminf(fmaxf(__builtin_rintf(n[i] / by), -127.0f), 127.0f);
        w[i >> 2] |= ((uint32_t)(int)q & 0xffu) << (8 * (i & 3));
        v[i] = q * scale;
    }
    *reinterpret_cast<v2u *>(a.codes + row * a.kpad + c) = w;
    if (a.n.values) store8<DT>(a.n.values, row * a.n.ld_values + c, left, v);
}
template <int DT>
__device__ __forceinline__ void put_mx4(const NormArgs &a, int64_t row, int64_t c, int left, const float *n, int lane) {
    const uint32_t byte = mx4_byte<HBFP_RNE>(largest_of_quad(mx4_largest8(n)));
    const uint32_t w = mx4_codes<8>(n, byte);
    const int64_t group = c >> 8;
    if (group >= a.mx4.groups) return;
    *reinterpret_cast<uint32_t *>(a.mx4.codes + (group * a.mx4.rows + row) * 128 + ((c & 255) >> 1)) = w;
    if (lane % 4 == 0) a.mx4.scales[(group * a.mx4.scale_rows + row) * 8 + ((c & 255) >> 5)] = (uint8_t)byte;
    if (!a.n.values) return;
    float v[8];
    mx4_values8(w, byte, v);
    store8<DT>(a.n.values, row * a.n.ld_values + c, left, v);
}

// A row belongs to W waves; a workgroup has 4 / W rows, or one.  Up to KEEP x 8 columns a lane stay in registers from the read to the codes;
// longer rows walk the rest again (LOOP).
template <int DT, int FORM, int W, int KEEP, bool LOOP>
__global__ __launch_bounds__(W < 4 ? 256 : 64 * W) void norm_kernel(const NormArgs a) {
    constexpr int kRows = W < 4 ? 4 / W : 1;
    static_assert(W == 1 || kRows == 1, "rows of a workgroup meet no one");
    __shared__ double meet_sum[W];
    __shared__ uint32_t meet_top[W];
    const hbfp_norm &n = a.n;
    const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : threadIdx.x >> 6;
    const int64_t row = (int64_t)workgroup() * kRows + (W == 1 ? threadIdx.x >> 6 : 0);
    if (row >= n.rows) return;                               // (a whole wave, and W = 1 has no barrier)
    constexpr int64_t kStep = 512 * W;
    const int64_t c0 = 8 * (64 * wave + lane);
    const auto left_at = [&](int64_t c) { return n.cols - c < 8 ? (int)(n.cols - c < 0 ? 0 : n.cols - c) : 8; };
    float kept[KEEP][8];
    double sq = 0.0;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int64_t c = c0 + kStep * i;
        sum8<DT>(n, row, c, left_at(c), kept[i]);
    }
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int64_t c = c0 + kStep * i;
        if (n.sum) store8<DT>(n.sum, row * n.ld_sum + c, left_at(c), kept[i]);
        sq += sum_of_squares8(kept[i]);
    }
    if constexpr (LOOP)
        for (int64_t c = c0 + kStep * KEEP; c < n.cols; c += kStep) {
            float s[8];
            sum8<DT>(n, row, c, left_at(c), s);
            if (n.sum) store8<DT>(n.sum, row * n.ld_sum + c, left_at(c), s);
            sq += sum_of_squares8(s);
        }
    sq = over_row<W>(sq, meet_sum, wave, lane, Add());
    const double rstd = 1.0 / __builtin_sqrt(sq / (double)n.cols + (double)n.eps);
    if (n.rstd && wave == 0 && lane == 0) n.rstd[row] = (float)rstd;
    // a row walked again reads what was stored: x or the residual may be gone
    const auto again = [&](int64_t c, float *s) {
        if (n.sum) load8<DT>(n.sum, row * n.ld_sum + c, left_at(c), s);
        else sum8<DT>(n, row, c, left_at(c), s);
        normalise8(s, rstd, n.weight, c, left_at(c));
    };
#pragma unroll
    for (int i = 0; i < KEEP; ++i) normalise8(kept[i], rstd, n.weight, c0 + kStep * i, left_at(c0 + kStep * i));
    if constexpr (FORM == kNormI8) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < KEEP; ++i) top = Larger()(top, mx4_largest8(kept[i]));
        if constexpr (LOOP)
            for (int64_t c = c0 + kStep * KEEP; c < n.cols; c += kStep) {
                float s[8];
                again(c, s);
                top = Larger()(top, mx4_largest8(s));
            }
        top = over_row<W>(top, meet_top, wave, lane, Larger());
        const float scale = __uint_as_float(top) * (1.0f / 127.0f);
        if (wave == 0 && lane == 0) a.scales[row] = scale;
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            if (c0 + kStep * i < a.kpad) put_i8<DT>(a, row, c0 + kStep * i, left_at(c0 + kStep * i), kept[i], scale);
        if constexpr (LOOP)
            for (int64_t c = c0 + kStep * KEEP; c < a.kpad; c += kStep) {
                float s[8];
                again(c, s);
                put_i8<DT>(a, row, c, left_at(c), s, scale);
            }
    } else {
#pragma unroll
        for (int i = 0; i < KEEP; ++i) put_mx4<DT>(a, row, c0 + kStep * i, left_at(c0 + kStep * i), kept[i], lane);
        if constexpr (LOOP)
            for (int64_t c = c0 + kStep * KEEP; c < 256 * a.mx4.groups; c += kStep) {
                float s[8];
                again(c, s);
                put_mx4<DT>(a, row, c, left_at(c), s, lane);
            }
    }
}

template <int DT, int FORM, int W, int KEEP, bool LOOP>
int launch(const NormArgs &a, hipStream_t s) {
    constexpr int kRows = W < 4 ? 4 / W : 1;
    const int64_t wgs = ceil_div(a.n.rows, kRows);
    hipLaunchKernelGGL((norm_kernel<DT, FORM, W, KEEP, LOOP>), grid_of(wgs), dim3(W < 4 ? 256 : 64 * W), 0, s, a);
    return launch_status();
}
// us (bf16, 8-bit rows) on as many waves, with as many times 8 columns a lane: 8192 x 2048 on 4 28.2, on 1 (x 4) 29.9, on 8 40.4; 4096 x 4096 on 4 (x 2) 27.7,
// on 8 29.1, on 16 47.3; 2048 x 8192 on 8 (x 2) 28.8, on 4 (x 4) 29.8, on 16 32.3; 16384 x 1024 on 1 (x 2) 27.4, on 4 42.4; 32768 x 512 on 1 28.1, on 4 71
template <int DT, int FORM>
int launch_form(const NormArgs &a, hipStream_t s) {
    const int64_t cols = a.n.cols;
    if (cols <= 512) return launch<DT, FORM, 1, 1, false>(a, s);
    if (cols <= 1024) return launch<DT, FORM, 1, 2, false>(a, s);
    if (cols <= 2048) return launch<DT, FORM, 4, 1, false>(a, s);
    if (cols <= 4096) return launch<DT, FORM, 4, 2, false>(a, s);
    if (cols <= 8192) return launch<DT, FORM, 8, 2, false>(a, s);
    if (cols <= 16384) return launch<DT, FORM, 16, 2, false>(a, s);
    return launch<DT, FORM, 16, 2, true>(a, s);
}
template <int DT>
int launch_type(const NormArgs &a, hipStream_t s) {
    return a.codes ? launch_form<DT, kNormI8>(a, s) : launch_form<DT, kNormMx4>(a, s);
}

// ---- the gradient.  With u = sum * rstd:  dx = g_sum + rstd (g w - u mean(g w u)),  dweight = sum over rows of g u.
// A workgroup takes rows wg, wg + G, ... and its threads keep their columns: weight and the sums of dweight stay in registers, and
// each row is read once, the next one's while this one is worked on (AHEAD).  The partial sums of the G workgroups are added in their
// order by a second kernel.
struct GradParams {
    NormGradArgs a;
    int32_t wgs;
};

// eight consecutive elements as they lie in memory; of which n (may be <= 0) exist, the others 0
template <int DT>
struct Raw8 {
    static constexpr int kWords = DT == HBFP_F32 ? 8 : 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const void *p, int64_t i, int n) {
        typedef uint32_t words_at __attribute__((ext_vector_type(4), aligned(2)));
        if (n >= 8) {
#pragma unroll
            for (int k = 0; k < kWords / 4; ++k) {
                const words_at x = *reinterpret_cast<const words_at *>(reinterpret_cast<const uint8_t *>(p) + i * (kWords / 2) + 16 * k);
#pragma unroll
                for (int j = 0; j < 4; ++j) w[4 * k + j] = x[j];
            }
            return;
        }
#pragma unroll
        for (int k = 0; k < kWords; ++k) w[k] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) {
                if constexpr (DT == HBFP_F32) w[j] = reinterpret_cast<const uint32_t *>(p)[i + j];
                else w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[i + j] << (16 * (j & 1));
            }
    }
    __device__ __forceinline__ float get(int j) const {
        if constexpr (DT == HBFP_F32) return __uint_as_float(w[j]);
        const uint32_t h = j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xffffu;
        return DT == HBFP_BF16 ? __uint_as_float(h << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)h);
    }
};

template <int DT, int W, int KEEP, bool AHEAD>
__global__ __launch_bounds__(64 * W) void norm_grad_kernel(const GradParams p) {
    __shared__ float meet[2][W];
    const NormGradArgs &a = p.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int64_t kStep = 512 * W;
    const int64_t c0 = 8 * threadIdx.x;
    int left[KEEP];
    float weight[KEEP][8], dw[KEEP][8];
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int64_t l = a.cols - c0 - kStep * i;
        left[i] = l < 0 ? 0 : l < 8 ? (int)l : 8;
        if (a.weight) load8<HBFP_F32>(a.weight, c0 + kStep * i, left[i], weight[i]);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (!a.weight) weight[i][k] = 1.0f;
            dw[i][k] = 0.0f;
        }
    }
    Raw8<DT> g[KEEP], s[KEEP], o[KEEP];
    float r = 0.0f;
    const auto request = [&](int64_t row) {
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
            g[i].load(a.g, row * a.ldg + c0 + kStep * i, left[i]);
            s[i].load(a.sum, row * a.ld_sum + c0 + kStep * i, left[i]);
            if (a.g_sum) o[i].load(a.g_sum, row * a.ld_g_sum + c0 + kStep * i, left[i]);
        }
        r = a.rstd[row];
    };
    const float inv = 1.0f / (float)a.cols;
    int turn = 0;
    if (AHEAD) request(blockIdx.x);
    for (int64_t row = blockIdx.x; row < a.rows; row += p.wgs, turn ^= 1) {
        if (!AHEAD) request(row);
        float u[KEEP][8], v[KEEP][8];
        float dot = 0.0f;
        const float rr = r;
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float gk = g[i].get(k);
                u[i][k] = s[i].get(k) * rr;
                v[i][k] = gk * weight[i][k];
                dw[i][k] = __builtin_fmaf(gk, u[i][k], dw[i][k]);
                dot = __builtin_fmaf(v[i][k], u[i][k], dot);
            }
        Raw8<DT> other[KEEP];
#pragma unroll
        for (int i = 0; i < KEEP; ++i) other[i] = o[i];
        if (AHEAD && row + p.wgs < a.rows) request(row + p.wgs);
        dot = over_row<W>(dot, meet[turn], wave, lane, Add());      // (two rooms: the next row's may be written while this one is read)
        const float mean = dot * inv;
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
            float d[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float e = __builtin_fmaf(-u[i][k], mean, v[i][k]);
                d[k] = a.g_sum ? __builtin_fmaf(rr, e, other[i].get(k)) : rr * e;
            }
            store8<DT>(a.dx, row * a.ldx + c0 + kStep * i, left[i], d);
        }
    }
    if (!a.dweight) return;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) store8<HBFP_F32>(a.partial, (int64_t)blockIdx.x * a.cols + c0 + kStep * i, left[i], dw[i]);
}

// rows longer than what a workgroup keeps: dx in two walks of a row, dweight by columns
template <int DT>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(const NormGradArgs a) {
    __shared__ float meet[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = workgroup();
    if (row >= a.rows) return;
    const float r = a.rstd[row];
    const auto load = [&](int64_t c, int left, float *g, float *u, float *w) {
        load8<DT>(a.g, row * a.ldg + c, left, g);
        load8<DT>(a.sum, row * a.ld_sum + c, left, u);
        if (a.weight) load8<HBFP_F32>(a.weight, c, left, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            u[k] *= r;
            if (!a.weight) w[k] = 1.0f;
        }
    };
    float dot = 0.0f;
    for (int64_t c = 8 * threadIdx.x; c < a.cols; c += 8192) {
        const int left = a.cols - c < 8 ? (int)(a.cols - c) : 8;
        float g[8], u[8], w[8];
        load(c, left, g, u, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) dot = __builtin_fmaf(g[k] * u[k], w[k], dot);
    }
    dot = over_row<16>(dot, meet, wave, lane, Add());
    const float mean = dot / (float)a.cols;
    for (int64_t c = 8 * threadIdx.x; c < a.cols; c += 8192) {
        const int left = a.cols - c < 8 ? (int)(a.cols - c) : 8;
        float g[8], u[8], w[8], o[8];
        load(c, left, g, u, w);
        if (a.g_sum) load8<DT>(a.g_sum, row * a.ld_g_sum + c, left, o);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float v = __builtin_fmaf(-u[k], mean, g[k] * w[k]);
            g[k] = a.g_sum ? __builtin_fmaf(r, v, o[k]) : r * v;
        }
        store8<DT>(a.dx, row * a.ldx + c, left, g);
    }
}
// blockIdx.x: 2048 columns; blockIdx.y: rows y, y + G, ...
template <int DT>
__global__ __launch_bounds__(256) void norm_dweight_kernel(const GradParams p) {
    const NormGradArgs &a = p.a;
    const int64_t c = (int64_t)blockIdx.x * 2048 + 8 * threadIdx.x;
    if (c >= a.cols) return;
    const int left = a.cols - c < 8 ? (int)(a.cols - c) : 8;
    float dw[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int64_t row = blockIdx.y; row < a.rows; row += p.wgs) {
        float g[8], s[8];
        load8<DT>(a.g, row * a.ldg + c, left, g);
        load8<DT>(a.sum, row * a.ld_sum + c, left, s);
        const float r = a.rstd[row];
#pragma unroll
        for (int k = 0; k < 8; ++k) dw[k] += g[k] * (s[k] * r);
    }
    store8<HBFP_F32>(a.partial, (int64_t)blockIdx.y * a.cols + c, left, dw);
}

// dweight from the partial sums: a workgroup has 32 columns, its 32 half waves a share of the G sums each; both steps add in order
constexpr int kShares = 32;
__global__ __launch_bounds__(32 * kShares) void norm_dweight_sum_kernel(const GradParams p) {
    __shared__ float meet[kShares][32];
    const NormGradArgs &a = p.a;
    const int lane = threadIdx.x & 31, share = threadIdx.x >> 5;
    const int64_t c = (int64_t)workgroup() * 32 + lane;
    const int per = (p.wgs + kShares - 1) / kShares, end = (share + 1) * per < p.wgs ? (share + 1) * per : p.wgs;
    float sum = 0.0f;
    if (c < a.cols)
        for (int i = share * per; i < end; i += 8) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = i + k < end ? a.partial[(int64_t)(i + k) * a.cols + c] : 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += v[k];
        }
    meet[share][lane] = sum;
    __syncthreads();
    if (share > 0 || c >= a.cols) return;
    for (int i = 1; i < kShares; ++i) sum += meet[i][lane];
    a.dweight[c] = sum;
}

constexpr int64_t kGradKept = 16384;
// Workgroups that share the rows: waves enough to keep the memory busy, few enough for the partial sums not to matter.  us with 2048 and with
// 4096 waves in all (bf16): 777 x 4096 11.7, 13.7, 777 x 2048 9.9, 11.4, 32768 x 512 29.8, 36.1, 4096 x 4096 26.7, 26.9; but 2048 x 8192 29.3,
// 27.1, 65536 x 256 49, 41
int64_t grad_wgs(int64_t rows, int64_t cols) {
    const int64_t waves = cols <= 512 ? 1 : cols <= 1024 ? 2 : cols <= 2048 ? 4 : cols <= 4096 ? 8 : 16;
    const int64_t most = cols > kGradKept ? 64 : (cols <= 256 || cols > 4096 ? 4096 : 2048) / waves;
    return rows < most ? rows : most;
}

template <int DT, int W, int KEEP, bool AHEAD>
void launch_grad_rows(const GradParams &p, hipStream_t s) {
    hipLaunchKernelGGL((norm_grad_kernel<DT, W, KEEP, AHEAD>), dim3((unsigned)p.wgs), dim3(64 * W), 0, s, p);
}
// Eight columns a thread and the next row ahead as far as a workgroup of 16 waves goes.  us (bf16) of 4096 x 4096 on 8 waves 26.9, on 4 with 16
// columns a thread 32.0, without the next row ahead 27.1 and 32.9; 2048 x 8192 on 16 waves 27.1, on 8 31.3; 1024 x 16384, 16 columns a thread,
// without the next row ahead 32.4, with it 48.9 (registers in scratch; without it FP32 keeps two there, the 16-bit types none)
template <int DT>
int launch_grad(const NormGradArgs &a, hipStream_t s) {
    const GradParams p = {a, (int32_t)grad_wgs(a.rows, a.cols)};
    if (a.cols <= 512) launch_grad_rows<DT, 1, 1, true>(p, s);
    else if (a.cols <= 1024) launch_grad_rows<DT, 2, 1, true>(p, s);
    else if (a.cols <= 2048) launch_grad_rows<DT, 4, 1, true>(p, s);
    else if (a.cols <= 4096) launch_grad_rows<DT, 8, 1, true>(p, s);
    else if (a.cols <= 8192) launch_grad_rows<DT, 16, 1, true>(p, s);
    else if (a.cols <= kGradKept) launch_grad_rows<DT, 16, 2, false>(p, s);
    else {
        // (dx may be written over g)
        if (a.dweight) hipLaunchKernelGGL(norm_dweight_kernel<DT>, dim3((unsigned)ceil_div(a.cols, 2048), (unsigned)p.wgs), dim3(256), 0, s, p);
        hipLaunchKernelGGL(norm_grad_long_kernel<DT>, grid_of(a.rows), dim3(1024), 0, s, a);
    }
    if (a.dweight) hipLaunchKernelGGL(norm_dweight_sum_kernel, grid_of(ceil_div(a.cols, 32)), dim3(32 * kShares), 0, s, p);
    return launch_status();
}

}  // namespace

int launch_norm(const NormArgs &a, hipStream_t s) {
    return a.n.dtype == HBFP_F32 ? launch_type<HBFP_F32>(a, s) : a.n.dtype == HBFP_BF16 ? launch_type<HBFP_BF16>(a, s) : launch_type<HBFP_F16>(a, s);
}

size_t norm_grad_workspace(int64_t rows, int64_t cols) { return (size_t)grad_wgs(rows, cols) * (size_t)cols * 4; }

int launch_norm_grad(const NormGradArgs &a, hipStream_t s) {
    return a.dtype == HBFP_F32 ? launch_grad<HBFP_F32>(a, s) : a.dtype == HBFP_BF16 ? launch_grad<HBFP_BF16>(a, s) : launch_grad<HBFP_F16>(a, s);
}

}  // namespace hbfp
