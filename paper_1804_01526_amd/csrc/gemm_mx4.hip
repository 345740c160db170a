// Products of microscaled 4-bit operands:
//     y[m][n] = sum over blocks of 32 of 2^(sa + sb - 254) * (sum of the block's products) + bias[n]
// on v_mfma_scale_f32_*_f8f6f4 with both operands in 4 bits: a lane hands the instruction one block, 32 codes in 16 bytes as they
// are stored, and its scale byte, and the instruction multiplies, scales and accumulates in FP32.
#include <math.h>

#include "gemm_wide.h"
#include "mx4.h"

namespace hbfp {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));

// the builtin takes eight registers an operand and drops the last four for this format
__device__ __forceinline__ v8i four_bit(const v4i &x) { return v8i{x[0], x[1], x[2], x[3], 0, 0, 0, 0}; }

// ---- many tokens: tiles of 64 T x 64 T.  The frame is that of the int8 kernel for one exponent per row (gemm_wide.h): four waves of
// 32 T x 32 T, so that a pair of matrix instructions needs one 16-byte LDS read a lane; operands copied global -> LDS asynchronously
// into a ring of stages; fragments read a k-step ahead, between the matrix instructions; a ring buffer handed over in the stage's
// last k-step.  A stage is one group of 256 k: 128 bytes of codes a row, and 8 scale bytes.  Lanes 0..31 of a fragment have the
// group's first four blocks, lanes 32..63 the others, so that a row's four bytes are one word of a lane for the whole stage and a
// k-step picks its byte in the instruction.
// Bound by the chip's power and by what a tile has around its loop: 4096^3 on tiles of 256, one round: ring filled after 2.2 us, loop 26 us at
// 1.64 GHz with the matrix core busy 76 % of it (of the 5.9 PFLOP/s that a register-only loop gets at 1.5 GHz, 5.2), store 6.5 us with all compute
// units at once: 38.4 us, 3.6 PFLOP/s; 8192^3 248 us, 4.4 PFLOP/s.  With the requests and copies behind whole rows of matrix instructions instead of
// single ones 8192^3 took 253, with a unit's tiles in one workgroup and copies running on 258 (copies and stores share a counter).  Tiles of 256 take
// 252 registers and 256 accumulators; with FP32 outputs one register more is in scratch, around the loop.
struct Mx4Params {
    Mx4Product q;
    float *partial;              // split along k: FP32 sums [splits][M][N]
    int32_t groups, splits, groups_per_split;
    int32_t tiles_m, tiles_n;
};
template <int T, int RING>
struct Mx4Tile {
    static constexpr int kRows = 64 * T;
    static constexpr int kOperand = kRows * 128, kCodes = 2 * kOperand;
    static constexpr int kScales = 2 * kRows * 8;          // T pieces of 1 KB
    static constexpr int kStage = kCodes + kScales;
    static constexpr int kLds = RING * kStage;
    static constexpr int kCopies = kCodes / 1024 / 4;      // of codes per wave and stage; and one of scales
    static __device__ __forceinline__ int swizzle(int row) { return (row >> 1) & 7; }
};

template <int T, int RING, int OUT, bool STREAM>
__global__ __launch_bounds__(256, T > 2 ? 1 : T == 2 ? 2 : 4) void gemm_mx4_kernel(const Mx4Params p) {
    typedef Mx4Tile<T, RING> W;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const Mx4Product &q = p.q;
    int tm, tn, split = blockIdx.y;
    if (p.splits >= 8 ? !tile_and_split_of_workgroup(blockIdx.x, p.tiles_m, p.tiles_n, p.splits, tm, tn, split)
                      : !tile_of_workgroup(blockIdx.x, p.tiles_m, p.tiles_n, tm, tn))
        return;                                                                 // whole workgroup, before any barrier
    const int st_begin = split * p.groups_per_split;
    const int nstage = p.groups - st_begin < p.groups_per_split ? p.groups - st_begin : p.groups_per_split;   // at least 1

    const int t = threadIdx.x, lane = t & 63;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wm = wave & 1, wn = wave >> 1;
    const int l32 = lane & 31, lh = lane >> 5;
    const int64_t M = q.a.rows, N = q.b.rows;
    const int64_t row0 = (int64_t)tm * W::kRows, col0 = (int64_t)tn * W::kRows;

    // ---- copies: piece c of a stage's codes is 1 KB, 8 rows; the first half are pieces of A, the others of B; wave w moves pieces w,
    // w + 4, ...  A lane copies 16 bytes: LDS chunk lane % 8 of its row, which holds source chunk (lane % 8) ^ swizzle(row).  Rows past the
    // edge re-read the last row (their results are never stored).
    constexpr int kHalf = W::kCopies / 2;
    const uint8_t *abase = q.a.codes + ((int64_t)st_begin * M + row0) * 128, *bbase = q.b.codes + ((int64_t)st_begin * N + col0) * 128;
    uint32_t cvoff[W::kCopies];
#pragma unroll
    for (int i = 0; i < W::kCopies; ++i) {
        const int r = (wave + 4 * (i < kHalf ? i : i - kHalf)) * 8 + lane / 8;
        const int64_t lim = i < kHalf ? M - row0 : N - col0;
        const int rr = r < lim ? r : (int)lim - 1;
        cvoff[i] = (uint32_t)rr * 128 + (((lane & 7) ^ W::swizzle(r)) * 16);
    }
    // scales: rows of A, then rows of B, 8 bytes each, in T pieces of 1 KB, two rows a lane; waves past T move a piece again
    const uint8_t *sbase;
    int64_t sstep;
    const int spiece = wave % T;
    {
        int r = spiece * 128 + 2 * lane;
        const bool is_a = r < W::kRows;
        r -= is_a ? 0 : W::kRows;
        const Mx4View &v = is_a ? q.a : q.b;
        const int64_t at = (is_a ? row0 : col0) + r, last = v.scale_rows - 2;
        sbase = v.scales + ((int64_t)st_begin * v.scale_rows + (at < last ? at : last)) * 8;
        sstep = v.scale_rows * 8;
    }
#define HBFP_MX4_COPY(i, ring_) \
    async_copy16((i) < kHalf ? abase : bbase, cvoff[i], (uint32_t)((ring_) * W::kStage + (wave + 4 * (i)) * 1024))
#define HBFP_MX4_COPY_LAST(ring_)                                                                            \
    {                                                                                                       \
        async_copy16_at(sbase, (uint32_t)((ring_) * W::kStage + W::kCodes + spiece * 1024));                \
        sbase += sstep;                                                                                     \
        abase += M * 128;                                                                                   \
        bbase += N * 128;                                                                                   \
    }
#define HBFP_MX4_COPY_STAGE(ring_)                                                                           \
    {                                                                                                       \
        _Pragma("unroll") for (int i = 0; i < W::kCopies; ++i) HBFP_MX4_COPY(i, ring_);                    \
        HBFP_MX4_COPY_LAST(ring_);                                                                          \
    }

    // ---- fragment addresses inside a stage: row tile i of A is rows 32 T wm + 32 i + l32, k-step s its chunk 4 lh + s
    int fa[4], fb[4];
    const int ra = 32 * T * wm + l32, rb = 32 * T * wn + l32;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        fa[s] = ra * 128 + (((4 * lh + s) ^ W::swizzle(ra)) * 16);
        fb[s] = W::kOperand + rb * 128 + (((4 * lh + s) ^ W::swizzle(rb)) * 16);
    }
    const int ga = W::kCodes + ra * 8 + 4 * lh, gb = W::kCodes + (W::kRows + rb) * 8 + 4 * lh;

    v16f acc[T][T];
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
        for (int j = 0; j < T; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;

    v4i a[2][T], b[2][T];                               // [buffer][tile]
    int as[2][T], bs[2][T];                             // scale words of this stage and of the next
    // request r of a k-step's fragments, in the order in which its matrix instructions want them: row tile 0, all column tiles, the other row tiles
#define HBFP_MX4_READ(buf, base_, s, r)                                                                        \
    {                                                                                                         \
        if ((r) == 0 || (r) > T) a[buf][(r) ? (r) - T : 0] = *reinterpret_cast<const v4i *>((base_) + fa[s] + ((r) ? (r) - T : 0) * 32 * 128); \
        else b[buf][(r) - 1] = *reinterpret_cast<const v4i *>((base_) + fb[s] + ((r) - 1) * 32 * 128);        \
    }
#define HBFP_MX4_READ_SCALE(buf, base_, r)                                                                     \
    {                                                                                                         \
        if ((r) == 0 || (r) > T) as[buf][(r) ? (r) - T : 0] = *reinterpret_cast<const int *>((base_) + ga + ((r) ? (r) - T : 0) * 32 * 8); \
        else bs[buf][(r) - 1] = *reinterpret_cast<const int *>((base_) + gb + ((r) - 1) * 32 * 8);            \
    }
#define HBFP_MX4_FENCE                  \
    asm volatile("" ::: "memory");      \
    __builtin_amdgcn_sched_barrier(0)
#define HBFP_MX4_MFMA(buf, s, i, j)                                                                            \
    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(four_bit(a[buf][i]), four_bit(b[buf][j]), acc[i][j], 4, 4, s, as[0][i], s, bs[0][j])
    // one k-step of 64: T x T matrix instructions on one buffer, and behind the first of them, one by one, the requests of the next k-step's
    // fragments into the other: what stands behind a matrix instruction issues while it runs
#define HBFP_MX4_KSTEP(s, base_)                                                                               \
    {                                                                                                         \
        constexpr int per_ = (2 * T + T * T - 1) / (T * T);                                                   \
        _Pragma("unroll") for (int e_ = 0; e_ < T * T; ++e_) {                                                \
            HBFP_MX4_MFMA((s) & 1, s, e_ / T, e_ % T);                                                        \
            _Pragma("unroll") for (int r_ = e_ * per_; r_ < (e_ + 1) * per_ && r_ < 2 * T; ++r_)              \
                HBFP_MX4_READ(1 - ((s) & 1), base_, (s) + 1, r_);                                             \
            HBFP_MX4_FENCE;                                                                                   \
        }                                                                                                     \
    }
    // A stage is four k-steps; the fragments of its first, and its scale words, were requested during the stage before.  The hand-over,
    // behind the second matrix instruction of its last: this wave has its last fragments of the stage, and its copies of the next stage have
    // landed when only those of the AFTER stages behind it are in flight; after the barrier that holds for everybody, and the buffer takes the
    // copies of stage st + RING (COPY), spread over the rest of the k-step.  LAST: nothing follows.
#define HBFP_MX4_STAGE(AFTER, COPY, LAST)                                                                      \
    {                                                                                                         \
        const uint8_t *base = lds + ring * W::kStage;                                                         \
        const int next = ring + 1 == RING ? 0 : ring + 1;                                                     \
        const uint8_t *nbase = lds + next * W::kStage;                                                        \
        HBFP_MX4_KSTEP(0, base);                                                                              \
        HBFP_MX4_KSTEP(1, base);                                                                              \
        HBFP_MX4_KSTEP(2, base);                                                                              \
        constexpr int hand_ = T > 1 ? 1 : 0, slots_ = T * T - hand_, per_ = (2 * T + slots_ - 1) / slots_;    \
        _Pragma("unroll") for (int e_ = 0; e_ < T * T; ++e_) {                                                \
            HBFP_MX4_MFMA(1, 3, e_ / T, e_ % T);                                                              \
            if (!(LAST) && e_ >= hand_) {                                                                     \
                if (e_ == hand_) {                                                                            \
                    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((AFTER) * (W::kCopies + 1)) : "memory"); \
                    __builtin_amdgcn_s_barrier();                                                             \
                    asm volatile("" ::: "memory");                                                            \
                }                                                                                             \
                _Pragma("unroll") for (int r_ = (e_ - hand_) * per_; r_ < (e_ - hand_ + 1) * per_ && r_ < 2 * T; ++r_) { \
                    HBFP_MX4_READ(0, nbase, 0, r_);                                                           \
                    HBFP_MX4_READ_SCALE(1, nbase, r_);                                                        \
                }                                                                                             \
                if (COPY) {                                                                                   \
                    _Pragma("unroll") for (int c_ = (e_ - hand_) * W::kCopies / slots_; c_ < (e_ - hand_ + 1) * W::kCopies / slots_; ++c_) \
                        HBFP_MX4_COPY(c_, ring);                                                              \
                    if (e_ == T * T - 1) HBFP_MX4_COPY_LAST(ring);                                            \
                }                                                                                             \
            }                                                                                                 \
            HBFP_MX4_FENCE;                                                                                   \
        }                                                                                                     \
        _Pragma("unroll") for (int i_ = 0; i_ < T; ++i_) {                                                    \
            as[0][i_] = as[1][i_];                                                                            \
            bs[0][i_] = bs[1][i_];                                                                            \
        }                                                                                                     \
        ring = next;                                                                                          \
    }

    // prologue: up to RING stages on their way, the fragments of k-step 0 when the first has landed
    HBFP_MX4_COPY_STAGE(0);
    if (RING > 2 && nstage > 2) {
        HBFP_MX4_COPY_STAGE(1);
        HBFP_MX4_COPY_STAGE(2);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * (W::kCopies + 1)) : "memory");
    } else if (nstage > 1) {
        HBFP_MX4_COPY_STAGE(1);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(W::kCopies + 1) : "memory");
    } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int r = 0; r < 2 * T; ++r) {
        HBFP_MX4_READ(0, lds, 0, r);
        HBFP_MX4_READ_SCALE(0, lds, r);
    }
#pragma unroll
    for (int i = 0; i < T; ++i) as[1][i] = bs[1][i] = 0;
    __builtin_amdgcn_sched_barrier(0);
    if (RING > 3 && nstage > 3) HBFP_MX4_COPY_STAGE(3);
    int ring = 0;
    int st = 0;
    for (; st + RING < nstage; ++st) HBFP_MX4_STAGE(RING - 2, true, false);
    if (RING > 3 && nstage - st == 4) {
        HBFP_MX4_STAGE(2, false, false);
        ++st;
    }
    if (RING > 2 && nstage - st == 3) {
        HBFP_MX4_STAGE(1, false, false);
        ++st;
    }
    if (nstage - st == 2) HBFP_MX4_STAGE(0, false, false);
    HBFP_MX4_STAGE(0, false, true);
#undef HBFP_MX4_STAGE
#undef HBFP_MX4_KSTEP
#undef HBFP_MX4_MFMA
#undef HBFP_MX4_READ_SCALE
#undef HBFP_MX4_READ
#undef HBFP_MX4_FENCE
#undef HBFP_MX4_COPY_STAGE
#undef HBFP_MX4_COPY_LAST
#undef HBFP_MX4_COPY

    const int64_t i0 = row0 + 32 * T * wm, j0 = col0 + 32 * T * wn;
    if (T == 1 && p.splits > 1) {
        store_result<T, T, false>(p.partial + ((int64_t)split * M + i0) * N + j0, N, M - i0, N - j0, false, lane,
                                  [&](int i, int j, int v) { return acc[i][j][v]; });
        return;
    }
    float bias[T];
    const bool has_bias = q.bias != nullptr;
#pragma unroll
    for (int j = 0; j < T; ++j) {
        const int64_t col = j0 + 32 * j + l32;
        bias[j] = has_bias ? q.bias[col < N ? col : N - 1] : 0.0f;
    }
    const auto value = [&](int i, int j, int v) { return has_bias ? acc[i][j][v] + bias[j] : acc[i][j][v]; };
    if constexpr (OUT == kWideF32) store_result<T, T, STREAM>((float *)q.y + i0 * q.ldy + j0, q.ldy, M - i0, N - j0, false, lane, value);
    else
        store_result16<T, T, OUT>((uint16_t *)q.y + i0 * q.ldy + j0, q.ldy, M - i0, N - j0, true, lane, value);
}

// The slices of a product split along k, summed in their order.  A thread sums four outputs 256 apart.  19 x 516 x 55804: 16 slices 11.1 us
// with their sum, unsplit 46.
template <int OUT>
__global__ __launch_bounds__(256) void mx4_sum_kernel(const Mx4Params p) {
    const Mx4Product &q = p.q;
    const int64_t N = q.b.rows, n = q.a.rows * N;
    const int64_t e0 = (int64_t)blockIdx.x * 1024 + threadIdx.x;
    float sum[4] = {0, 0, 0, 0};
    for (int z = 0; z < p.splits; z += 8) {
        float v[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[u][k] = e0 + u * 256 < n && z + k < p.splits ? p.partial[(int64_t)(z + k) * n + e0 + u * 256] : 0.0f;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[u] += v[u][k];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int64_t e = e0 + u * 256;
        if (e >= n) return;
        const int64_t row = n < ((int64_t)1 << 31) ? (int64_t)((uint32_t)e / (uint32_t)N) : e / N, col = e - row * N;
        store_float<OUT - 1>(q.y, row * q.ldy + col, q.bias ? sum[u] + q.bias[col] : sum[u]);
    }
}

// ---- up to 16 tokens: one pass over b.  A wave has 16 channels and a share of the groups; the waves' sums meet in LDS, in the order of the
// waves.  Lane c + 16 g of a fragment has the blocks 2 g and 2 g + 1 of row c of a group, for two matrix instructions, so that the four
// lanes of a row read its whole line.  U groups are on their way at once.
// FUSED: x is converted by every workgroup for itself, into LDS, while the first of b are on their way.
// Bound by the first bytes of b and the way through LDS at the end: one token 4096 x 4096 3.9 us between others (2.3 TB/s), 16384 x 8192 13.4 (5.3).
struct Mx4FewParams {
    Mx4Product q;
    const void *x;
    int64_t ldx;
    int32_t groups;
};

template <int U, int W, int DT, bool FUSED>
__global__ __launch_bounds__(64 * W) void gemm_mx4_few_kernel(const Mx4FewParams p) {
    __shared__ v4f sums[W][64];
    extern __shared__ __attribute__((aligned(16))) uint8_t own[];            // FUSED: codes of the tokens, and their scales
    const Mx4Product &q = p.q;
    const int t = threadIdx.x, lane = t & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int M = (int)q.a.rows;
    const int64_t N = q.b.rows, n0 = (int64_t)workgroup() * 16;
    const int64_t nr = n0 + c < N ? n0 + c : N - 1;
    const uint8_t *const b = q.b.codes + nr * 128 + 32 * g, *const bs = q.b.scales + nr * 8 + 2 * g;
    const int64_t b_step = N * 128, bs_step = q.b.scale_rows * 8, a_step = M * 128, as_step = q.a.scale_rows * 8;
    const uint8_t *const a = q.a.codes + (c < M ? c : M - 1) * 128 + 32 * g, *const as = q.a.scales + (c < M ? c : M - 1) * 8 + 2 * g;
    v4i bw[U][2], aw[U][2];
    int bsw[U], asw[U];
    const auto request = [&](int s0) {                      // groups s0, s0 + W, ...; past the end the last one again
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = s0 + u * W < p.groups ? s0 + u * W : p.groups - 1;
            bw[u][0] = *reinterpret_cast<const v4i *>(b + at * b_step);
            bw[u][1] = *reinterpret_cast<const v4i *>(b + at * b_step + 16);
            bsw[u] = *reinterpret_cast<const uint16_t *>(bs + at * bs_step);
            if constexpr (!FUSED) {
                aw[u][0] = *reinterpret_cast<const v4i *>(a + at * a_step);
                aw[u][1] = *reinterpret_cast<const v4i *>(a + at * a_step + 16);
                asw[u] = *reinterpret_cast<const uint16_t *>(as + at * as_step);
            }
        }
    };
    request(wave);
    const int row_bytes = p.groups * 128;
    uint8_t *const own_scales = own + M * row_bytes;
    if constexpr (FUSED) {
        const int64_t K = q.b.kdim;
        for (int m = 0; m < M; ++m) {
            for (int64_t k = 8 * t; k < p.groups * 256; k += 512 * W) {
                float x[8];
                const int64_t left = K - k;
                load8<DT>(p.x, m * p.ldx + k, left < 8 ? (int)(left < 0 ? 0 : left) : 8, x);
                const uint32_t byte = mx4_byte<HBFP_RNE>(largest_of_quad(mx4_largest8(x)));
                *reinterpret_cast<uint32_t *>(own + m * row_bytes + k / 2) = mx4_codes<8>(x, byte);
                if (t % 4 == 0) own_scales[(m * row_bytes + k / 2) / 16] = (uint8_t)byte;
            }
        }
        __syncthreads();
    }
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = wave; s0 < p.groups; s0 += W * U) {
        if (s0 != wave) request(s0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + u * W;
            if (s < p.groups) {
                if constexpr (FUSED) {
                    const int at = (c < M ? c : 0) * row_bytes + s * 128 + 32 * g;
                    aw[u][0] = *reinterpret_cast<const v4i *>(own + at);
                    aw[u][1] = *reinterpret_cast<const v4i *>(own + at + 16);
                    asw[u] = *reinterpret_cast<const uint16_t *>(own_scales + at / 16);
                }
                acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(four_bit(bw[u][0]), four_bit(aw[u][0]), acc, 4, 4, 0, bsw[u], 0, asw[u]);
                acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(four_bit(bw[u][1]), four_bit(aw[u][1]), acc, 4, 4, 1, bsw[u], 1, asw[u]);
            }
        }
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave > 0 || c >= M) return;
    // lane: token c, channels 4 g + v
    acc = sums[0][lane];
#pragma unroll
    for (int w = 1; w < W; ++w) acc += sums[w][lane];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int64_t n = n0 + 4 * g + v;
        if (n < N) store_float<DT>(q.y, c * q.ldy + n, q.bias ? acc[v] + q.bias[n] : acc[v]);
    }
}

template <int U, int W, int DT, bool FUSED>
int launch_few(Mx4FewParams p, hipStream_t s) {
    p.groups = (int32_t)p.q.b.groups;
    const size_t own = FUSED ? (size_t)p.q.a.rows * (size_t)p.groups * 136 : 0;
    hipLaunchKernelGGL((gemm_mx4_few_kernel<U, W, DT, FUSED>), grid_of(ceil_div(p.q.b.rows, 16)), dim3(64 * W), own, s, p);
    return launch_status();
}
// Waves of a workgroup and groups on their way (W x U).  us with 4 x 4, 8 x 1, 8 x 2: 16 x 4096 x 4096 4.3 all, 1 x 4096 x 4096 3.5, 3.7, 3.6;
// converting inside, with 8 x 1, 8 x 2, 16 x 1: 1 x 4096 x 4096 3.9, 3.8, 3.9, 1 x 16384 x 4096 7.4, 7.8, 8.7, but 1 x 8192 x 8192 8.5, 8.1, 7.4, 4 x 8192 x
// 8192 11.4, 11.4, 10.5
template <int DT>
int launch_few_of(const Mx4FewParams &p, hipStream_t s) {
    return launch_few<2, 8, DT, false>(p, s);
}
template <int DT>
int launch_fused_of(const Mx4FewParams &p, hipStream_t s) {
    return p.q.b.groups >= 32 && p.q.b.rows <= 8192 ? launch_few<1, 16, DT, true>(p, s) : launch_few<1, 8, DT, true>(p, s);
}

// Tile, ring and split of a product: the smallest estimate in us.  `load` workgroups share a compute unit (tiles of 256 x 256 have one to
// themselves and go in rounds); a launch costs `base`, a workgroup `start`, a group `step` where all units are busy and `lone` more that
// it takes alone; y costs `out` a Mi output, the slices of a split product `out` for every one written and read.  Fitted to 140 shapes of 17 to
// 8192 rows and contractions of 100 to 60 000: 0.9 % behind the best of the kernels on average, 18 % at the worst (19 x 516 x 55804).
// us on tiles of 256, 128 and 64: 8192^3 248, 275, 423; 4096^3 38.4, 41.0, 58.4; 2048 x 4096 x 4096 33.1, 23.3, 32.0; 3000 x 6000 x 3000 57, 39, 50;
// 512 x 4096 x 4096 26.9, 11.7, 9.0; 70 x 5003 x 2730 34, 10.9, 7.3.  Tiles of 64 have a ring of two (four workgroups a unit) or of four (two), which is ahead where
// fewer find a place anyhow: 24 x 16384 x 8192 13.7 against 17, 512 x 4096 x 4096 9.5 against 9.0.
struct Mx4Plan {
    int T, ring, splits;
};
Mx4Plan mx4_plan(int64_t M, int64_t N, int64_t groups) {
    struct Cost {
        int T, ring;
        double base, start, step, lone, out;
    };
    static const Cost whole[4] = {{4, 2, 5.4, 10.2, 1.29, 0.0, 0.0},
                                  {2, 2, 5.3, 0.0, 0.45, 0.14, 0.40},
                                  {1, 2, 3.3, 0.35, 0.22, 0.10, 0.0},
                                  {1, 4, 3.2, 0.51, 0.19, 0.06, 0.30}};
    static const Cost split = {1, 4, 4.9, 2.0, 0.17, 0.11, 0.63};
    const double outputs = (double)M * (double)N * 1e-6;
    Mx4Plan best = {1, 4, 1};
    double least = 0.0;
    const auto consider = [&](const Cost &c, int64_t splits) {
        const double wgs = (double)(ceil_div(M, 64 * c.T) * ceil_div(N, 64 * c.T) * splits), g = (double)ceil_div(groups, splits);
        const double load = c.T == 4 ? ceil(wgs / 256.0) : wgs > 256.0 ? wgs / 256.0 : 1.0, busy = wgs < 256.0 ? wgs / 256.0 : 1.0;
        const double us = c.base + load * (c.start + g * c.step) + busy * g * c.lone + (double)(splits > 1 ? splits + 1 : 1) * outputs * c.out;
        if (least == 0.0 || us < least) least = us, best = {c.T, c.ring, (int)splits};
    };
    for (const Cost &c : whole) consider(c, 1);
    for (int64_t s = 2; s <= 32 && groups / s >= 4 && ceil_div(M, 64) * ceil_div(N, 64) * s <= 600; s *= 2) consider(split, s);
    return best;
}

template <int T, int RING, int OUT>
int launch_tiles(const Mx4Params &p, bool stream, hipStream_t s) {
    static std::atomic<bool> configured[2];
    constexpr int lds_bytes = Mx4Tile<T, RING>::kLds;
    constexpr bool kStreams = OUT == kWideF32;      // (16-bit outputs leave by ordinary stores)
    stream = stream && kStreams;
    void (*const kernel)(Mx4Params) = stream ? &gemm_mx4_kernel<T, RING, OUT, kStreams> : &gemm_mx4_kernel<T, RING, OUT, false>;
    if (allow_dynamic_lds(configured[stream], reinterpret_cast<const void *>(kernel), lds_bytes) != HBFP_OK) return HBFP_ERR_LAUNCH;
    const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
    const dim3 grid = p.splits >= 8 ? dim3((unsigned)(8 * tiles * ceil_div(p.splits, 8))) : dim3((unsigned)(ceil_div(tiles, 8) * 8), (unsigned)p.splits);
    hipLaunchKernelGGL(kernel, grid, dim3(256), lds_bytes, s, p);
    return launch_status();
}
template <int OUT>
int launch_planned(Mx4Params p, const Mx4Plan &plan, hipStream_t s) {
    p.groups = (int32_t)p.q.b.groups;
    p.groups_per_split = (int32_t)ceil_div(p.groups, plan.splits);
    p.splits = (int32_t)ceil_div(p.groups, p.groups_per_split);
    p.tiles_m = (int32_t)ceil_div(p.q.a.rows, 64 * plan.T);
    p.tiles_n = (int32_t)ceil_div(p.q.b.rows, 64 * plan.T);
    GemmArgs g = {};
    g.M = p.q.a.rows;
    g.N = p.q.b.rows;
    g.C = (float *)p.q.y;
    g.ldc = p.q.ldy;
    const bool stream = stores_stream(&g);
    const int rc = plan.T == 4   ? launch_tiles<4, 2, OUT>(p, stream, s)
                   : plan.T == 2 ? launch_tiles<2, 2, OUT>(p, stream, s)
                                 : (plan.ring == 2 ? launch_tiles<1, 2, OUT>(p, stream, s) : launch_tiles<1, 4, OUT>(p, stream, s));
    if (rc != HBFP_OK || p.splits == 1) return rc;
    hipLaunchKernelGGL(mx4_sum_kernel<OUT>, dim3((unsigned)ceil_div(g.M * g.N, 1024)), dim3(256), 0, s, p);
    return launch_status();
}

// Up to 16 tokens are one pass over b, on its own kernel or on tiles of 64 channels.  us on the one and the other: 16 x 4096 x 4096 4.3 and 6.4,
// 16 x 8192 x 1024 3.3 and 4.4, 1 x 1024 x 16384 7.2 and 14; but where there are tiles enough, 16 x 16384 x 8192 18.6 and 13.6, 16 x 12288 x 4096
// 8.2 and 6.9, and where the contraction is long enough to be split, 16 x 512 x 16384 10.5 and 8.2, 4 x 2048 x 30000 16.4 and 10.7.
bool few_rows(int64_t M, int64_t N, int64_t groups) { return M <= 16 && N < 12288 && groups < 64; }

}  // namespace

bool gemm_mx4_fits(int64_t M, int64_t N, int64_t groups) {
    if (one_row(round_up(ceil_div(M, 64) * ceil_div(N, 64), 8), 256) || few_rows(M, N, groups)) return true;
    const int T = mx4_plan(M, N, groups).T;
    return one_row(round_up(ceil_div(M, 64 * T) * ceil_div(N, 64 * T), 8), 256);
}

size_t gemm_mx4_workspace(int64_t M, int64_t N, int64_t groups) {
    if (few_rows(M, N, groups)) return 0;
    const Mx4Plan plan = mx4_plan(M, N, groups);
    return plan.splits > 1 ? (size_t)plan.splits * (size_t)M * (size_t)N * 4 : 0;
}

int launch_gemm_mx4(const Mx4Product &q, void *workspace, hipStream_t s) {
    const int64_t M = q.a.rows, N = q.b.rows, groups = q.b.groups;
    if (few_rows(M, N, groups)) {
        const Mx4FewParams p = {q, nullptr, 0, 0};
        return q.dtype == HBFP_F32 ? launch_few_of<HBFP_F32>(p, s) : q.dtype == HBFP_BF16 ? launch_few_of<HBFP_BF16>(p, s) : launch_few_of<HBFP_F16>(p, s);
    }
    const Mx4Plan plan = mx4_plan(M, N, groups);
    const Mx4Params p = {q, (float *)workspace, 0, 0, 0, 0, 0};
    return q.dtype == HBFP_F32    ? launch_planned<kWideF32>(p, plan, s)
           : q.dtype == HBFP_BF16 ? launch_planned<kWideBf16>(p, plan, s)
                                  : launch_planned<kWideF16>(p, plan, s);
}

// What converting x in every workgroup costs grows with the tokens and the workgroups.  us fused and in two launches (each of which also costs
// the host 4): 1 x 4096 x 4096 3.9 and 6.3, 4 x 4096 x 4096 5.0 and 6.5, 8 x 4096 x 4096 6.5 and 6.7, 16 x 4096 x 4096 9.0 and 7.0; 1 x 16384 x 8192
// 13.4 and 15.8, 2 x 16384 x 8192 15.0 and 15.8, 4 x 16384 x 8192 17.2 and 15.9
bool linear_mx4_fused_ok(int64_t M, int64_t N, int64_t groups) { return M * (groups > 16 ? groups : 16) <= (N <= 8192 ? 128 : 64); }

int launch_linear_mx4_fused(const Mx4Product &q, const void *x, int64_t ldx, hipStream_t s) {
    const Mx4FewParams p = {q, x, ldx, 0};
    return q.dtype == HBFP_F32 ? launch_fused_of<HBFP_F32>(p, s) : q.dtype == HBFP_BF16 ? launch_fused_of<HBFP_BF16>(p, s) : launch_fused_of<HBFP_F16>(p, s);
}

}  // namespace hbfp
