// BFP matrix product with one exponent per operand row: which products the kernel of gemm_wide.h takes, and its launch.
#include "gemm_wide.h"

namespace hbfp {

// One exponent per operand row, 8-bit mantissas, rows of the stored operands addressable with 32-bit offsets
bool gemm_wide_possible(const GemmArgs &a) {
    return !a.P && a.nblk == 1 && a.mA <= 8 && a.mB <= 8 && (uint64_t)255 * (uint64_t)a.kpad + 64 < ((uint64_t)1 << 32) &&
           ceil_div(a.M, 128) * ceil_div(a.N, 128) <= 0x7ffffff0 && a.kpad / 64 <= 0x7fffffff;
}

// ... and a contraction longer than 64, or enough full tiles of 256 x 256 to fill the chip (below, the kernels of short blocks
// scale once per workgroup too)
bool gemm_wide_ok(const GemmArgs &a) {
    if (!gemm_wide_possible(a)) return false;
    if (a.kbp >= 128) return true;
    const int64_t tiles = ceil_div(a.M, 256) * ceil_div(a.N, 256);
    return tiles >= 128 && (double)a.M * (double)a.N >= 0.75 * 65536.0 * (double)tiles;
}

// slices of a product split along k; a stand-by launch is not split, nor one whose caller brought no room for them
size_t gemm_wide_workspace(const GemmArgs &a) {
    const WidePlan plan = wide_plan(a.M, a.N, a.kpad / 64, !a.run_a && !a.unsplit);
    return plan.splits > 1 ? (size_t)plan.splits * (size_t)a.M * (size_t)a.N * 4 : 0;
}

int launch_gemm_wide(const GemmArgs &a, void *workspace, hipStream_t s) {
    const WidePlan plan = wide_plan(a.M, a.N, a.kpad / 64, !a.run_a && !a.unsplit);
    if (plan.splits > 1 && !workspace) return HBFP_ERR_WORKSPACE;
    WideParams p = {};
    p.A = (const uint8_t *)a.mantA;
    p.B = (const uint8_t *)a.mantB;
    p.eA = a.expA;
    p.eB = a.expB;
    p.C = a.C;
    p.partial = (int32_t *)workspace;
    p.M = a.M;
    p.N = a.N;
    p.kpad = a.kpad;
    p.eA_ld = a.expA_ld;
    p.eB_ld = a.expB_ld;
    p.ldc = a.ldc;
    p.beta = a.beta != 0.0f;
    p.exp_offset = -250 - a.mA - a.mB;
    p.run_a = a.run_a;
    p.run_b = a.run_b;
    // Only contractions up to 1024 end in so much of a burst that ordinary stores pay for what C takes of the last-level cache from the
    // conversions beside the product (conversions and product, streaming -> ordinary: 3001 x 600 x 2999 29.3 -> 26.9 us, 5000 x 1024 x
    // 4001 54.6 -> 54.1, 4100 x 1024 x 2501 38.9 -> 34.7, but 5000 x 1200 x 4001 60.5 -> 63.7, 3001 x 4500 x 2999 86.9 -> 88.4)
    const bool stream = a.kpad > 1024 || stores_stream(&a);
    return launch_wide_planned<kWideExponents>(p, plan, stream, s);
}

}  // namespace hbfp
