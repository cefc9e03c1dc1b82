// GEMM on 128-byte K stages with an activation, a gate and a residual in its epilogue (the kernel stands in gemm_dma128.h).  The ending is a
// build of its own: chosen at run time in every block of an epilogue that is unrolled over the wave tile, it would double its code.  One
// build serves layers with and without outliers.
#include "gemm_dma128.h"

namespace qarvd_gemm {

template <int BM, int BN, int WM, int WN, int NSTAGE, bool GEN, bool W4>
qarvd_status launch_dma128_fused(const GemmArgs &g0, qarvd_dtype ydt, hipStream_t st)
{
    GemmArgs g = g0;
    g.tiles_m = (g.M + BM - 1) / BM;
    g.tiles_n = (g.N + BN - 1) / BN;
    const bool gelu = g.act == QARVD_ACT_GELU_TANH, res = g.gate || g.R || !gelu;
    auto as = [&](auto out) {
        using OutT = decltype(out);
        if (!res) return launch128_one<BM, BN, WM, WN, NSTAGE, true, false, OutT, GEN, W4, true, ENDING_GELU>(g, st);
        if constexpr (BM * BN <= 128 * 256) {
            if (!gelu) return launch128_one<BM, BN, WM, WN, NSTAGE, true, false, OutT, GEN, W4, true, ENDING_RESIDUAL>(g, st);
            return launch128_one<BM, BN, WM, WN, NSTAGE, true, false, OutT, GEN, W4, true, ENDING_GELU | ENDING_RESIDUAL>(g, st);
        }
        return QARVD_ERR_UNSUPPORTED;       // no registers for the residual of a 256 x 256 tile
    };
    return ydt == QARVD_BF16 ? as(uint16_t{}) : as(float{});
}

#define QARVD_INST128_FUSED(BM, BN, WM, WN, NS, GEN, W4)                                                          \
    template qarvd_status launch_dma128_fused<BM, BN, WM, WN, NS, GEN, W4>(const GemmArgs &, qarvd_dtype, hipStream_t);
#ifndef QARVD_FUSED_GENERAL
QARVD_INST128_FUSED(256, 256, 2, 4, 2, false, false)
QARVD_INST128_FUSED(256, 128, 4, 2, 3, false, false)
QARVD_INST128_FUSED(128, 256, 2, 4, 3, false, false)
QARVD_INST128_FUSED(128, 128, 2, 4, 3, false, false)
QARVD_INST128_FUSED(64, 128, 2, 4, 4, false, false)
QARVD_INST128_FUSED(64, 64, 2, 2, 4, false, false)
#else
QARVD_INST128_FUSED(256, 256, 2, 4, 3, false, true)
QARVD_INST128_FUSED(256, 128, 4, 2, 3, false, true)
QARVD_INST128_FUSED(128, 256, 2, 4, 3, false, true)
QARVD_INST128_FUSED(128, 128, 2, 4, 3, true, true)
QARVD_INST128_FUSED(64, 64, 2, 2, 3, true, true)
QARVD_INST128_FUSED(128, 128, 2, 4, 3, true, false)
QARVD_INST128_FUSED(64, 128, 2, 4, 4, true, false)
QARVD_INST128_FUSED(64, 64, 2, 2, 4, true, false)
#endif

}  // namespace qarvd_gemm
