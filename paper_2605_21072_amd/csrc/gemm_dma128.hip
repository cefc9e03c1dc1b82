// Plain and chained (INT8 out) builds of the GEMM on 128-byte K stages; the kernel stands in gemm_dma128.h.
#include "gemm_dma128.h"

namespace qarvd_gemm {

template <int BM, int BN, int WM, int WN, int NSTAGE, bool DUAL, bool GEN, bool W4>
qarvd_status launch_dma128(const GemmArgs &g0, qarvd_dtype ydt, hipStream_t st)
{
    GemmArgs g = g0;
    g.tiles_m = (g.M + BM - 1) / BM;
    g.tiles_n = (g.N + BN - 1) / BN;
    const bool dbg = g.dbg_n != nullptr || g.dbg_o != nullptr;   // raw-accumulator dumps: separate, slower build
    if (ydt == QARVD_BF16)
        return !dbg ? launch128_one<BM, BN, WM, WN, NSTAGE, DUAL, false, uint16_t, GEN, W4>(g, st)
                    : launch128_one<BM, BN, WM, WN, NSTAGE, DUAL, true, uint16_t, GEN, W4>(g, st);
    return !dbg ? launch128_one<BM, BN, WM, WN, NSTAGE, DUAL, false, float, GEN, W4>(g, st)
                : launch128_one<BM, BN, WM, WN, NSTAGE, DUAL, true, float, GEN, W4>(g, st);
}

template <int BM, int BN, int WM, int WN, int NSTAGE, bool DUAL>
qarvd_status launch_dma128_q8(const GemmArgs &g0, hipStream_t st)
{
    GemmArgs g = g0;
    g.tiles_m = (g.M + BM - 1) / BM;
    g.tiles_n = (g.N + BN - 1) / BN;
    return g.act == 1 ? launch128_one<BM, BN, WM, WN, NSTAGE, DUAL, false, Int8GeluOut, false, false>(g, st)
                      : launch128_one<BM, BN, WM, WN, NSTAGE, DUAL, false, Int8Out, false, false>(g, st);
}

#define QARVD_INST128_Q8(BM, BN, WM, WN, NS)                                                         \
    template qarvd_status launch_dma128_q8<BM, BN, WM, WN, NS, true>(const GemmArgs &, hipStream_t); \
    template qarvd_status launch_dma128_q8<BM, BN, WM, WN, NS, false>(const GemmArgs &, hipStream_t);
QARVD_INST128_Q8(256, 256, 2, 4, 2)
QARVD_INST128_Q8(256, 128, 4, 2, 3)
QARVD_INST128_Q8(128, 256, 2, 4, 3)
QARVD_INST128_Q8(128, 128, 4, 2, 3)

#define QARVD_INST128(BM, BN, WM, WN, NS)                                                                        \
    template qarvd_status launch_dma128<BM, BN, WM, WN, NS, true, false, false>(const GemmArgs &, qarvd_dtype, hipStream_t);   \
    template qarvd_status launch_dma128<BM, BN, WM, WN, NS, false, false, false>(const GemmArgs &, qarvd_dtype, hipStream_t);
QARVD_INST128(256, 256, 2, 4, 2)
QARVD_INST128(256, 128, 4, 2, 3)
QARVD_INST128(128, 256, 2, 4, 3)
QARVD_INST128(128, 128, 2, 4, 3)
QARVD_INST128(64, 128, 2, 4, 4)
QARVD_INST128(64, 64, 2, 2, 4)

#define QARVD_INST128_GEN(BM, BN, WM, WN, NS)                                                                    \
    template qarvd_status launch_dma128<BM, BN, WM, WN, NS, true, true, false>(const GemmArgs &, qarvd_dtype, hipStream_t);
QARVD_INST128_GEN(128, 128, 2, 4, 3)
QARVD_INST128_GEN(64, 128, 2, 4, 4)
QARVD_INST128_GEN(64, 64, 2, 2, 4)

#define QARVD_INST128_W4(BM, BN, WM, WN, NS, GEN)                                                                    \
    template qarvd_status launch_dma128<BM, BN, WM, WN, NS, true, GEN, true>(const GemmArgs &, qarvd_dtype, hipStream_t);
QARVD_INST128_W4(256, 256, 2, 4, 3, false)
QARVD_INST128_W4(256, 128, 4, 2, 3, false)
QARVD_INST128_W4(128, 256, 2, 4, 3, false)
QARVD_INST128_W4(128, 128, 2, 4, 3, true)
QARVD_INST128_W4(64, 64, 2, 2, 3, true)

}  // namespace qarvd_gemm
