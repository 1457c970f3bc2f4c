// bfloat16 GEMMs of the token statistics and their gradient.
#include "stats_epilogues.h"

namespace dppo {
namespace {

DeviceSetup g_setup;
typedef EpiStore<2> EpiStoreDW16;

hipError_t allow_all() {
    hipError_t e = allow_logits<EpiStats<false, false>>();
    if (e == hipSuccess) e = allow_logits<EpiStats<false, true>>();
    if (e == hipSuccess) e = allow_lds<CfgBig, EpiStatsGrad>();
    if (e == hipSuccess) e = allow_lds<CfgGrad, EpiStoreDW16, A_BLK_KM, WG_RANGES, B_BLK>();
    return e;
}

}  // namespace

int mfma_stats_setup(int* compute_units) { return g_setup.run(&allow_all, compute_units); }

void launch_stats_bf16(const LogitsOut& g, const StatsTiles& t, hipStream_t st) {
    launch_stats_tiles<false>(g, OperandScales{nullptr, nullptr, nullptr, 0}, t, st);
}

void launch_mfma_stats_grad(const void* W, int32_t V, int32_t D, const void* Hc, ChunkView cv, const int32_t* y, const StatsGrad& g, void* G,
                            int32_t Vp, hipStream_t st) {
    EpiStatsGrad e{y, g, cv.n0, cv.n_c, reinterpret_cast<uint16_t*>(G), Vp, V};
    launch<CfgBig>(W, D, Hc, D, V, cv.n_cp, D, e, st);
}

void launch_mfma_dw_bf16(int cus, const void* G, int32_t Vp, const void* HcT, int32_t n_cp, int32_t V, int32_t D, void* dW, float* partial,
                         hipStream_t st) {
    EpiStoreDW16 e{nullptr, reinterpret_cast<uint16_t*>(dW), D, 0, nullptr, nullptr, nullptr};
    launch_dw_tiles(cus, G, Vp, HcT, n_cp, V, D, e, partial, n_cp <= 2 * CfgGrad::BK, st);
}

}  // namespace dppo
