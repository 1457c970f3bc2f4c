// bfloat16 GEMMs of the token statistics and their gradient.
#include "api_internal.h"
#include "few_tokens.h"

namespace dppo {
namespace {

DeviceSetup g_setup;
// Of the logits of a call with alternatives, those of leading tiles are stored whole, and of the rest what exceeds the bound found there (see
// stats_lead_tiles): 12 % and some 13 % with 20 alternatives of 151936. 8191 tokens of D = 2560, GEMM and bound, lead of a quarter / an
// eighth / a sixteenth / none 4545 / 4555 / 4618 / 4982 us (4435 without alternatives), 3000 tokens 1754 / 1731 / 1760 / -, 300 355 / 354
// / 400 / 377.
constexpr int LEAD_ROUNDS = 10;
typedef EpiStore<2> EpiStoreDW16;
// Gradient entries of up to 64 tokens, or where large tiles fill at most half the chip, by tiles of 64 tokens. D = 1152, 64 / 256 tokens a
// tile: 2 tokens, V = 20000 13 / 28 us; 1016, V = 1516 (24 large tiles) 14 / 32, V = 6000 (96) 27 / 32; 300, V = 15160 (120) 26 / 31;
// 250, V = 40000 (157) 40 / 33.
typedef PipeCfg<256, 64, 4, 2, 2, 4, 1> CfgGradFew;
constexpr int GRAD_FEW_TILES = 128;
// Eight wavefronts: where there are few workgroups, the reads of four from LDS show (D = 512, V = 5000: entries of 60 tokens 12.7 / 9.4 us with
// four / eight). Deeper rings of slices are no faster: two workgroups no longer fit a compute unit.
typedef Cfg128Eight CfgSmall;
static_assert(CfgSmall::BN == SMALL_BLOCK_ROWS && CfgSmall::BK == GEMM_B_BLOCK_K, "the blocks of HT");
static_assert((size_t)SMALL_PARTS_MOST * CfgSmall::BM * CfgSmall::BN <= (size_t)256 * CfgBig::BM * CfgBig::BN, "partial tiles fit mfma_dw_partial_bytes()");

hipError_t allow_all() {
    hipError_t e = allow_logits<EpiStats<false, false>>();
    if (e == hipSuccess) e = allow_logits<EpiStats<false, true>>();
    if (e == hipSuccess) e = allow_few<false, FewStats<false>>();
    if (e == hipSuccess) e = allow_lds<CfgBig, EpiStatsGrad>();
    if (e == hipSuccess) e = allow_lds<CfgGradFew, EpiStatsGrad>();
    if (e == hipSuccess) e = allow_lds<CfgSmall, EpiStatsGradBoth, A_ROWS, WG_ROUNDS, B_MAP>();
    if (e == hipSuccess) e = allow_lds<CfgSmall, EpiRows, A_ROWS, WG_ROUNDS, B_KM>();
    if (e == hipSuccess) e = allow_lds<CfgSmall, EpiStoreDW, A_ROWS, WG_RANGES, B_BLK>();
    if (e == hipSuccess) e = allow_lds<CfgSmall, EpiStoreDW16, A_ROWS, WG_RANGES, B_BLK>();
    if (e == hipSuccess) e = allow_lds<CfgGrad, EpiStoreDW16, A_BLK_KM, WG_RANGES, B_BLK>();
    return e;
}

}  // namespace

int mfma_stats_setup(int* compute_units) { return g_setup.run(&allow_all, compute_units); }

void launch_stats_bf16(const LogitsOut& g, const StatsTiles& t, int cus, hipStream_t st) {
    launch_stats_tiles<false>(g, OperandScales{nullptr, nullptr, nullptr, 0}, t, cus, st);
}

int stats_lead_tiles(int tile, int32_t V, int32_t n, int32_t top_k, int cus, int32_t* groups) {
    static_assert(CfgBig::GROUP_M == CfgBig192::GROUP_M && CfgBig::BM == CfgBig192::BM, "the same bands");
    *groups = 0;
    if (top_k == 0 || (tile != TILE_256x256 && tile != TILE_256x192)) return 0;
    const int tiles_m = (int)ceil_div(V, CfgBig::BM), tiles_n = (int)ceil_div(n, tile == TILE_256x256 ? CfgBig::BN : CfgBig192::BN);
    const int tiles = tiles_m * tiles_n, bands = tiles_m / CfgBig::GROUP_M, band = CfgBig::GROUP_M * tiles_n;
    // L leading groups of all G are stored whole, and of the others those that are among a token's top_k of L + 1: a share of top_k / L.
    // L = sqrt(top_k G) stores the least.
    const double all = (double)tiles_m * STATS_GROUPS, best = sqrt(top_k * all);
    const int least = (int)ceil_div(2 * top_k, CfgBig::GROUP_M * STATS_GROUPS);
    int lead = (int)(best / (CfgBig::GROUP_M * STATS_GROUPS) + 0.5);
    // what fits the nearest number of rounds of the chip, one more where that is too little
    int rounds = (lead * band + cus / 2) / cus;
    if (rounds * cus / band < least) ++rounds;
    lead = rounds * cus / band;
    if (2 * lead > bands || lead < least) return 0;
    // a launch more may cost a round more: few rounds are only cut where it does not
    auto in_rounds = [&](int t) { return (t + cus - 1) / cus; };
    if (in_rounds(tiles) < LEAD_ROUNDS && in_rounds(lead * band) + in_rounds(tiles - lead * band) > in_rounds(tiles)) return 0;
    *groups = lead * CfgBig::GROUP_M * STATS_GROUPS;
    return lead * band;
}

void launch_mfma_stats_grad(const void* W, int32_t V, int32_t D, const void* Hc, ChunkView cv, const int32_t* y, const StatsGrad& g, void* G,
                            int32_t Vp, hipStream_t st) {
    EpiStatsGrad e{y, g, cv.n0, cv.n_c, reinterpret_cast<uint16_t*>(G), Vp, V};
    if (cv.n_c <= CfgGradFew::BN || ceil_div(V, CfgBig::BM) * ceil_div(cv.n_c, CfgBig::BN) <= GRAD_FEW_TILES)
        launch<CfgGradFew>(W, D, Hc, D, V, round_up32(cv.n_c, CfgGradFew::BN), D, e, st);
    else
        launch<CfgBig>(W, D, Hc, D, V, cv.n_cp, D, e, st);
}

void launch_mfma_dw_bf16(int cus, const void* G, int32_t Vp, const void* HcT, int32_t n_cp, int32_t V, int32_t D, void* dW, float* partial,
                         hipStream_t st) {
    EpiStoreDW16 e{nullptr, reinterpret_cast<uint16_t*>(dW), D, 0, nullptr, nullptr, nullptr};
    launch_dw_tiles(cus, G, Vp, HcT, n_cp, V, D, e, partial, n_cp <= 2 * CfgGrad::BK, st);
}

void launch_small_grad(const SmallGrad& s, const int32_t* y, const StatsGrad& g, hipStream_t st) {
    EpiStatsGradBoth e{y, g, s.cv.n0, reinterpret_cast<uint16_t*>(s.G), s.Vk, reinterpret_cast<uint16_t*>(s.GT), s.n_sum};
    launch<CfgSmall, A_ROWS, WG_ROUNDS, B_MAP>(s.W, s.D, s.H, s.D, s.V, s.cv.n_c, s.D, e, st, 0, -1, 1, -1, (int)s.h_rows, 0, s.map);
}

void launch_small_dh(const SmallGrad& s, const StoreSpec& out, int cus, hipStream_t st) {
    const int tiles_m = (int)ceil_div(s.cv.n_c, CfgSmall::BM), tiles_n = (int)ceil_div(s.D, CfgSmall::BN), tiles = tiles_m * tiles_n;
    const int parts = small_tiles_parts(cus, tiles, s.Vk / CfgSmall::BK);
    EpiRows e{reinterpret_cast<uint16_t*>(out.C), out.ldc, out.row_map, parts > 1 ? s.partial : nullptr};
    launch<CfgSmall, A_ROWS, WG_ROUNDS, B_KM>(s.G, s.Vk, s.W, s.D, s.cv.n_c, s.D, s.Vk, e, st, 0, tiles, parts, -1, s.V);
    if (parts > 1)
        sum_partial_tiles_kernel<CfgSmall><<<dim3(tiles, CfgSmall::BM / sum_rows<CfgSmall>()), 256, 0, st>>>(
            s.partial, 0, parts, tiles_m, tiles_n, nullptr, out.ldc, s.cv.n_c, s.D, 0, e.C, out.row_map, nullptr);
}

void launch_small_dw(const SmallGrad& s, const StoreSpec& out, bool bf16, int cus, hipStream_t st) {
    const int tiles_m = (int)ceil_div(s.V, CfgSmall::BM), tiles_n = (int)ceil_div(s.D, CfgSmall::BN), tiles = tiles_m * tiles_n;
    const int parts = small_tiles_parts(cus, tiles, s.n_sum / CfgSmall::BK);
    float *Cf = bf16 ? nullptr : reinterpret_cast<float*>(out.C), *partial = parts > 1 ? s.partial : nullptr;
    uint16_t* Cb = bf16 ? reinterpret_cast<uint16_t*>(out.C) : nullptr;
    if (bf16) {
        EpiStoreDW16 e{Cf, Cb, out.ldc, 0, nullptr, nullptr, partial};
        launch<CfgSmall, A_ROWS, WG_RANGES, B_BLK>(s.GT, s.n_sum, s.HT, 0, s.V, s.D, s.n_sum, e, st, 0, tiles, parts);
    } else {
        EpiStoreDW e{Cf, Cb, out.ldc, out.accumulate, nullptr, nullptr, partial};
        launch<CfgSmall, A_ROWS, WG_RANGES, B_BLK>(s.GT, s.n_sum, s.HT, 0, s.V, s.D, s.n_sum, e, st, 0, tiles, parts);
    }
    if (parts > 1)
        sum_partial_tiles_kernel<CfgSmall><<<dim3(tiles, CfgSmall::BM / sum_rows<CfgSmall>()), 256, 0, st>>>(
            s.partial, 0, parts, tiles_m, tiles_n, Cf, out.ldc, s.V, s.D, out.accumulate, Cb, nullptr, nullptr);
}

}  // namespace dppo
