// Instantiations and host launchers of the bf16 MFMA GEMM kernels (see gemm_mfma_kernel.h).
#include <atomic>

#include "gemm_mfma_launch.h"

namespace dppo {

namespace {
std::atomic<unsigned long long*> g_phase_counters{nullptr};
DeviceSetup g_setup;

hipError_t allow_all() {
    hipError_t e = allow_lds<CfgGrad, EpiStoreDW, A_BLK_KM, WG_RANGES, B_BLK>();
    if (e == hipSuccess) e = allow_lds<CfgGrad, EpiStoreDH, A_BLK_ROWS, WG_RANGES, B_BLK>();
    if (e == hipSuccess) e = allow_lds<CfgGrad, EpiStoreDH, A_BLK_ROWS, WG_RANGES, B_KM>();
    if (e == hipSuccess) e = allow_lds<CfgBig, EpiLogits>();
    if (e == hipSuccess) e = allow_lds<CfgBig192, EpiScore, A_ROWS, WG_ROUNDS, B_MAP>();
    if (e == hipSuccess) e = allow_lds<CfgFew<96>, EpiScore, A_ROWS, WG_ROUNDS, B_MAP>();
    if (e == hipSuccess) e = allow_lds<CfgFew<128>, EpiScore, A_ROWS, WG_ROUNDS, B_MAP>();
    if (e == hipSuccess) e = allow_lds<CfgBig, EpiLogitsExp>();
    if (e == hipSuccess) e = allow_lds<CfgBig, EpiLogitsGrad>();
    return e;
}
}  // namespace

int mfma_setup(int* compute_units) { return g_setup.run(&allow_all, compute_units); }

unsigned long long* mfma_phase_counters() { return g_phase_counters.load(); }
void mfma_set_phase_counters(unsigned long long* counters) { g_phase_counters.store(counters); }

int32_t mfma_logits_row_tiles(int32_t V) { return (int32_t)ceil_div(V, CfgBig::BM); }
int32_t mfma_vocab_tile() { return CfgBig::BM; }

// Columns of 192 tokens where they cover the chunk with as many tiles as columns of 256.
static bool narrow_columns(int32_t n_c) { return n_c <= (int32_t)ceil_div(n_c, CfgBig::BN) * CfgBig192::BN; }
bool mfma_logits_reads_tokens(int32_t n_c) { return narrow_columns(n_c); }

LogitsPart launch_mfma_logits(const void* W, int32_t V, int32_t D, const void* Hc, const TokenArgs& tokens, bool look_up, ChunkView cv, float2* part,
                              float* zy, hipStream_t st) {
    const int32_t n_c = cv.n_c;
    LogitsPart lp{mfma_logits_row_tiles(V), cv.n_cp};
    const int32_t* map = tokens.loss_pos ? tokens.loss_pos + cv.n0 : nullptr;
    const uint16_t* rows = reinterpret_cast<const uint16_t*>(tokens.H) + (map ? 0 : (size_t)cv.n0 * D);
    auto narrow = [&](auto cfg, int64_t pitch) {
        typedef decltype(cfg) Cfg;
        EpiScore e{{part, pitch}, tokens, cv.n0, n_c, zy};
        launch<Cfg, A_ROWS, WG_ROUNDS, B_MAP>(W, D, rows, D, V, n_c, D, e, st, 0, -1, 1, -1, (int)tokens.T, 0, map,
                                              look_up ? (int)ceil_div(n_c, Cfg::NW) : 0);
    };
    if (n_c <= LOGITS_FEW_TOKENS) {
        // as many pairs in all as with 256-row tiles: twice the row tiles, half the pitch
        lp = LogitsPart{(int32_t)ceil_div(V, CfgFew<128>::BM), LOGITS_FEW_TOKENS};
        if (n_c <= 96) narrow(CfgFew<96>{}, lp.pitch);
        else narrow(CfgFew<128>{}, lp.pitch);
    } else if (narrow_columns(n_c)) {
        narrow(CfgBig192{}, cv.n_cp);
    } else {
        launch<CfgBig>(W, D, Hc, D, V, cv.n_cp, D, EpiLogits{part, cv.n_cp}, st, 0, -1, 1, PHASE_LOGITS);
    }
    return lp;
}

int launch_mfma_logits_exp(const void* W, int32_t V, int32_t D, const void* Hc, int32_t n_cp, float2* part,
                           const float* bref, void* E, int64_t lde, int32_t Vp, hipStream_t st) {
    // the epilogue stores whole tiles: the caller pads the row pitch to whole vocabulary tiles
    if (Vp % CfgBig::BM != 0 || lde != Vp || Vp < V)
        return fail(DPPO_ERR_UNSUPPORTED, "chunk buffer not padded to whole vocabulary tiles (Vp %d, pitch %lld)", Vp,
                    (long long)lde);
    EpiLogitsExp e{part, n_cp, bref, reinterpret_cast<uint16_t*>(E), lde};
    launch<CfgBig>(W, D, Hc, D, V, n_cp, D, e, st, 0, -1, 1, PHASE_LOGITS);
    return DPPO_OK;
}

int launch_mfma_logits_grad(const void* W, int32_t V, int32_t D, const void* Hc, int32_t n_cp,
                            const int32_t* y, const float* lse, const float* c, void* G, int64_t ldg,
                            int32_t Vp, hipStream_t st) {
    if (Vp % CfgBig::BM != 0 || ldg != Vp || Vp < V)
        return fail(DPPO_ERR_UNSUPPORTED, "gradient-logits buffer not padded to whole vocabulary tiles (Vp %d, pitch %lld)",
                    Vp, (long long)ldg);
    EpiLogitsGrad e{y, lse, c, reinterpret_cast<uint16_t*>(G), ldg, n_cp, V};
    launch<CfgBig>(W, D, Hc, D, V, n_cp, D, e, st);
    return DPPO_OK;
}

size_t mfma_dw_partial_bytes() { return (size_t)256 * CfgBig::BM * CfgBig::BN * 4; }

// One workgroup per compute unit at a time: the last round of tiles holds tiles % cus of them. If
// that is at most half the chip, those tiles are cut along K into as many parts as fill it (at
// least 16 slices each), each part writes its partial tile to scratch, and a small
// kernel adds the parts up in order (the same sums in a different association; deterministic).
// The parts of a launch never hold more than one tile per compute unit, so many parts of few tiles cost the sum no
// more than few parts of many (64 MB in all). With at most 8 parts, 250 tokens of D = 4096 (16 tiles of dH) kept half the
// chip idle: 437 us, now 290.
int mfma_tail_parts(int cus, int tail, int k_slices) {
    if (tail <= 0 || 2 * tail > cus) return 1;
    int parts = cus / tail;
    if (parts > k_slices / 16) parts = k_slices / 16;
    if ((size_t)tail * parts * CfgBig::BM * CfgBig::BN * 4 > mfma_dw_partial_bytes()) parts = 1;
    return parts < 2 ? 1 : parts;
}
int mfma_dh_slices(int32_t V) { return mfma_logits_row_tiles(V) * (CfgBig::BM / CfgGrad::BK); }

namespace {
// Parts along K for the `tail` tiles of dH's last round where the scratch holds `room` partial tiles. With room for one per
// compute unit only whole sets of parts fit beside each other (and a round that is more than half full stays whole). With more,
// several rounds of parts: what is least of rounds / parts of a tile's time and a fifth of a slice's time for every partial tile
// (512 KB to write and read, and dW's stores behind it find its memory dirty). A round that is partly full is not that much
// longer than its share, as the chip runs at its power limit: 140, 220 and 250 tiles 3.13, 3.43 and 3.66 ms. V = 151936, D = 2560,
// dH and dW, whole / split: 3800 tokens (150 tiles) 5.40 / 4.76 ms, 4900 (200) 6.26 / 6.13, 5400 (220) 6.71 / 6.88, 10500 (420)
// 12.22 / 12.00; D = 4096, V = 100000 2300 tokens (144) 3.57 / 3.22.
int dh_tail_parts(int cus, int tail, int k_slices, int64_t room) {
    if (cus <= 0 || tail <= 0) return 1;
    int best = mfma_tail_parts(cus, tail, k_slices);
    if (room <= cus) return best;
    auto time = [&](int p) {
        const int items = tail * p;
        const double rounds = items / cus + (items % cus ? 0.7 + 0.3 * (items % cus) / cus : 0.0);
        return rounds / p + (p > 1 ? (0.2 * items + 5.0) / k_slices : 0.0);
    };
    double best_t = 0.98 * time(best);
    for (int p = best + 1; p <= k_slices / 16 && (int64_t)tail * p <= room && tail * p <= 8 * cus; ++p)
        if (time(p) < best_t) { best_t = time(p); best = p; }
    return best;
}

template <int BL>
void launch_dh(int cus, const void* G, int32_t Vp, const void* B, int64_t ldb, int b_rows, int32_t n_c, int32_t D,
               const float* row_scale, const StoreSpec& out, float* partial, int64_t partial_floats, hipStream_t st) {
    EpiStoreDH e{nullptr, reinterpret_cast<uint16_t*>(out.C), out.ldc, 0, out.row_map, row_scale, nullptr};
    const int tiles_m = (int)ceil_div(n_c, CfgGrad::BM), tiles_n = (int)ceil_div(D, CfgGrad::BN);
    const int tiles = tiles_m * tiles_n;
    const int tail = cus > 0 ? tiles % cus : 0;
    const int parts = partial ? dh_tail_parts(cus, tail, Vp / CfgGrad::BK, partial_floats / (CfgGrad::BM * CfgGrad::BN)) : 1;
    if (parts == 1) {
        launch<CfgGrad, A_BLK_ROWS, WG_RANGES, BL>(G, Vp, B, ldb, n_c, D, Vp, e, st, 0, -1, 1, PHASE_DH, b_rows);
        return;
    }
    launch<CfgGrad, A_BLK_ROWS, WG_RANGES, BL>(G, Vp, B, ldb, n_c, D, Vp, e, st, 0, tiles - tail, 1, PHASE_DH, b_rows);
    EpiStoreDH ep = e;
    ep.partial = partial;
    launch<CfgGrad, A_BLK_ROWS, WG_RANGES, BL>(G, Vp, B, ldb, n_c, D, Vp, ep, st, tiles - tail, tail, parts, -1, b_rows);
    sum_partial_tiles_kernel<CfgGrad><<<dim3(tail, CfgGrad::BM / sum_rows<CfgGrad>()), 256, 0, st>>>(
        partial, tiles - tail, parts, tiles_m, tiles_n, nullptr, out.ldc, n_c, D, 0, reinterpret_cast<uint16_t*>(out.C),
        out.row_map, row_scale);
}
}  // namespace

void launch_mfma_dh(int cus, const void* G, int32_t Vp, const void* WT, const void* W, int32_t V, int32_t n_c, int32_t D,
                    const float* row_scale, const StoreSpec& out, float* partial, int64_t partial_floats, hipStream_t st) {
    if (WT) launch_dh<B_BLK>(cus, G, Vp, WT, 0, 0, n_c, D, row_scale, out, partial, partial_floats, st);
    else launch_dh<B_KM>(cus, G, Vp, W, D, V, n_c, D, row_scale, out, partial, partial_floats, st);
}

// Whether dW's tiles are walked by resident workgroups, one per compute unit, that load a tile's first slices while the one
// before is stored. Added to what is there, that hides the reading of the old values, until a long chunk's shared panels
// matter more: residents drift apart, and a chunk of 32234 tokens of D = 2560 misses the L2 for 65 GB instead of 48. Overwritten,
// it pays with one or two slices a tile only; further on the loads disturb the stores. dW stage, resident / one tile each, V =
// 151936:
//   added        D = 4096: 250 tokens 1.058 / 1.140 ms, 4000 4.186 / 4.239, 24576 21.94 / 21.80
//                D = 2560: 1300 tokens 1.245 / 1.289, 16384 9.297 / 9.324, 32256 17.81 / 17.67
//   overwritten  D = 4096: 40 tokens 0.473 / 0.496, 100 0.647 / 0.620, 130 0.743 / 0.675, 1500 1.901 / 1.820, 24576 21.64 / 21.51
//                D = 2560: 100 tokens 0.361 / 0.372, 250 0.473 / 0.446, 1300 1.031 / 1.059, 32256 17.63 / 17.48
static bool dw_resident(int32_t tokens, int accumulate) {
    return tokens <= (accumulate ? 16384 : 2 * CfgGrad::BK);
}

void launch_mfma_dw(int cus, const void* G, int32_t Vp, const void* HcT, int32_t n_cp, int32_t V, int32_t D,
                    const StoreSpec& out, float* partial, hipStream_t st) {
    EpiStoreDW e{reinterpret_cast<float*>(out.C), nullptr, out.ldc, out.accumulate, nullptr, nullptr, nullptr};
    launch_dw_tiles(cus, G, Vp, HcT, n_cp, V, D, e, partial, dw_resident(n_cp, out.accumulate), st);
}

// Register-only loop of the GEMMs' MFMA instruction (8 wavefronts per compute unit, 32 independent
// accumulator blocks each, operands never leave the registers): the rate the matrix pipes sustain
// when nothing has to be loaded, which is the ceiling the GEMMs are priced against. With random operand
// values the chip's power limit lowers the clock, so the ceiling depends on the data.
namespace {
__device__ __forceinline__ mfma::bf16x8 probe_operand(unsigned seed, int random_values) {
    mfma::bf16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        unsigned h = (seed * 8u + (unsigned)i) * 2654435761u;
        h ^= h >> 15; h *= 2246822519u; h ^= h >> 13;
        const float f = random_values ? (float)((int)(h % 2001u) - 1000) * 0.001f : 1.0f;
        v[i] = (__bf16)f;
    }
    return v;
}
__global__ __launch_bounds__(512) void mfma_rate_kernel(float* out, int iters, int random_values) {
    mfma::bf16x8 a[8], b[4];
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = probe_operand(threadIdx.x * 7u + (unsigned)i + blockIdx.x * 1000u, random_values);
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = probe_operand(threadIdx.x * 13u + (unsigned)i + 77u, random_values);
    mfma::f32x4 acc[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) acc[i] = mfma::f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int it = 0; it < iters; ++it) {
#pragma unroll
        for (int q = 0; q < 32; ++q) acc[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[q / 4], b[q % 4], acc[q], 0, 0, 0);
    }
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += acc[i][0] + acc[i][1] + acc[i][2] + acc[i][3];
    if (threadIdx.x == 0) out[blockIdx.x] = s;      // keeps the loop alive; one float per workgroup
}
}  // namespace

double launch_mfma_rate_probe(int cus, int iters, int random_values, float* out, hipStream_t st) {
    mfma_rate_kernel<<<cus, 512, 0, st>>>(out, iters, random_values);
    return (double)cus * 8.0 * (double)iters * 32.0 * 16384.0;   // 8 wavefronts x 32 MFMAs x 2 x 16 x 16 x 32 flop
}

}  // namespace dppo
