// Tile shapes, launchers and per-device setup shared by the translation units that instantiate the MFMA GEMM kernel
// (gemm_mfma_kernel.h): each instantiates its own epilogues.
#pragma once
#include <mutex>

#include "gemm_mfma_kernel.h"

namespace dppo {

// Tile-phase counters of the benchmark aid (NULL = off): 4 counters per GEMM stage, see gemm_nt_kernel.
unsigned long long* mfma_phase_counters();

namespace {
using namespace mfma;

// 256x256x64 tile, 2x4 wavefronts (128x64 each), 3 A slices and 2 B slices in flight (all 160 KB of
// LDS), all loads of a slice issued in the k-step that frees its buffers. The blocked chunk layout
// (64 x 256 element blocks) is tied to this tile. The GEMMs differ only in the band height of the
// tile walk: 4 tile rows for the vocabulary GEMM (126 token tiles per row: 4 x 8 blocks per L2);
// 1 for dH and dW, whose rows have only D / 256 = 10 tiles: the A panels there are pieces of the
// 10 GB chunk that streams from HBM, and with one-row bands all 10 users of a panel are
// consecutive tiles and run in the same round (bands of 4 x 10 tiles straddle the rounds of 32:
// dH +1.6 %, dW +1.2 % in time); with such bands a contiguous range of rows per XCD (WG_RANGES)
// is as good (dW) or 0.9 % better (dH) than interleaved rounds.
typedef PipeCfg<256, 256, 2, 4, 2, 4, 1> CfgBig;
typedef PipeCfg<256, 256, 2, 4, 2, 1, 1> CfgGrad;
// Forward-only vocabulary GEMM of few tokens. Up to LOGITS_FEW_TOKENS it is bound by reading W once: 128 vocabulary rows by one
// column of 96 or 128 tokens, four wavefronts, 72 or 80 KB of LDS, so that two workgroups share a compute unit and
// one's prologue, barriers and epilogue fall into the other's loads (33 tokens, whole call: V = 151936, D = 2560
// 222 -> 175 us, D = 4096 361 -> 280 us = W at 4.4 TB/s; V = 32000, D = 1024 35 -> 25 us). 64 columns are no faster
// than 96 (178 and 303 us: too few MFMAs between a k-step's LDS reads). Beyond, the matrix pipes bound it, and where columns of 192 tokens
// cover the chunk with as many tiles as columns of 256, a quarter of the products is saved (333 tokens, D = 4096:
// 478 -> 437 us; 192 tokens 362 -> 347; 520 tokens 658 -> 586).
template <int BN> using CfgFew = PipeCfg<128, BN, 2, 2, 2, 1, 1>;
typedef PipeCfg<256, 192, 2, 4, 2, 4, 1> CfgBig192;
static_assert(CfgGrad::BN == GEMM_B_BLOCK_ROWS && CfgGrad::BK == GEMM_B_BLOCK_K, "blocked B operand = the tile's slices");

// Dynamic LDS of a kernel: the operand slices, or the epilogue's staging area if that is larger.
template <class Cfg, class Epi>
constexpr int lds_request() {
    constexpr int e = Epi::template lds_bytes<Cfg>();
    static_assert(e <= 160 * 1024, "epilogue LDS");
    return Cfg::LDS_BYTES > e ? Cfg::LDS_BYTES : e;
}

enum { PHASE_LOGITS = 0, PHASE_DH = 1, PHASE_DW = 2 };

// Launches the tiles [tile0, tile0 + n_tiles) of the tile walk, each cut into k_parts work items
// along K; n_tiles < 0: all tiles. max_workgroups > 0: at most that many workgroups, which take several items each.
template <class Cfg, int AM = A_ROWS, int MAP = WG_ROUNDS, int BL = B_ROWS, class Epi>
void launch(const void* A, int64_t lda, const void* B, int64_t ldb, int M, int N, int K, const Epi& epi,
            hipStream_t st, int tile0 = 0, int n_tiles = -1, int k_parts = 1, int phase_stage = -1, int b_rows = 0,
            int max_workgroups = 0, const int32_t* b_map = nullptr, int extra_workgroups = 0) {
    const int tiles_m = (int)ceil_div(M, Cfg::BM), tiles_n = (int)ceil_div(N, Cfg::BN);
    if (n_tiles < 0) n_tiles = tiles_m * tiles_n - tile0;
    if (n_tiles <= 0) return;
    unsigned long long* phase = phase_stage >= 0 && k_parts == 1 ? mfma_phase_counters() : nullptr;
    if (phase) phase += 4 * phase_stage;
    const int items = n_tiles * k_parts, workgroups = max_workgroups > 0 && items > max_workgroups ? max_workgroups : items;
    gemm_nt_kernel<Cfg, Epi, AM, MAP, BL><<<dim3(workgroups + extra_workgroups), dim3(Cfg::NT), lds_request<Cfg, Epi>(), st>>>(
        reinterpret_cast<const uint16_t*>(A), lda, reinterpret_cast<const uint16_t*>(B), ldb, b_rows, M, N, K, tiles_m,
        tiles_n, tile0, k_parts, items, epi, phase, b_map);
}

// Sums the k_parts partial tiles of each of the n_tiles tiles from tile0 on, in part order, into
// C (overwrite or accumulate). One workgroup per sum_rows<Cfg>() rows of a tile, a 16-byte vector per thread; N and ldc
// multiples of 4.
// With Cb != NULL the sums go out as bf16 instead: row m times row_scale[m] (if not NULL) to row
// row_map[m] (if not NULL) of Cb.
template <class Cfg> constexpr int sum_rows() { return 256 / (Cfg::BN / 4); }
template <class Cfg>
__global__ __launch_bounds__(256) void sum_partial_tiles_kernel(const float* __restrict__ partial, int tile0,
                                                                int k_parts, int tiles_m, int tiles_n, float* C,
                                                                int64_t ldc, int M, int N, int accumulate,
                                                                uint16_t* Cb, const int32_t* __restrict__ row_map,
                                                                const float* __restrict__ row_scale) {
    typedef float f32x4v __attribute__((ext_vector_type(4)));
    constexpr int VPR = Cfg::BN / 4;
    int tm, tn;
    tile_coords<Cfg::GROUP_M>(tile0 + blockIdx.x, tiles_m, tiles_n, tm, tn);
    const float* src = partial + (size_t)blockIdx.x * k_parts * (Cfg::BM * Cfg::BN);
    static_assert(sum_rows<Cfg>() * VPR == 256 && Cfg::BM % sum_rows<Cfg>() == 0, "one vector per thread");
    const int r = blockIdx.y * sum_rows<Cfg>() + threadIdx.x / VPR, cv = threadIdx.x % VPR;
    const int row = tm * Cfg::BM + r, col = tn * Cfg::BN + cv * 4;
    if (row >= M || col >= N) return;
    f32x4v v = *reinterpret_cast<const f32x4v*>(src + (size_t)r * Cfg::BN + cv * 4);
#pragma unroll 8
    for (int p = 1; p < k_parts; ++p)
        v += *reinterpret_cast<const f32x4v*>(src + (size_t)p * (Cfg::BM * Cfg::BN) + (size_t)r * Cfg::BN + cv * 4);
    if (Cb) {
        const float rs = row_scale ? row_scale[row] : 1.0f;
        const int64_t orow = row_map ? (int64_t)row_map[row] : (int64_t)row;
        const __bf16 b0 = (__bf16)(v[0] * rs), b1 = (__bf16)(v[1] * rs), b2 = (__bf16)(v[2] * rs), b3 = (__bf16)(v[3] * rs);
        const uint32_t lo = (uint32_t)__builtin_bit_cast(uint16_t, b0) | ((uint32_t)__builtin_bit_cast(uint16_t, b1) << 16);
        const uint32_t hi = (uint32_t)__builtin_bit_cast(uint16_t, b2) | ((uint32_t)__builtin_bit_cast(uint16_t, b3) << 16);
        *reinterpret_cast<uint2*>(Cb + (size_t)orow * ldc + col) = make_uint2(lo, hi);
        return;
    }
    f32x4v* dst = reinterpret_cast<f32x4v*>(C + (size_t)row * ldc + col);
    if (accumulate) v += *dst;
    *dst = v;
}

template <class Cfg, class Epi, int AM = A_ROWS, int MAP = WG_ROUNDS, int BL = B_ROWS>
hipError_t allow_lds() {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&gemm_nt_kernel<Cfg, Epi, AM, MAP, BL>),
                               hipFuncAttributeMaxDynamicSharedMemorySize, lds_request<Cfg, Epi>());
}


// dW[V, D] of a chunk by epilogue Epi (EpiStore<0>: float32, EpiStore<2>: bfloat16, overwritten): G is read k-major from its blocks.
// The tiles of a sparsely filled last round are cut along K where `partial` is scratch for the partial tiles
// (mfma_dw_partial_bytes), which a second kernel adds up. resident: at most one workgroup per compute unit, which walks the
// tiles.
template <class Epi>
void launch_dw_tiles(int cus, const void* G, int32_t Vp, const void* HcT, int32_t n_cp, int32_t V, int32_t D, const Epi& e, float* partial,
                     bool resident, hipStream_t st) {
    const int tiles_m = (int)ceil_div(V, CfgGrad::BM), tiles_n = (int)ceil_div(D, CfgGrad::BN);
    const int tiles = tiles_m * tiles_n, tail = cus > 0 ? tiles % cus : 0;
    const int parts = partial ? mfma_tail_parts(cus, tail, n_cp / CfgGrad::BK) : 1;
    const int workgroups = resident ? cus : 0;
    const int whole = parts == 1 ? tiles : tiles - tail;
    launch<CfgGrad, A_BLK_KM, WG_RANGES, B_BLK>(G, Vp, HcT, 0, V, D, n_cp, e, st, 0, whole, 1, PHASE_DW, 0, workgroups);
    if (parts == 1) return;
    Epi ep = e;
    ep.partial = partial;
    launch<CfgGrad, A_BLK_KM, WG_RANGES, B_BLK>(G, Vp, HcT, 0, V, D, n_cp, ep, st, whole, tail, parts);
    sum_partial_tiles_kernel<CfgGrad><<<dim3(tail, CfgGrad::BM / sum_rows<CfgGrad>()), 256, 0, st>>>(
        partial, whole, parts, tiles_m, tiles_n, e.Cf, e.ldc, V, D, e.accumulate, e.Cb, nullptr, nullptr);
}

// Per-device state: the dynamic-LDS attributes of a translation unit's GEMM kernels (`allow` sets them on the current device) and
// the number of compute units, looked up once for each device that a call runs on. Returns a dppo status.
class DeviceSetup {
    static constexpr int MAX_DEVICES = 64;
    std::mutex mu_;
    bool done_[MAX_DEVICES] = {};
    int cus_[MAX_DEVICES] = {};

public:
    int run(hipError_t (*allow)(), int* compute_units) {
        int dev = 0;
        hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) return fail(DPPO_ERR_DEVICE, "hipGetDevice: %s", hipGetErrorString(e));
        if (dev < 0 || dev >= MAX_DEVICES) return fail(DPPO_ERR_UNSUPPORTED, "device index %d", dev);
        std::lock_guard<std::mutex> lk(mu_);
        if (!done_[dev]) {       // (a failed setup is tried again by the next call)
            e = hipDeviceGetAttribute(&cus_[dev], hipDeviceAttributeMultiprocessorCount, dev);
            if (e == hipSuccess) e = allow();
            if (e != hipSuccess) return fail(DPPO_ERR_DEVICE, "device %d setup (dynamic LDS): %s", dev, hipGetErrorString(e));
            done_[dev] = true;
        }
        if (compute_units) *compute_units = cus_[dev];
        return DPPO_OK;
    }
};

}  // namespace
}  // namespace dppo
