// Epilogues of the vocabulary GEMM (rows = vocabulary entries, columns = tokens) for the token statistics, their gradient and the
// 8-bit product.
#pragma once
#include "gemm_mfma_launch.h"
#include "stats_internal.h"

namespace dppo {
namespace mfma {

template <bool I8> struct OperandTag {};
template <> struct OperandTag<true> { typedef void Int8; };

// Scales of a wavefront's logits (8-bit operands): of its rows' blocks and of its columns.
template <class Cfg> struct TileScales { f32x4 w[Cfg::MI]; float h[Cfg::NI]; };
template <class Cfg>
__device__ __forceinline__ TileScales<Cfg> load_scales(const TileCtx& c, const OperandScales& s) {
    TileScales<Cfg> t;
    struct __attribute__((packed, aligned(4))) Four { f32x4 x; };
#pragma unroll
    for (int ni = 0; ni < Cfg::NI; ++ni) {
        const int n = c.n0 + ni * MB + acc_col(c.lane);
        int row = n < c.N ? n : c.N - 1;
        if (s.map) row = s.map[row];
        t.h[ni] = s.h[row < 0 ? 0 : row < s.rows ? row : s.rows - 1];
    }
    if (c.bm0 + Cfg::BM <= c.M) {
#pragma unroll
        for (int mi = 0; mi < Cfg::MI; ++mi) t.w[mi] = reinterpret_cast<const Four*>(s.w + c.m0 + mi * MB + acc_row(c.lane, 0))->x;
    } else {
#pragma unroll
        for (int mi = 0; mi < Cfg::MI; ++mi)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int v = c.m0 + mi * MB + acc_row(c.lane, j);
                t.w[mi][j] = s.w[v < c.M ? v : c.M - 1];
            }
    }
    return t;
}
// The wavefront's accumulators as logits: as they are (bfloat16 operands), or sum * w[v] * h[row] with both scales applied in 32
// bits, in this order (8-bit operands; the sum itself is exact and is rounded once, to 32 bits).
template <class Cfg, class Acc>
__device__ __forceinline__ void to_logits(Acc (&acc)[Cfg::MI][Cfg::NI], f32x4 (&z)[Cfg::MI][Cfg::NI], const TileScales<Cfg>& s) {
#pragma unroll
    for (int mi = 0; mi < Cfg::MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < Cfg::NI; ++ni) {
            if constexpr (std::is_same<Acc, f32x4>::value) {
                z[mi][ni] = acc[mi][ni];
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) z[mi][ni][j] = (float)acc[mi][ni][j] * s.w[mi][j] * s.h[ni];
            }
        }
}

// 16 bytes of results at any element's address (rows of any length follow each other).
template <class Out> struct __attribute__((packed, aligned(sizeof(Out)))) Packed16 { Out x[16 / sizeof(Out)]; };

__device__ __forceinline__ float as_out(float v, float) { return v; }
__device__ __forceinline__ uint16_t as_out(float v, uint16_t) {
    const __bf16 b = (__bf16)v;
    return __builtin_bit_cast(uint16_t, b);
}

// Four neighbouring logits of a token: one store, or the first `left` of them one by one.
template <class Out>
__device__ __forceinline__ void store_logits(Out* dst, const f32x4& v, int left) {
    struct __attribute__((packed, aligned(sizeof(Out)))) Four { Out x[4]; };
    if (left >= 4) {
        *reinterpret_cast<Four*>(dst) = Four{{as_out(v[0], Out()), as_out(v[1], Out()), as_out(v[2], Out()), as_out(v[3], Out())}};
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < left) dst[j] = as_out(v[j], Out());
}

// Stores the logits, row-major by token: C[n, v]. The tile goes through LDS as [token][vocabulary row], in as many parts as fit, and leaves
// it in runs of whole tile rows, 16 bytes a lane: straight from the accumulators (32 or 64 bytes a token and instruction) 2047
// tokens of D = 4096, V = 32000 in bfloat16 took 284 us instead of 235 (536 G products: 2.28 P/s).
template <bool I8, class Out>
struct EpiOut : OperandTag<I8> {
    Out* C; int64_t ldc;
    OperandScales scales;

    template <class Cfg> static constexpr int pitch() { return Cfg::BM * (int)sizeof(Out) + 16; }
    template <class Cfg> static constexpr int parts() { return Cfg::BN * pitch<Cfg>() <= 160 * 1024 ? 1 : 2; }
    __device__ __forceinline__ void look_up(int, int) const {}
    template <class Cfg, class Acc>
    __device__ __forceinline__ void run(Acc (&acc)[Cfg::MI][Cfg::NI], const TileCtx& c) const {
        constexpr int PITCH = pitch<Cfg>(), PARTS = parts<Cfg>(), WPP = Cfg::WGN / PARTS, TOKS = Cfg::BN / PARTS;
        constexpr int PER = 16 / (int)sizeof(Out), CH = Cfg::BM / PER, RPP = Cfg::NT / CH;      // elements of a chunk, chunks of a row, rows of a pass
        static_assert(Cfg::WGN % PARTS == 0 && TOKS % RPP == 0, "whole wavefronts, whole passes");
        f32x4 z[Cfg::MI][Cfg::NI];
        TileScales<Cfg> ts;
        if constexpr (I8) ts = load_scales<Cfg>(c, scales);
        to_logits<Cfg>(acc, z, ts);
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
            if (part > 0) __syncthreads();
            if (c.wave_n / WPP == part) {
#pragma unroll
                for (int ni = 0; ni < Cfg::NI; ++ni) {
                    char* row = c.smem + ((c.wave_n % WPP) * Cfg::WTN + ni * MB + acc_col(c.lane)) * PITCH;
#pragma unroll
                    for (int mi = 0; mi < Cfg::MI; ++mi) {
                        const f32x4 v = z[mi][ni];
                        Out* dst = reinterpret_cast<Out*>(row) + c.wave_m * Cfg::WTM + mi * MB + acc_row(c.lane, 0);
                        if constexpr (sizeof(Out) == 4) *reinterpret_cast<f32x4*>(dst) = v;
                        else *reinterpret_cast<uint2*>(dst) = make_uint2(as_out(v[0], Out()) | (uint32_t)as_out(v[1], Out()) << 16,
                                                                        as_out(v[2], Out()) | (uint32_t)as_out(v[3], Out()) << 16);
                    }
                }
            }
            __syncthreads();
            const int ch = c.tid % CH, v0 = c.bm0 + ch * PER;
#pragma unroll
            for (int p = 0; p < TOKS / RPP; ++p) {
                const int t = p * RPP + c.tid / CH, n = c.bn0 + part * TOKS + t;
                if (n >= c.N || v0 >= c.M) continue;
                const Out* src = reinterpret_cast<const Out*>(c.smem + t * PITCH) + ch * PER;
                Out* dst = C + (size_t)n * ldc + v0;
                if (v0 + PER <= c.M) {
                    *reinterpret_cast<Packed16<Out>*>(dst) = *reinterpret_cast<const Packed16<Out>*>(src);
                } else {
                    for (int k = 0; v0 + k < c.M; ++k) dst[k] = src[k];
                }
            }
        }
    }

    template <class Cfg>
    static constexpr int lds_bytes() { return Cfg::BN / parts<Cfg>() * pitch<Cfg>(); }
    static constexpr bool SWAP = false;
};

// Softmax statistics of every token over a wavefront's vocabulary rows (a group, see Stats and StatsPart), in registers; the target's logit
// from the accumulator that holds it; with STORE the logits that may be among the top alternatives, row-major by token. A group is
// stored for the tokens whose bound tau its maximum exceeds: top_k groups of lower vocabulary entries reach tau, so nothing else can be
// among the alternatives (an equal logit loses to theirs).
// (Nothing goes through LDS, so a resident workgroup could load its next tile's first slices meanwhile; it was slower: 8191 tokens of
// D = 2560, V = 151936 4.68 against 4.55 ms, as the 256 registers do not hold both and the tiles that share panels drift apart.)
template <bool I8, bool STORE>
struct EpiStats : OperandTag<I8> {
    StatsPart part;
    OperandScales scales;
    // y[n]: targets looked up before, or NULL: from tokens.ids
    TokenArgs tokens; const int32_t* y; int64_t n0; int n_c;
    float* Z; int64_t ldz; const float* tau;

    template <class Cfg> struct Pre { int at[Cfg::NI]; float tau[Cfg::NI]; TileScales<Cfg> scales; };
    // What the epilogue needs from memory, all loads at once: targets relative to the wavefront's rows, bounds, scales.
    template <class Cfg>
    __device__ __forceinline__ Pre<Cfg> preload(const TileCtx& c) const {
        Pre<Cfg> p;
#pragma unroll
        for (int ni = 0; ni < Cfg::NI; ++ni) {
            const int n = c.n0 + ni * MB + acc_col(c.lane);
            p.at[ni] = -1;
            p.tau[ni] = -__builtin_inff();
            if (n < n_c) {
                if (part.zy) {
                    int32_t t;
                    if (y) {
                        t = y[n];
                    } else {
                        int64_t row;
                        locate_token(tokens.ids, tokens.loss_pos, tokens.T, tokens.V, n0 + n, row, t);
                    }
                    p.at[ni] = t - c.m0;
                }
                if (STORE && tau) p.tau[ni] = tau[n];
            }
        }
        if constexpr (I8) p.scales = load_scales<Cfg>(c, scales);
        return p;
    }
    __device__ __forceinline__ void look_up(int, int) const {}
    template <class Cfg, class Acc>
    __device__ __forceinline__ void run(Acc (&acc)[Cfg::MI][Cfg::NI], const TileCtx& c) const {
        const Pre<Cfg> pre = preload<Cfg>(c);
        constexpr int MI = Cfg::MI, NI = Cfg::NI;
        const float NEG_INF = -__builtin_inff();
        f32x4 z[MI][NI];
        to_logits<Cfg>(acc, z, pre.scales);
        static_assert(Cfg::WGM == STATS_GROUPS, "a wavefront's rows = a group");
        const int g = c.tm * STATS_GROUPS + c.wave_m;
        auto reduce = [&](auto full_tag) __attribute__((always_inline)) {
            constexpr bool FULL = decltype(full_tag)::value;
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) {
                float m = NEG_INF;
#pragma unroll
                for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (!FULL && c.m0 + mi * MB + acc_row(c.lane, j) >= c.M) z[mi][ni][j] = NEG_INF;
                        m = fmaxf(m, z[mi][ni][j]);
                    }
                m = pair_max<32>(pair_max<16>(m));
                const int n = c.n0 + ni * MB + acc_col(c.lane);
                if (STORE) {
                    // whole groups, the padding of the vocabulary too (the pitch holds it)
                    const bool store = n < n_c && (!tau || m > pre.tau[ni]);
                    if (store) {
                        float* dst = Z + (size_t)n * ldz + c.m0 + acc_row(c.lane, 0);
#pragma unroll
                        for (int mi = 0; mi < MI; ++mi) *reinterpret_cast<f32x4*>(dst + mi * MB) = z[mi][ni];
                    }
                }
                const float ref = m == NEG_INF ? 0.0f : m;
                float sum = 0.0f, dev = 0.0f;
#pragma unroll
                for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float d = z[mi][ni][j] - ref, e = exp_fast(d);
                        sum += e;
                        dev = fmaf(fmaxf(d, DEV_MIN), e, dev);
                    }
                sum = pair_sum<32>(pair_sum<16>(sum));
                dev = pair_sum<32>(pair_sum<16>(dev));
                if (c.lane < MB && n < n_c) {
                    part.mx[part.at(g, n)] = m;
                    part.sd[part.at(g, n)] = make_float2(sum, dev);
                }
            }
        };
        if (c.bm0 + Cfg::BM <= c.M) reduce(std::true_type{});
        else reduce(std::false_type{});
        if (part.zy) {
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) {
                if (!__any(pre.at[ni] >= 0 && pre.at[ni] < Cfg::WTM)) continue;
#pragma unroll
                for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (pre.at[ni] == mi * MB + acc_row(c.lane, j)) part.zy[c.n0 + ni * MB + acc_col(c.lane)] = z[mi][ni][j];
            }
        }
    }

    template <class Cfg>
    static constexpr int lds_bytes() { return 0; }
    static constexpr bool SWAP = false;
};

// Gradient entries of the statistics straight from the logits (see grad_entry), staged through LDS as [token][vocabulary row] and
// stored to the blocked chunk. The logits are summed over K as the forward pass's tiles sum them; up to 16 tokens that pass cuts K between
// wavefronts (few_tokens.h), so that its lse differs from these logits by the roundings of such sums.
// An entry is formed in 32 bits and rounded once to bfloat16: it is an operand of the matrix instructions that form dH and dW (with float32 sums), as
// in the policy loss. 4111 tokens of D = 2560, V = 151936, norm of the error: 1.7e-3 of a float32 dW's; of results in bfloat16 2.35e-3, of which
// their own rounding is 1.66e-3. Entries in two halves would take both products, two thirds of the time, twice.
struct EpiStatsGrad {
    const int32_t* y; StatsGrad grad; int64_t n0; int n_c;
    uint16_t* G; int64_t ldg; int V;

    template <class Cfg>
    __device__ __forceinline__ void run(f32x4 (&acc)[Cfg::MI][Cfg::NI], const TileCtx& c) const {
        constexpr int ZPITCH = StagedStore<Cfg>::ZPITCH;
        // all columns' loads at once (beyond the last token its own)
        TokenGrad tokens[Cfg::NI];
        int targets[Cfg::NI];                                       // among the wavefront's rows
#pragma unroll
        for (int ni = 0; ni < Cfg::NI; ++ni) {
            const int n = c.n0 + ni * MB + acc_col(c.lane), in = n < n_c ? n : n_c - 1;
            tokens[ni] = load_grad(grad, n0 + in);
            targets[ni] = n < n_c ? y[in] - c.m0 : -1;
        }
        auto body = [&](auto full_tag) __attribute__((always_inline)) {
            constexpr bool FULL = decltype(full_tag)::value;        // neither vocabulary nor tokens end in the tile
#pragma unroll
            for (int ni = 0; ni < Cfg::NI; ++ni) {
                const int tok = c.wave_n * Cfg::WTN + ni * MB + acc_col(c.lane), at = targets[ni];
                const bool token = FULL || c.bn0 + tok < n_c;
                const TokenGrad t = tokens[ni];
#pragma unroll
                for (int mi = 0; mi < Cfg::MI; ++mi) {
                    const int vloc = c.wave_m * Cfg::WTM + mi * MB + acc_row(c.lane, 0);
                    bf16x4 h;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float lp = acc[mi][ni][q] - t.lse;
                        float g = grad_entry(t, lp, exp_fast(lp), false);
                        // (a padding token's row of zeros times a weight of -infinity is NaN, which dW would sum)
                        g = token && (FULL || c.bm0 + vloc + q < V) ? g : 0.0f;
                        const __bf16 b = (__bf16)g;   // scalar copy: reading h[q] back right after writing it miscompiles
                        h[q] = b;
                    }
                    *reinterpret_cast<bf16x4*>(c.smem + tok * ZPITCH + vloc * 2) = h;
                }
                if (!__any(at >= 0 && at < Cfg::WTM)) continue;
#pragma unroll
                for (int mi = 0; mi < Cfg::MI; ++mi)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        if (at != mi * MB + acc_row(c.lane, q)) continue;
                        const float lp = acc[mi][ni][q] - t.lse;
                        const __bf16 b = (__bf16)grad_entry(t, lp, exp_fast(lp), true);
                        *reinterpret_cast<__bf16*>(c.smem + tok * ZPITCH + (c.wave_m * Cfg::WTM + at) * 2) = b;
                    }
            }
        };
        if (c.bm0 + Cfg::BM <= V && c.bn0 + Cfg::BN <= n_c) body(std::true_type{});
        else body(std::false_type{});
        __syncthreads();
        const StagedStore<Cfg> staged(c, G, ldg);
#pragma unroll
        for (int b = 0; b < Cfg::BN / BLK_R; ++b)
#pragma unroll
            for (int p = 0; p < BLK_R / MB; ++p) staged.pass(b, p);
    }

    template <class Cfg>
    static constexpr int lds_bytes() { return Cfg::BN * (Cfg::BM * 2 + 16); }
    static constexpr bool SWAP = false;
};

// Four rows' bfloat16 values of a column (lane), rows 0, 1 and 2, 3 packed in w0 and w1, to four neighbouring columns of row (lane & 3): the
// 4 x 4 values of four lanes transposed. First pairs of lanes: the even one rows 0 and 2, the odd one rows 1 and 3; then pairs of pairs.
__device__ __forceinline__ uint2 transpose4(uint32_t w0, uint32_t w1, int lane) {
    const uint32_t o0 = xor_lane<1>(w0), o1 = xor_lane<1>(w1);
    const bool odd = lane & 1, upper = lane & 2;
    const uint32_t x = odd ? o0 >> 16 | (w0 & 0xffff0000u) : (w0 & 0xffffu) | o0 << 16;
    const uint32_t z = odd ? o1 >> 16 | (w1 & 0xffff0000u) : (w1 & 0xffffu) | o1 << 16;
    const uint32_t px = xor_lane<2>(x), pz = xor_lane<2>(z);
    return upper ? make_uint2(pz, z) : make_uint2(x, px);
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) { return (uint32_t)as_out(a, uint16_t()) | (uint32_t)as_out(b, uint16_t()) << 16; }

// dH by small tiles: bfloat16 rows (all of a lane's entries of row_map at once, 8-byte stores), or, with `partial`, the raw tile as EpiStore's.
struct EpiRows {
    uint16_t* C; int64_t ldc; const int32_t* row_map; float* partial;

    template <class Cfg>
    __device__ __forceinline__ void run(f32x4 (&acc)[Cfg::MI][Cfg::NI], const TileCtx& c) const {
        if (partial) {
            float* dst = partial + (size_t)c.slot * (Cfg::BM * Cfg::BN) + c.wave_n * Cfg::WTN + acc_col(c.lane);
#pragma unroll
            for (int mi = 0; mi < Cfg::MI; ++mi)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int ni = 0; ni < Cfg::NI; ++ni)
                        dst[(size_t)(c.wave_m * Cfg::WTM + mi * MB + acc_row(c.lane, j)) * Cfg::BN + ni * MB] = acc[mi][ni][j];
            return;
        }
        int64_t to[Cfg::MI];
#pragma unroll
        for (int mi = 0; mi < Cfg::MI; ++mi) {
            const int row = c.m0 + mi * MB + acc_row(c.lane, 0) + (c.lane & 3);
            to[mi] = row < c.M ? (row_map ? (int64_t)row_map[row] : (int64_t)row) : -1;
        }
#pragma unroll
        for (int mi = 0; mi < Cfg::MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < Cfg::NI; ++ni) {
                const f32x4 v = acc[mi][ni];
                const uint2 w = transpose4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), c.lane);
                const int col = c.n0 + ni * MB + (c.lane & 12);
                if (to[mi] >= 0 && col < c.N) *reinterpret_cast<uint2*>(C + (size_t)to[mi] * ldc + col) = w;
            }
    }

    template <class Cfg>
    static constexpr int lds_bytes() { return 0; }
    static constexpr bool SWAP = false;
};

// EpiStatsGrad's entries (rounded alike) row-major, straight from the registers: G[n, v] (pitch ldg, zero from V on) and their transpose GT[v, n] (pitch ldt, zero
// from the N-th token on, both), 8 bytes a lane each.
struct EpiStatsGradBoth {
    const int32_t* y; StatsGrad grad; int64_t n0;
    uint16_t* G; int64_t ldg; uint16_t* GT; int64_t ldt;

    __device__ __forceinline__ void look_up(int, int) const {}
    template <class Cfg>
    __device__ __forceinline__ void run(f32x4 (&acc)[Cfg::MI][Cfg::NI], const TileCtx& c) const {
        TokenGrad tokens[Cfg::NI];               // (of all columns at once; beyond the last token its own)
        int targets[Cfg::NI];
#pragma unroll
        for (int ni = 0; ni < Cfg::NI; ++ni) {
            const int n = c.n0 + ni * MB + acc_col(c.lane), in = n < c.N ? n : c.N - 1;
            tokens[ni] = load_grad(grad, n0 + in);
            targets[ni] = y[in];
        }
#pragma unroll
        for (int ni = 0; ni < Cfg::NI; ++ni) {
            const int n = c.n0 + ni * MB + acc_col(c.lane);
            const bool token = n < c.N;
            const TokenGrad t = tokens[ni];
#pragma unroll
            for (int mi = 0; mi < Cfg::MI; ++mi) {
                const int v = c.m0 + mi * MB + acc_row(c.lane, 0);
                uint32_t w[2];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float lp = acc[mi][ni][q] - t.lse, g = grad_entry(t, lp, exp_fast(lp), v + q == targets[ni]);
                    const __bf16 b = (__bf16)(token && v + q < c.M ? g : 0.0f);
                    const uint32_t h = __builtin_bit_cast(uint16_t, b);
                    w[q / 2] = q % 2 ? w[q / 2] | h << 16 : h;
                }
                if (n < ldt && v < ldg) *reinterpret_cast<uint2*>(G + (size_t)n * ldg + v) = make_uint2(w[0], w[1]);
                const uint2 t4 = transpose4(w[0], w[1], c.lane);
                const int row = v + (c.lane & 3), col = c.n0 + ni * MB + (c.lane & 12);
                if (row < c.M && col < ldt) *reinterpret_cast<uint2*>(GT + (size_t)row * ldt + col) = t4;
            }
        }
    }

    template <class Cfg>
    static constexpr int lds_bytes() { return 0; }
    static constexpr bool SWAP = false;
};

}  // namespace mfma

namespace {
typedef PipeCfg<128, 128, 2, 4, 2, 1, 1> Cfg128Eight;       // (see eight_wavefronts)
template <class Epi>
void launch_logits(const LogitsOut& g, const Epi& e, hipStream_t st, int first = 0, int count = -1) {
    auto mapped = [&](auto cfg) {
        launch<decltype(cfg), A_ROWS, WG_ROUNDS, B_MAP>(g.W, g.k2, g.H, g.k2, g.V, g.n, g.k2, e, st, first, count, 1, -1, (int)g.h_rows, 0, g.map, 0);
    };
    if (g.tile == TILE_128x96) mapped(CfgFew<96>{});
    else if (g.tile == TILE_128x128 && eight_wavefronts(g.n, g.V, g.k2)) mapped(Cfg128Eight{});
    else if (g.tile == TILE_128x128) mapped(CfgFew<128>{});
    else if (g.tile == TILE_256x192) mapped(CfgBig192{});
    else launch<CfgBig>(g.W, g.k2, g.H, g.k2, g.V, g.n, g.k2, e, st, first, count, 1, PHASE_LOGITS);
}
template <class Epi>
hipError_t allow_logits() {
    hipError_t e = allow_lds<CfgFew<96>, Epi, A_ROWS, WG_ROUNDS, B_MAP>();
    if (e == hipSuccess) e = allow_lds<CfgFew<128>, Epi, A_ROWS, WG_ROUNDS, B_MAP>();
    if (e == hipSuccess) e = allow_lds<Cfg128Eight, Epi, A_ROWS, WG_ROUNDS, B_MAP>();
    if (e == hipSuccess) e = allow_lds<CfgBig192, Epi, A_ROWS, WG_ROUNDS, B_MAP>();
    if (e == hipSuccess) e = allow_lds<CfgBig, Epi>();
    return e;
}
}  // namespace
}  // namespace dppo
