// Epilogues of the vocabulary GEMM (rows = vocabulary entries, columns = tokens) for the token statistics, their gradient and the
// 8-bit product.
#pragma once
#include "gemm_mfma_launch.h"
#include "stats_internal.h"

namespace dppo {
namespace mfma {

template <bool I8> struct OperandTag {};
template <> struct OperandTag<true> { typedef void Int8; };

// The wavefront's accumulators as logits: as they are (bfloat16 operands), or sum * w[v] * h[row] with both scales applied in 32
// bits, in this order (8-bit operands; the sum itself is exact and is rounded once, to 32 bits).
template <class Cfg, class Acc>
__device__ __forceinline__ void to_logits(Acc (&acc)[Cfg::MI][Cfg::NI], f32x4 (&z)[Cfg::MI][Cfg::NI], const TileCtx& c, const OperandScales& s) {
    if constexpr (std::is_same<Acc, f32x4>::value) {
#pragma unroll
        for (int mi = 0; mi < Cfg::MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < Cfg::NI; ++ni) z[mi][ni] = acc[mi][ni];
    } else {
        float h[Cfg::NI];
#pragma unroll
        for (int ni = 0; ni < Cfg::NI; ++ni) {
            const int n = c.n0 + ni * MB + acc_col(c.lane);
            int row = n < c.N ? n : c.N - 1;
            if (s.map) row = s.map[row];
            h[ni] = s.h[row < 0 ? 0 : row < s.rows ? row : s.rows - 1];
        }
#pragma unroll
        for (int mi = 0; mi < Cfg::MI; ++mi)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int v = c.m0 + mi * MB + acc_row(c.lane, j);
                const float w = s.w[v < c.M ? v : c.M - 1];
#pragma unroll
                for (int ni = 0; ni < Cfg::NI; ++ni) z[mi][ni][j] = (float)acc[mi][ni][j] * w * h[ni];
            }
    }
}

// Four neighbouring logits of a token: one aligned store, or the first `left` of them one by one.
template <class Out>
__device__ __forceinline__ void store_logits(Out* dst, const f32x4& v, bool whole, int left) {
    if constexpr (sizeof(Out) == 4) {
        if (whole) { *reinterpret_cast<f32x4*>(dst) = v; return; }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) dst[j] = v[j];
    } else {
        const __bf16 b0 = (__bf16)v[0], b1 = (__bf16)v[1], b2 = (__bf16)v[2], b3 = (__bf16)v[3];
        const uint16_t h[4] = {__builtin_bit_cast(uint16_t, b0), __builtin_bit_cast(uint16_t, b1), __builtin_bit_cast(uint16_t, b2),
                               __builtin_bit_cast(uint16_t, b3)};
        if (whole) { *reinterpret_cast<uint2*>(dst) = make_uint2(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16); return; }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) dst[j] = h[j];
    }
}

// Stores the logits, row-major by token: C[n, v]. A lane's four accumulators are four neighbouring vocabulary entries of one token,
// one store where the pitch allows it.
template <bool I8, class Out>
struct EpiOut : OperandTag<I8> {
    Out* C; int64_t ldc; int vec;          // vec: whole groups of four are aligned
    OperandScales scales;

    __device__ __forceinline__ void look_up(int, int) const {}
    template <class Cfg, class Acc>
    __device__ __forceinline__ void run(Acc (&acc)[Cfg::MI][Cfg::NI], const TileCtx& c) const {
        f32x4 z[Cfg::MI][Cfg::NI];
        to_logits<Cfg>(acc, z, c, scales);
        auto store = [&](auto full_tag) __attribute__((always_inline)) {
            constexpr bool FULL = decltype(full_tag)::value;
#pragma unroll
            for (int ni = 0; ni < Cfg::NI; ++ni) {
                const int n = c.n0 + ni * MB + acc_col(c.lane);
                if (!FULL && n >= c.N) continue;
                Out* dst = C + (size_t)n * ldc + c.m0 + acc_row(c.lane, 0);
#pragma unroll
                for (int mi = 0; mi < Cfg::MI; ++mi)
                    store_logits(dst + mi * MB, z[mi][ni], FULL, c.M - (c.m0 + mi * MB + acc_row(c.lane, 0)));
            }
        };
        if (vec && c.bm0 + Cfg::BM <= c.M && c.bn0 + Cfg::BN <= c.N) store(std::true_type{});
        else store(std::false_type{});
    }

    template <class Cfg>
    static constexpr int lds_bytes() { return 0; }
    static constexpr bool SWAP = false;
};

// Softmax statistics of every token over the tile's vocabulary rows (see Stats and StatsPart), in registers and combined across the
// wavefronts through LDS; the target's logit from the accumulator that holds it; with STORE the logits that may be among the top
// alternatives, row-major by token. A group (the rows of one wavefront) is stored for the tokens whose bound tau its maximum exceeds:
// top_k groups of lower vocabulary entries reach tau, so nothing else can be among the alternatives (an equal logit loses to theirs).
template <bool I8, bool STORE>
struct EpiStats : OperandTag<I8> {
    StatsPart part;
    OperandScales scales;
    // y[n]: targets looked up before, or NULL: from tokens.ids (NULL: no targets)
    TokenArgs tokens; const int32_t* y; int64_t n0; int n_c;
    float* Z; int64_t ldz; const float* tau;

    __device__ __forceinline__ void look_up(int, int) const {}
    template <class Cfg, class Acc>
    __device__ __forceinline__ void run(Acc (&acc)[Cfg::MI][Cfg::NI], const TileCtx& c) const {
        constexpr int MI = Cfg::MI, NI = Cfg::NI;
        const float NEG_INF = -__builtin_inff();
        f32x4 z[MI][NI];
        to_logits<Cfg>(acc, z, c, scales);
        static_assert(Cfg::WGM == STATS_GROUPS, "a wavefront's rows = a group");
        float* mx_out = part.mx + (size_t)(c.tm * STATS_GROUPS + c.wave_m) * part.pitch;
        float3* red = reinterpret_cast<float3*>(c.smem);
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
                m = fmaxf(m, __shfl_xor(m, 16, 64));
                m = fmaxf(m, __shfl_xor(m, 32, 64));
                const int n = c.n0 + ni * MB + acc_col(c.lane);
                if (n < n_c) {
                    if (c.lane < MB) mx_out[n] = m;
                    // whole groups, the padding of the vocabulary too (the pitch holds it)
                    if (STORE && (!tau || m > tau[n])) {
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
                sum += __shfl_xor(sum, 16, 64);
                sum += __shfl_xor(sum, 32, 64);
                dev += __shfl_xor(dev, 16, 64);
                dev += __shfl_xor(dev, 32, 64);
                if (c.lane < MB) red[c.wave_m * Cfg::BN + c.wave_n * Cfg::WTN + ni * MB + c.lane] = make_float3(m, sum, dev);
            }
        };
        if (c.bm0 + Cfg::BM <= c.M) reduce(std::true_type{});
        else reduce(std::false_type{});
        if (part.zy) {
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) {
                const int n = c.n0 + ni * MB + acc_col(c.lane);
                int at = -1;                                        // target among the wavefront's rows
                if (n < n_c) {
                    int32_t t;
                    if (y) {
                        t = y[n];
                    } else {
                        int64_t row;
                        locate_token(tokens.ids, tokens.loss_pos, tokens.T, tokens.V, n0 + n, row, t);
                    }
                    at = t - c.m0;
                }
                if (!__any(at >= 0 && at < Cfg::WTM)) continue;
#pragma unroll
                for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (at == mi * MB + acc_row(c.lane, j)) part.zy[n] = z[mi][ni][j];
            }
        }
        __syncthreads();
        for (int t = c.tid; t < Cfg::BN; t += Cfg::NT) {
            const int n = c.bn0 + t;
            if (n >= n_c) continue;
            Stats s = no_stats();
#pragma unroll
            for (int w = 0; w < Cfg::WGM; ++w) {
                const float3 r = red[w * Cfg::BN + t];
                s = join(s, Stats{r.x, r.y, r.z});
            }
            const size_t at = (size_t)c.tm * part.pitch + n;
            part.sd[at] = make_float2(s.sum, s.dev);
        }
    }

    template <class Cfg>
    static constexpr int lds_bytes() { return Cfg::WGM * Cfg::BN * 12; }
    static constexpr bool SWAP = false;
};

// Gradient entries of the statistics straight from the logits (see grad_entry), staged through LDS as [token][vocabulary row] and
// stored to the blocked chunk. Everything, the target's entry too, comes from the accumulators that the forward pass summed the
// same way.
struct EpiStatsGrad {
    const int32_t* y; StatsGrad grad; int64_t n0; int n_c;
    uint16_t* G; int64_t ldg; int V;

    template <class Cfg>
    __device__ __forceinline__ void run(f32x4 (&acc)[Cfg::MI][Cfg::NI], const TileCtx& c) const {
        constexpr int ZPITCH = StagedStore<Cfg>::ZPITCH;
        auto body = [&](auto full_tag) __attribute__((always_inline)) {
            constexpr bool FULL = decltype(full_tag)::value;
#pragma unroll
            for (int ni = 0; ni < Cfg::NI; ++ni) {
                const int tok = c.wave_n * Cfg::WTN + ni * MB + acc_col(c.lane);
                const int n = c.bn0 + tok;
                TokenGrad t{0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
                int at = -1;                                        // target among the wavefront's rows
                if (n < n_c) {
                    t = load_grad(grad, n0 + n);
                    at = y[n] - (c.bm0 + c.wave_m * Cfg::WTM);
                }
#pragma unroll
                for (int mi = 0; mi < Cfg::MI; ++mi) {
                    const int vloc = c.wave_m * Cfg::WTM + mi * MB + acc_row(c.lane, 0);
                    bf16x4 h;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float lp = acc[mi][ni][q] - t.lse;
                        float g = grad_entry(t, lp, exp_fast(lp), false);
                        // (a padding token's row of zeros times a weight of -infinity is NaN, which dW would sum)
                        g = n < n_c && (FULL || c.bm0 + vloc + q < V) ? g : 0.0f;
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
        if (c.bm0 + Cfg::BM <= V) body(std::true_type{});
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

}  // namespace mfma

namespace {
// The tile of the vocabulary GEMM by the number of tokens, as for the log-probabilities alone (see CfgFew): up to 192 tokens
// columns that read the tokens' rows of H where they lie, through the map. Beyond, the rows are contiguous.
template <class Epi>
void launch_logits(const LogitsOut& g, const Epi& e, hipStream_t st, int first = 0, int count = -1) {
    auto mapped = [&](auto cfg) {
        launch<decltype(cfg), A_ROWS, WG_ROUNDS, B_MAP>(g.W, g.k2, g.H, g.k2, g.V, g.n, g.k2, e, st, first, count, 1, -1, (int)g.h_rows, 0, g.map, 0);
    };
    if (g.n <= 96) mapped(CfgFew<96>{});
    else if (g.n <= 128) mapped(CfgFew<128>{});
    else if (g.n <= STATS_MAP_TOKENS) mapped(CfgBig192{});
    else launch<CfgBig>(g.W, g.k2, g.H, g.k2, g.V, g.n, g.k2, e, st, first, count);
}
template <class Epi>
hipError_t allow_logits() {
    hipError_t e = allow_lds<CfgFew<96>, Epi, A_ROWS, WG_ROUNDS, B_MAP>();
    if (e == hipSuccess) e = allow_lds<CfgFew<128>, Epi, A_ROWS, WG_ROUNDS, B_MAP>();
    if (e == hipSuccess) e = allow_lds<CfgBig192, Epi, A_ROWS, WG_ROUNDS, B_MAP>();
    if (e == hipSuccess) e = allow_lds<CfgBig, Epi>();
    return e;
}
}  // namespace
}  // namespace dppo
