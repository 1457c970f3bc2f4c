// Logits of up to 16 tokens: reading W once is all that counts.
//
// Resident workgroups walk contiguous shares of the vocabulary in units of 32 rows (two MFMA blocks by the 16 token
// columns). The wavefronts of one cut K between them, so that the tokens' operands of a wavefront's share stay in its registers from
// beginning to end, and the only loads are those of W: straight into operand registers, each reloaded for the next unit as
// soon as it has been multiplied, 4 L loads of 1 KB in flight per wavefront without a pause at the units' ends. The partial
// blocks of a unit meet in LDS (one barrier a unit, two buffers); the wavefronts take turns in adding them up and with the epilogue,
// which loads nothing from memory: it would wait for the loads of W ahead of it.
#pragma once
#include "stats_epilogues.h"

namespace dppo {
namespace mfma {

constexpr int FEW_TOKENS = FEW_TILE_TOKENS, FEW_UNIT = FEW_TILE_ROWS;
static_assert(FEW_TOKENS == MB && FEW_UNIT == 2 * MB, "a unit is two MFMA blocks");

struct FewToken { float h; int32_t target; };

// Waits for this wavefront's LDS accesses, not for its loads of W, and joins the barrier.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <class Epi, int WAVES, int L>
__global__ __launch_bounds__(WAVES * 64, 4) void few_tokens_kernel(const char* __restrict__ W, int V, const char* __restrict__ H, int64_t h_rows,
                                                                    const int32_t* __restrict__ map, int n, int row_bytes, int units, int longer,
                                                                    Epi epi) {
    typedef typename OperandsOf<Epi>::type Operands;
    typedef typename Operands::acc_t acc_t;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    acc_t* parts = reinterpret_cast<acc_t*>(smem);                            // [2][WAVES][2][64]
    // per token: scale (8-bit operands) and target; then the scales of the workgroup's rows (8-bit operands)
    FewToken* tokens = reinterpret_cast<FewToken*>(smem + 2 * WAVES * 2 * 64 * sizeof(acc_t));
    float* scales = reinterpret_cast<float*>(tokens + FEW_TOKENS);
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    // the first `longer` workgroups have a unit more than the others
    const int u0 = blockIdx.x * units + ((int)blockIdx.x < longer ? (int)blockIdx.x : longer), u1 = u0 + units + ((int)blockIdx.x < longer ? 1 : 0);
    // K in steps of 64 bytes, whole lines per wavefront: L or L - 1 of them
    constexpr int S = 2 * L;
    const int lines = row_bytes / 128, l0 = lines * wave / WAVES, s0 = 2 * l0;
    const bool last = lines * (wave + 1) / WAVES - l0 == L;

    int64_t row = r < n ? r : n - 1;
    if (map) row = map[row];
    row = row < 0 ? 0 : row < h_rows ? row : h_rows - 1;
    if ((int)threadIdx.x < n) tokens[r] = epi.token(r, row);
    if constexpr (std::is_same<Operands, Int8Operands>::value) {
        for (int i = threadIdx.x; i < (u1 - u0) * FEW_UNIT; i += WAVES * 64) {
            const int v = u0 * FEW_UNIT + i;
            scales[i] = epi.s.w[v < V ? v : V - 1];
        }
    }
    __syncthreads();
    u32x4 y[S];
    {
        const u32x4* h = reinterpret_cast<const u32x4*>(H + (size_t)row * row_bytes) + s0 * 4 + q;
#pragma unroll
        for (int s = 0; s < S; ++s)
            if (s < S - 2 || last) y[s] = h[s * 4];
    }

    u32x4 x[2][S];
    // step s of block i of unit u; the last unit's rows beyond V read the last row
    const char* w0 = W + (size_t)s0 * 64;
    auto row_offset = [&](int u, int i) __attribute__((always_inline)) {
        const int left = V - 1 - u * FEW_UNIT, in = i * MB + r;
        return (uint32_t)(in < left ? in : left) * (uint32_t)row_bytes + 16u * q;
    };
    auto load = [&](int i, int s, const char* base, uint32_t offset) __attribute__((always_inline)) {
        x[i][s] = *reinterpret_cast<const u32x4*>(base + s * 64 + offset);
    };
    if (u0 < u1) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t offset = row_offset(u0, i);
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (s < S - 2 || last) load(i, s, w0 + (size_t)u0 * FEW_UNIT * row_bytes, offset);
        }
    }
    for (int u = u0; u < u1; ++u) {
        // (behind the last unit its own rows once more: the loop has no branch around its loads)
        const int next = u + 1 < u1 ? u + 1 : u;
        const char* base = w0 + (size_t)next * FEW_UNIT * row_bytes;
        acc_t* out = parts + (((u & 1) * WAVES + wave) * 2) * 64 + lane;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            acc_t acc;
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = 0;
            const uint32_t offset = row_offset(next, i);
            auto step = [&](int s) __attribute__((always_inline)) {
                acc = Operands::mfma(__builtin_bit_cast(bf16x8, x[i][s]), __builtin_bit_cast(bf16x8, y[s]), acc);
                __builtin_amdgcn_sched_barrier(0);
                load(i, s, base, offset);
                __builtin_amdgcn_sched_barrier(0);
            };
#pragma unroll
            for (int s = 0; s < S - 2; ++s) step(s);
            if (last) {
                step(S - 2);
                step(S - 1);
            }
            out[i * 64] = acc;
        }
        lds_barrier();
        if (wave != (u & (WAVES - 1))) continue;
        // lane: token r, rows 4 q .. + 3 of each block. (What follows from the lane's number is formed here, not kept over the loop: the
        // registers are full of loads under way.)
        int at = lane;
        asm volatile("" : "+v"(at));
        const acc_t* in = parts + ((u & 1) * WAVES * 2) * 64 + at;
        constexpr int AT_ONCE = S > 6 ? 1 : WAVES == 8 ? 7 : 5;
        static_assert((WAVES - 1) % AT_ONCE == 0, "parts of a sum");
        typename Epi::State state;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            acc_t sum = in[i * 64];
#pragma unroll 1
            for (int w = 1; w < WAVES; w += AT_ONCE) {
                acc_t p[AT_ONCE];
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) p[k] = in[((w + k) * 2 + i) * 64];
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) sum += p[k];
            }
            const int v = i * MB + 4 * (at >> 4);
            epi.block(state, sum, u * FEW_UNIT + v, at & 15, V, n, tokens, scales + (u - u0) * FEW_UNIT + v);
        }
        epi.finish(state, u, n, at);
    }
}

// What the epilogues share: a lane's four logits of a block, scaled where the operands are 8-bit.
template <bool I8>
struct FewScales : OperandTag<I8> {
    OperandScales s;
    template <class Acc>
    __device__ __forceinline__ f32x4 logits(const Acc& acc, float h, const float* scales) const {
        if constexpr (I8) {
            f32x4 z;
#pragma unroll
            for (int j = 0; j < 4; ++j) z[j] = (float)acc[j] * scales[j] * h;
            return z;
        } else {
            return acc;
        }
    }
};

template <bool I8, class Out>
struct FewOut : FewScales<I8> {
    struct State {};
    Out* C; int64_t ldc;
    __device__ __forceinline__ FewToken token(int, int64_t row) const { return FewToken{I8 ? this->s.h[row] : 1.0f, -1}; }
    template <class Acc>
    __device__ __forceinline__ void block(State&, const Acc& acc, int v, int t, int V, int n, const FewToken* tok, const float* scales) const {
        if (t < n) store_logits(C + (size_t)t * ldc + v, this->logits(acc, tok[t].h, scales), V - v);
    }
    __device__ __forceinline__ void finish(const State&, int, int, int) const {}
};

// As EpiStats; a unit is a tile of one group.
template <bool I8>
struct FewStats : FewScales<I8> {
    struct State { Stats s = no_stats(); };        // of the lane's rows
    StatsPart part;
    TokenArgs tokens; int64_t n0;
    float* Z; int64_t ldz;         // Z NULL: the logits are not stored
    __device__ __forceinline__ FewToken token(int t, int64_t row) const {
        FewToken f{I8 ? this->s.h[row] : 1.0f, -1};
        int64_t at;
        if (part.zy) locate_token(tokens.ids, tokens.loss_pos, tokens.T, tokens.V, n0 + t, at, f.target);
        return f;
    }
    template <class Acc>
    __device__ __forceinline__ void block(State& state, const Acc& acc, int v, int t, int V, int n, const FewToken* tok, const float* scales) const {
        const float NEG_INF = -__builtin_inff();
        if (t >= n) return;
        const FewToken f = tok[t];
        f32x4 z = this->logits(acc, f.h, scales);
        if (Z) *reinterpret_cast<f32x4*>(Z + (size_t)t * ldz + v) = z;
        const int hit = f.target - v;
        float m = NEG_INF, zy = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            zy = hit == j ? z[j] : zy;
            if (v + j >= V) z[j] = NEG_INF;
            m = fmaxf(m, z[j]);
        }
        if (hit >= 0 && hit < 4) part.zy[t] = zy;
        const float ref = m == NEG_INF ? 0.0f : m;
        Stats b{m, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float d = z[j] - ref, e = exp_fast(d);
            b.sum += e;
            b.dev = fmaf(fmaxf(d, DEV_MIN), e, b.dev);
        }
        state.s = join(state.s, b);
    }
    __device__ __forceinline__ void finish(const State& state, int u, int n, int lane) const {
        // a token's rows are in four lanes
        const Stats s = join_lanes<MB>(state.s);
        if (lane < n) {                          // (lanes 0 to 15 hold the tokens)
            part.mx[part.at(u, lane)] = s.m;
            part.sd[part.at(u, lane)] = make_float2(s.sum, s.dev);
        }
    }
};

}  // namespace mfma

namespace {
// Wavefronts of a workgroup, and how many lines of a row each takes (f(WAVES, L)): rows of up to FEW_SHORT_ROW bytes by two workgroups of 8
// per compute unit, longer ones by one of 16. V = 151936, one token, two of 8 / one of 16: int8 D = 1024 32.2 / 38.6 us, 2048 58.6 / 57.3,
// 2560 74.0 / 70.7, 4096 119 / 113; bfloat16 D = 1024 67 / 80, 2048 136 / 121.
constexpr int FEW_SHORT_ROW = 2048;
template <bool I8, class F>
void for_few_lines(int row_bytes, F&& f) {
    const std::integral_constant<int, 8> w8;
    const std::integral_constant<int, 16> w16;
    const int lines = row_bytes / 128;
    if (lines <= 8) f(w8, std::integral_constant<int, 1>{});
    else if (row_bytes <= FEW_SHORT_ROW) f(w8, std::integral_constant<int, 2>{});
    else if (lines <= 32) f(w16, std::integral_constant<int, 2>{});
    else if (I8 || lines <= 48) f(w16, std::integral_constant<int, 3>{});
    else if constexpr (!I8) f(w16, std::integral_constant<int, 4>{});
}
static_assert(FEW_SHORT_ROW == 8 * 128 * 2 && FEW_ROW_BYTES_I8 == 16 * 128 * 3 && FEW_ROW_BYTES_BF16 == 16 * 128 * 4, "instances");
constexpr int few_lds_bytes(int waves, bool i8, int most_units) { return 2 * waves * 2 * 64 * 16 + FEW_TOKENS * (int)sizeof(FewToken) + (i8 ? most_units * FEW_UNIT * 4 : 0); }
// 8-bit operands: the scales of a workgroup's share lie in LDS, 16 KB of them; a larger share is cut.
constexpr int FEW_MOST_UNITS = 128;
template <bool I8, class Epi>
void launch_few(const LogitsOut& g, const Epi& e, int cus, hipStream_t st) {
    const int units = (int)ceil_div(g.V, FEW_UNIT);
    for_few_lines<I8>(2 * g.k2, [&](auto waves, auto l) {
        constexpr int WAVES = decltype(waves)::value;
        int grid = cus * (16 / WAVES);
        if (grid > units) grid = units;
        if (ceil_div(units, grid) > FEW_MOST_UNITS) grid = (int)ceil_div(units, FEW_MOST_UNITS);
        const int most = (int)ceil_div(units, grid);
        few_tokens_kernel<Epi, WAVES, decltype(l)::value><<<grid, WAVES * 64, few_lds_bytes(WAVES, I8, most), st>>>(
            reinterpret_cast<const char*>(g.W), g.V, reinterpret_cast<const char*>(g.H), g.h_rows, g.map, g.n, 2 * g.k2, units / grid, units % grid, e);
    });
}
template <bool I8, class Epi>
hipError_t allow_few() {
    hipError_t e = hipSuccess;
    for (int row_bytes = 1024; row_bytes <= (I8 ? FEW_ROW_BYTES_I8 : FEW_ROW_BYTES_BF16); row_bytes += 1024)
        for_few_lines<I8>(row_bytes, [&](auto waves, auto l) {
            constexpr int WAVES = decltype(waves)::value;
            if (e == hipSuccess)
                e = hipFuncSetAttribute(reinterpret_cast<const void*>(&few_tokens_kernel<Epi, WAVES, decltype(l)::value>),
                                        hipFuncAttributeMaxDynamicSharedMemorySize, few_lds_bytes(WAVES, I8, FEW_MOST_UNITS));
        });
    return e;
}
template <bool I8>
void launch_stats_tiles(const LogitsOut& g, const OperandScales& s, const StatsTiles& t, int cus, hipStream_t st) {
    if (g.tile == TILE_FEW) {
        FewStats<I8> e;
        e.s = s; e.part = t.part; e.tokens = t.tokens; e.n0 = t.cv.n0;
        e.Z = reinterpret_cast<float*>(g.C); e.ldz = g.ldc;
        launch_few<I8>(g, e, cus, st);
        return;
    }
    auto go = [&](auto e) {
        e.part = t.part; e.scales = s; e.tokens = t.tokens; e.y = t.y; e.n0 = t.cv.n0; e.n_c = t.cv.n_c;
        e.Z = reinterpret_cast<float*>(g.C); e.ldz = g.ldc; e.tau = t.tau;
        launch_logits(g, e, st, t.first, t.count);
    };
    if (g.C) go(EpiStats<I8, true>{});
    else go(EpiStats<I8, false>{});
}
template <bool I8, class Out>
void launch_logits_out(const LogitsOut& g, const OperandScales& s, int cus, hipStream_t st) {
    auto fill = [&](auto& e) {
        e.C = reinterpret_cast<Out*>(g.C);
        e.ldc = g.ldc;
    };
    if (g.tile == TILE_FEW) {
        FewOut<I8, Out> e;
        fill(e);
        e.s = s;
        launch_few<I8>(g, e, cus, st);
        return;
    }
    EpiOut<I8, Out> e;
    fill(e);
    e.scales = s;
    launch_logits(g, e, st);
}
}  // namespace
}  // namespace dppo
