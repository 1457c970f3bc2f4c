// Internal declarations of the token statistics, their gradient and the 8-bit operators.
#pragma once
#include "dppo_internal.h"
#include "lanes.h"
#include "stats_plan.h"

namespace dppo {

// ---- token statistics (stats_rows.hip) ---------------------------------------
struct StatsOut {
    float* lse; float* entropy; float* logp;     // each may be NULL
    int32_t* top_ids; float* top_logp; int32_t top_k;
};
// Statistics of a set of logits against its maximum m: sum = sum exp(z - m), dev = sum (z - m) exp(z - m). With them
// lse = m + log(sum) and the entropy -sum p log p = log(sum) - dev / sum, in which nothing of the size of the logits cancels.
struct Stats { float m, sum, dev; };
// exp() is 0 in 32 bits below -104: differences are cut at -150 where they are multiplied by it, so that a logit at -infinity (or
// at the type's lowest value, whose difference overflows) adds 0 and not 0 * infinity.
constexpr float DEV_MIN = -150.0f;
// exp by the hardware's 2^x: one rounding of the argument (relative error 2 d half steps at exp(-d), whose share of a sum is e^-d) and
// one unit of its own.
__device__ __forceinline__ float exp_fast(float d) { return __builtin_amdgcn_exp2f(d * 1.4426950408889634f); }
__device__ __forceinline__ Stats no_stats() { return Stats{-__builtin_inff(), 0.0f, 0.0f}; }
__device__ __forceinline__ Stats join(const Stats& a, const Stats& b) {
    const float m = fmaxf(a.m, b.m), ref = m == -__builtin_inff() ? 0.0f : m;
    const float da = a.m - ref, db = b.m - ref, ea = exp_fast(da), eb = exp_fast(db);
    return Stats{m, a.sum * ea + b.sum * eb,
                 ea * (a.dev + fmaxf(da, DEV_MIN) * a.sum) + eb * (b.dev + fmaxf(db, DEV_MIN) * b.sum)};
}
// Over the lanes whose numbers differ in bit FROM and above.
template <int FROM>
__device__ __forceinline__ Stats join_lanes(Stats s) {
    s = join(s, Stats{xor_lane<FROM>(s.m), xor_lane<FROM>(s.sum), xor_lane<FROM>(s.dev)});
    if constexpr (FROM < 32) s = join_lanes<2 * FROM>(s);
    return s;
}
// Rows of logits cut into parts: per (token, part) the statistics {max, sum, dev, -} and the top_k keys.
struct PartialStats {
    float4* stats; uint64_t* keys; int32_t parts;
};
// Parts that the rows of n_c tokens are cut into.
int stats_row_parts(int32_t n_c, int32_t V, int cus);
void launch_stats_rows(const float* Z, int64_t ldz, const TokenArgs& a, const StatsOut& o, ChunkView cv, PartialStats partial, hipStream_t st);

// Statistics of the vocabulary GEMM by groups of rows, STATS_GROUPS of a tile (a unit of the kernel for few tokens is one): mx[at(g, n)]
// is group g's maximum for token n, sd[at(g, n)] = {sum, dev} against it; zy[n]: target logits (or NULL). A token's groups lie side by side
// up to JOIN_ALONE tokens, which a workgroup each joins, beyond that the tokens of a group.
struct StatsPart {
    float* mx; float2* sd; float* zy; int32_t group_step, token_step;
    __device__ __forceinline__ size_t at(int g, int n) const { return (size_t)g * group_step + (size_t)n * token_step; }
};
// Joins a token's groups (of `rows` rows) and picks the top alternatives from the stored logits of the groups that can hold them.
void launch_stats_join(const StatsPart& part, int rows, const float* Z, int64_t ldz, const TokenArgs& a, bool look_up,
                       const StatsOut& o, ChunkView cv, hipStream_t st);
// tau[n] = the top_k-th largest maximum of token n's first `groups` groups (at least top_k).
void launch_stats_bound(const StatsPart& part, int32_t groups, int32_t top_k, ChunkView cv, float* tau, hipStream_t st);

// Copies of the tokens' rows (row_bytes: a multiple of 4; below 16-byte alignment they are taken for float32), their targets (-1 without ids), clamped rows and scales;
// any of the outputs may be NULL.
struct GatherRows {
    TokenArgs tokens; size_t row_bytes; const float* scale;
    void* out; int32_t* y; int32_t* rowc; float* scale_out;
    void* clear; size_t clear_bytes;        // cleared by further workgroups of the launch
    // bfloat16: the rows' transpose [D, transpose_cols] in the blocked B-operand layout, zero from n_c on, by further workgroups too (NULL: none)
    void* transpose; int32_t transpose_cols, transpose_block;      // transpose_block: rows of a block
};
void launch_stats_gather(const GatherRows& g, ChunkView cv, hipStream_t st);

// ---- gradient of the statistics ----------------------------------------------
// Incoming gradients (each may be NULL = 0) and the forward's results, per loss token.
struct StatsGrad {
    const float* g_logp; const float* g_lse; const float* g_entropy;
    const float* lse; const float* entropy;
};
struct TokenGrad { float lse, ent, gl, ge, gs, c; };
__device__ __forceinline__ TokenGrad load_grad(const StatsGrad& g, int64_t n) {
    TokenGrad t;
    t.lse = g.lse[n];
    t.gl = g.g_logp ? g.g_logp[n] : 0.0f;
    t.gs = g.g_lse ? g.g_lse[n] : 0.0f;
    t.ge = g.g_entropy ? g.g_entropy[n] : 0.0f;
    t.ent = g.g_entropy ? g.entropy[n] : 0.0f;
    t.c = t.gs - t.gl - t.ge * t.ent;
    return t;
}
// Gradient entry of a logit of log-probability lp and probability p. lp is cut where p is 0 in 32 bits (0, not 0 * infinity); the
// target's 1 - p is formed as such: p near 1 must cancel against the 1 before anything is added.
__device__ __forceinline__ float grad_entry(const TokenGrad& t, float lp, float p, bool target) {
    const float cut = fmaxf(lp, -150.0f);
    return target ? fmaf(t.gl, 1.0f - p, p * (t.gs - t.ge * (cut + t.ent))) : p * fmaf(-t.ge, cut, t.c);
}
// float32 entries in place over the stored logits, and the gathering beside them (no transpose).
void launch_stats_grad_f32(float* ZG, int32_t Vp, const StatsGrad& g, const GatherRows& rows, ChunkView cv, hipStream_t st);
// dst (bfloat16) = src, n a multiple of 4, both 16-byte aligned.
void launch_to_bf16(const float* src, void* dst, size_t n, hipStream_t st);

// ---- GEMMs (gemm_stats.hip, gemm_i8.hip) --------------------------------------
// Scales of 8-bit operands: logit = sum * w[v] * h[row]; row = map[n] clamped to `rows` (map NULL: n).
struct OperandScales {
    const float* w; const float* h; const int32_t* map; int32_t rows;
};
// Logits of n tokens, C[n, V] = H W^T with pitch ldc, by tiles of the given kind. k2: bytes of an operand row / 2 (a multiple of 64). Row n
// of the tokens is row map[n] (clamped to h_rows) of H, or n where map is NULL, as it has to be for the largest tile.
struct LogitsOut {
    int tile;
    const void* W; int32_t V; int32_t k2;
    const void* H; int64_t h_rows; const int32_t* map; int32_t n;
    void* C; int64_t ldc;
};
// The same GEMM with the statistics in its epilogue (C NULL: the logits are not stored; otherwise ldc holds whole tiles).
// tau: of groups whose maximum does not exceed tau[n] the logits are not stored (NULL: all are). first, count: tiles of the launch in the
// order of the walk (count < 0: to the last).
struct StatsTiles { StatsPart part; TokenArgs tokens; const int32_t* y; ChunkView cv; const float* tau; int first, count; };
// Leading tiles of the walk (256 rows), whole bands of rows from vocabulary entry 0 on, that a call with alternatives launches ahead of the rest
// (0: none), and how many groups of rows they are.
int stats_lead_tiles(int tile, int32_t V, int32_t n, int32_t top_k, int cus, int32_t* groups);
int mfma_stats_setup(int* compute_units);
int mfma_i8_setup(int* compute_units);
void launch_stats_bf16(const LogitsOut& g, const StatsTiles& t, int cus, hipStream_t st);
void launch_stats_i8(const LogitsOut& g, const OperandScales& s, const StatsTiles& t, int cus, hipStream_t st);
void launch_logits_i8(const LogitsOut& g, const OperandScales& s, bool out_bf16, int cus, hipStream_t st);  // C float32 or bfloat16
// bfloat16 gradient entries of a chunk in the blocked layout (see launch_mfma_logits_grad).
void launch_mfma_stats_grad(const void* W, int32_t V, int32_t D, const void* Hc, ChunkView cv, const int32_t* y, const StatsGrad& g, void* G,
                            int32_t Vp, hipStream_t st);
// launch_mfma_dw with a bfloat16 result, overwritten.
void launch_mfma_dw_bf16(int cus, const void* G, int32_t Vp, const void* HcT, int32_t n_cp, int32_t V, int32_t D, void* dW, float* partial,
                         hipStream_t st);
// The gradient by tiles of 128 x 128 (see small_grad): the entries row-major both ways, G[n_c, Vk] and GT[V, n_sum] (Vk, n_sum: V, n_c up to
// multiples of 64, zero there), H's rows through a map. HT: see GatherRows::transpose, by blocks of 128.
struct SmallGrad {
    const void* W; int32_t V, D;
    const void* H; int64_t h_rows; const int32_t* map; ChunkView cv; int32_t n_sum, Vk;
    void* G; void* GT; const void* HT; float* partial;
};
constexpr int32_t SMALL_BLOCK_ROWS = 128;
void launch_small_grad(const SmallGrad& s, const int32_t* y, const StatsGrad& g, hipStream_t st);
void launch_small_dh(const SmallGrad& s, const StoreSpec& out, int cus, hipStream_t st);
void launch_small_dw(const SmallGrad& s, const StoreSpec& out, bool bf16, int cus, hipStream_t st);

// ---- 8-bit rows (quantize.hip) -------------------------------------------------
void launch_quantize_rows(int dtype, const void* X, int64_t rows, int32_t D, int8_t* q, int64_t pitch, float* scale, hipStream_t st);

}  // namespace dppo
