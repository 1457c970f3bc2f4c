// C entry points of the token statistics, their gradient and the 8-bit operators: argument validation, workspace planning and the
// kernels' order on the caller's stream. No device memory is allocated here.
#include "api_internal.h"
#include "gemm_f32_plan.h"
#include "stats_internal.h"

namespace dppo {
namespace {

enum { F32 = 0, BF16 = 1, I8 = 2 };
constexpr int32_t I8_ROW = 128;             // 8-bit rows are whole GEMM slices
constexpr int32_t I8_D_MAX = 130944;        // 128 * 128 * D stays below 2^31 (-128 is no result of quantisation, but a value)
constexpr int32_t V_MAX = 1 << 30;
// Logits of a forward chunk, where they are stored (elsewhere a bound alike: larger chunks gain nothing there).
constexpr size_t LOGITS_CHUNK_BYTES = (size_t)8 << 30;

struct Regions {                            // offsets into the workspace
    int32_t Vp, n_cp;
    size_t row_bytes;
    size_t o_hc, o_scale, o_z, o_pstats, o_pkeys, o_mx, o_sd, o_zy, o_tau;                    // forward
    size_t o_wt, o_dwpart, o_dwacc, o_hct, o_gt, o_fpart, o_y, o_rowc;                      // backward
    bool direct_w;
    bool small;                             // the gradient by small tiles (see SmallGrad), of one chunk
    int f32_parts;
    size_t total;
};
size_t element_bytes(int dtype) { return dtype == F32 ? 4 : dtype == BF16 ? 2 : 1; }

enum { FORWARD = 0, BACKWARD = 1, BACKWARD_BF16_DW = 2 };

void layout(const dppo_head_shape& s, int32_t top_k, int what, int32_t n_cp, Regions& r) {
    r = Regions{};
    r.Vp = round_up32(s.V, mfma_vocab_tile());
    r.n_cp = n_cp;
    r.row_bytes = (size_t)s.D * element_bytes(s.dtype);
    size_t off = 0;
    auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes, REGION_ALIGN); return o; };
    const size_t n = (size_t)n_cp;
    if (what == FORWARD) {
        r.o_hc = take(s.dtype == F32 ? 0 : n * r.row_bytes);
        r.o_scale = take(s.dtype == I8 ? n * 4 : 0);
        r.o_z = take(s.dtype == F32 || top_k > 0 ? n * r.Vp * 4 : 0);
        // (16 tokens in 32-row tiles and 128 in 128-row ones are no more pairs than 256 in 256-row ones)
        const size_t large = n * mfma_logits_row_tiles(s.V), pairs = s.dtype == F32 ? 0 : large > SMALL_TILE_PAIRS ? large : SMALL_TILE_PAIRS;
        r.o_mx = take(pairs * STATS_GROUPS * 4);
        r.o_sd = take(pairs * STATS_GROUPS * sizeof(float2));
        r.o_tau = take(s.dtype == F32 ? 0 : n * 4);
        r.o_zy = take(s.dtype == F32 ? 0 : n * 4);
        r.o_y = take(s.dtype == F32 ? 0 : n * 4);
        // float32: rows are cut into parts only where there are fewer than 4 per compute unit: at most 8 * DEFAULT_CUS parts in all
        const size_t parts = s.dtype == F32 ? 8 * DEFAULT_CUS : 0;
        r.o_pstats = take(parts * sizeof(float4));
        r.o_pkeys = take(parts * top_k * sizeof(uint64_t));
        r.total = off;
        return;
    }
    const bool bf16 = s.dtype == BF16;
    r.small = bf16 && n_cp >= s.N && small_grad(s.N, s.D, s.V);
    r.direct_w = r.small || reads_w_directly(s.N, s.D);
    r.o_wt = take(bf16 && !r.direct_w ? gemm_b_blocked_elems(s.D, r.Vp) * 2 : 0);
    r.o_dwpart = take(bf16 ? mfma_dw_partial_bytes() : 0);
    r.o_dwacc = take(what == BACKWARD_BF16_DW && n_cp < s.N ? (size_t)s.V * s.D * 4 : 0);
    r.o_hc = take(n * r.row_bytes);
    r.o_hct = take(bf16 ? gemm_b_blocked_elems(s.D, n_cp) * 2 : 0);
    r.o_z = take(n * r.Vp * element_bytes(s.dtype));
    r.o_gt = take(r.small ? (size_t)round_up32(s.N, GEMM_B_BLOCK_K) * s.V * 2 : 0);
    const int64_t max_parts = r.Vp / s.D, k_parts = gemm_f32_max_parts(s.V);
    r.f32_parts = bf16 ? 0 : (int)(max_parts < k_parts ? max_parts : k_parts);
    r.o_fpart = take(r.f32_parts > 1 ? (size_t)r.f32_parts * n * s.D * 4 : 0);
    r.o_y = take(n * 4);
    r.o_rowc = take(n * 4);
    r.total = off;
}

int32_t wanted_chunk(const dppo_head_shape& s, int what, int cus) {
    if (what != FORWARD) return target_chunk(s.N, s.D, s.V, element_bytes(s.dtype), cus);
    const int64_t room = (int64_t)(LOGITS_CHUNK_BYTES / ((size_t)round_up32(s.V, mfma_vocab_tile()) * 4)) / CHUNK_ALIGN * CHUNK_ALIGN;
    const int64_t most = room < CHUNK_ALIGN ? CHUNK_ALIGN : room > 32768 ? 32768 : room;
    const int64_t chunks = s.N > 0 ? ceil_div(s.N, most) : 1;
    return round_up32(ceil_div(s.N > 0 ? s.N : 1, chunks), CHUNK_ALIGN);
}

// Fewest bytes that some chunk size fits: the smallest chunk's, or, as one chunk needs no float32 sum of a bfloat16 dW, the wanted one's.
size_t least_bytes(const dppo_head_shape& s, int32_t top_k, int what) {
    Regions r;
    layout(s, top_k, what, CHUNK_ALIGN, r);
    const size_t smallest = r.total;
    layout(s, top_k, what, wanted_chunk(s, what, DEFAULT_CUS), r);
    return r.total < smallest ? r.total : smallest;
}
int check_least(const dppo_head_shape& s, int32_t top_k, int what, size_t ws_bytes) {
    const size_t least = least_bytes(s, top_k, what);
    if (ws_bytes < least) return fail(DPPO_ERR_WORKSPACE, "workspace of %zu bytes is below the minimum of %zu", ws_bytes, least);
    return DPPO_OK;
}

// Largest chunk, up to the wanted one, whose regions fit.
int plan(const dppo_head_shape& s, int32_t top_k, int what, size_t ws_bytes, int cus, Regions& r) {
    int32_t hi = wanted_chunk(s, what, cus) / CHUNK_ALIGN;
    layout(s, top_k, what, hi * CHUNK_ALIGN, r);
    if (r.total <= ws_bytes) return DPPO_OK;
    layout(s, top_k, what, CHUNK_ALIGN, r);
    if (r.total > ws_bytes)
        return fail(DPPO_ERR_WORKSPACE, "workspace of %zu bytes is below the minimum of %zu", ws_bytes, r.total);
    int32_t lo = 1;
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) / 2;
        layout(s, top_k, what, mid * CHUNK_ALIGN, r);
        if (r.total <= ws_bytes) lo = mid; else hi = mid;
    }
    layout(s, top_k, what, lo * CHUNK_ALIGN, r);
    return DPPO_OK;
}

int validate(const dppo_head_shape* s, int32_t top_k, bool backward) {
    if (!s) return fail(DPPO_ERR_INVALID_ARG, "shape is NULL");
    if (s->dtype < F32 || s->dtype > I8 || (backward && s->dtype == I8))
        return fail(DPPO_ERR_UNSUPPORTED, "dtype %d (0 = float32, 1 = bfloat16, without gradients 2 = int8)", s->dtype);
    if (s->T < 0 || s->N < 0 || s->N > s->T) return fail(DPPO_ERR_SHAPE, "need 0 <= N <= T (T=%lld N=%lld)", (long long)s->T, (long long)s->N);
    if (s->D <= 0 || s->V <= 0) return fail(DPPO_ERR_SHAPE, "need D > 0 and V > 0 (D=%d V=%d)", s->D, s->V);
    if (s->T > 0x7fffffffLL || s->V > V_MAX) return fail(DPPO_ERR_UNSUPPORTED, "T above 2^31-1 packed tokens or V above 2^30");
    if (s->dtype == BF16 && s->D % 64 != 0) return fail(DPPO_ERR_UNSUPPORTED, "bfloat16 path needs D %% 64 == 0 (D=%d)", s->D);
    if (s->dtype == I8 && (s->D % I8_ROW != 0 || s->D > I8_D_MAX))
        return fail(DPPO_ERR_UNSUPPORTED, "int8 rows are padded to multiples of %d bytes, at most %d (D=%d)", I8_ROW, I8_D_MAX, s->D);
    if (top_k < 0 || top_k > DPPO_TOP_K_MAX || top_k > s->V)
        return fail(DPPO_ERR_INVALID_ARG, "top_k must lie in [0, min(%d, V)] (%d)", DPPO_TOP_K_MAX, top_k);
    return DPPO_OK;
}

int check_workspace(const void* ws) {
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u)) return fail(DPPO_ERR_WORKSPACE, "workspace is NULL or not 256-byte aligned");
    return DPPO_OK;
}

ChunkView view(int64_t n0, int64_t N, int32_t n_cp) {
    ChunkView cv;
    cv.n0 = n0;
    cv.n_c = (int32_t)(N - n0 < n_cp ? N - n0 : n_cp);
    cv.n_cp = round_up32(cv.n_c, CHUNK_ALIGN);
    return cv;
}

}  // namespace
}  // namespace dppo

using namespace dppo;

extern "C" {

size_t dppo_token_stats_workspace_bytes(const dppo_head_shape* shape, int32_t top_k, int want_backward) {
    if (want_backward < FORWARD || want_backward > BACKWARD_BF16_DW || validate(shape, top_k, want_backward != 0) != DPPO_OK) return 0;
    Regions r;
    layout(*shape, top_k, want_backward, wanted_chunk(*shape, want_backward, DEFAULT_CUS), r);
    return r.total;
}

size_t dppo_token_stats_workspace_min_bytes(const dppo_head_shape* shape, int32_t top_k, int want_backward) {
    if (want_backward < FORWARD || want_backward > BACKWARD_BF16_DW || validate(shape, top_k, want_backward != 0) != DPPO_OK) return 0;
    return least_bytes(*shape, top_k, want_backward);
}

int dppo_token_stats(const dppo_head_shape* shape, int32_t top_k, const void* H, const void* W, const float* h_scale,
                     const float* w_scale, const int32_t* ids, const int32_t* loss_pos, float* logp, float* lse, float* entropy,
                     int32_t* top_ids, float* top_logp, int32_t* status, void* ws, size_t ws_bytes, void* stream) {
    int rc = validate(shape, top_k, false);
    if (rc != DPPO_OK) return rc;
    const dppo_head_shape& s = *shape;
    if (s.N == 0) return finish_without_tokens("dppo_token_stats", status, (hipStream_t)stream);
    if (!H || !W) return fail(DPPO_ERR_INVALID_ARG, "H and W must not be NULL");
    if ((s.dtype == I8) != (h_scale != nullptr) || (s.dtype == I8) != (w_scale != nullptr))
        return fail(DPPO_ERR_INVALID_ARG, "h_scale and w_scale belong to int8 operands and to no others");
    if (logp && !ids) return fail(DPPO_ERR_INVALID_ARG, "logp needs the token ids");
    if (!logp && !lse && !entropy && top_k == 0) return fail(DPPO_ERR_INVALID_ARG, "no output is asked for");
    if ((top_k > 0) != (top_ids != nullptr) || (top_k > 0) != (top_logp != nullptr))
        return fail(DPPO_ERR_INVALID_ARG, "top_ids and top_logp are needed where top_k > 0, and only there");
    if (s.dtype != F32 && (!aligned16(H) || !aligned16(W))) return fail(DPPO_ERR_INVALID_ARG, "H and W must be 16-byte aligned");
    if ((rc = check_workspace(ws)) != DPPO_OK) return rc;
    if ((rc = check_least(s, top_k, FORWARD, ws_bytes)) != DPPO_OK) return rc;
    int cus = DEFAULT_CUS;
    if (s.dtype == BF16 && (rc = mfma_stats_setup(&cus)) != DPPO_OK) return rc;
    if (s.dtype == I8 && (rc = mfma_i8_setup(&cus)) != DPPO_OK) return rc;
    Regions r;
    if ((rc = plan(s, top_k, FORWARD, ws_bytes, cus, r)) != DPPO_OK) return rc;

    hipStream_t st = (hipStream_t)stream;
    char* w = reinterpret_cast<char*>(ws);
    float* Z = reinterpret_cast<float*>(w + r.o_z);
    const TokenArgs tokens{H, W, logp ? ids : nullptr, loss_pos, s.T, s.D, s.V, status};
    const StatsOut out{lse, entropy, logp, top_ids, top_logp, top_k};
    if (status) launch_fill_zero(nullptr, 0, status, st);
    for (int64_t n0 = 0; n0 < s.N; n0 += r.n_cp) {
        const ChunkView cv = view(n0, s.N, r.n_cp);
        const int32_t* map = loss_pos ? loss_pos + n0 : nullptr;
        if (s.dtype == F32) {
            const float* A = reinterpret_cast<const float*>(H) + (map ? 0 : (size_t)n0 * s.D);
            GemmF32 g{A, s.D, 0, reinterpret_cast<const float*>(W), s.D, 0, cv.n_c, s.V, s.D, Z, r.Vp, 0, nullptr, nullptr, 0,
                      map, (int32_t)s.T};
            launch_gemm_f32(g, cus, st);
            StageTimer tm(DPPO_STAGE_ELEMENTWISE, st);
            PartialStats partial{reinterpret_cast<float4*>(w + r.o_pstats), reinterpret_cast<uint64_t*>(w + r.o_pkeys),
                                 stats_row_parts(cv.n_c, s.V, DEFAULT_CUS)};
            launch_stats_rows(Z, r.Vp, tokens, out, cv, partial, st);
            continue;
        }
        // All tiles but the largest read the rows through loss_pos, and their epilogue looks the targets up. For the largest both are gathered first.
        const int32_t k2 = (int32_t)(r.row_bytes / 2);
        const int tile = logits_tile(cv.n_c, s.V, k2, s.dtype == I8);
        const bool gather = tile == TILE_256x256;
        const char* rows = reinterpret_cast<const char*>(H) + (map ? 0 : (size_t)n0 * r.row_bytes);
        LogitsOut g{tile, W, s.V, k2, rows, map ? s.T : (int64_t)cv.n_c, map, cv.n_c, top_k > 0 ? Z : nullptr, r.Vp};
        OperandScales sc{w_scale, h_scale ? h_scale + (map ? 0 : n0) : nullptr, map, (int32_t)g.h_rows};
        int32_t* y = reinterpret_cast<int32_t*>(w + r.o_y);
        if (gather && (map || logp)) {
            StageTimer tm(DPPO_STAGE_ELEMENTWISE, st);
            float* scale = reinterpret_cast<float*>(w + r.o_scale);
            GatherRows gr{tokens, r.row_bytes, h_scale, map ? w + r.o_hc : nullptr, y, nullptr, s.dtype == I8 ? scale : nullptr, nullptr, 0, nullptr, 0, 0};
            launch_stats_gather(gr, cv, st);
            if (map) { g.H = w + r.o_hc; g.h_rows = cv.n_c; g.map = nullptr; }
            if (map) { sc.h = scale; sc.map = nullptr; sc.rows = cv.n_c; }
        }
        const bool alone = cv.n_c <= JOIN_ALONE;
        StatsTiles t{{reinterpret_cast<float*>(w + r.o_mx), reinterpret_cast<float2*>(w + r.o_sd),
                      logp ? reinterpret_cast<float*>(w + r.o_zy) : nullptr, alone ? 1 : cv.n_c, alone ? groups_of_tiles(tile, s.V) : 1},
                     tokens, gather ? y : nullptr, cv, nullptr, 0, -1};
        auto gemm = [&]() {
            StageTimer tm(DPPO_STAGE_LOGITS_GEMM, st);
            if (s.dtype == BF16) launch_stats_bf16(g, t, cus, st);
            else launch_stats_i8(g, sc, t, cus, st);
        };
        int32_t groups = 0;
        const int lead = stats_lead_tiles(tile, s.V, cv.n_c, top_k, cus, &groups);
        if (lead > 0) {
            float* tau = reinterpret_cast<float*>(w + r.o_tau);
            t.count = lead;
            gemm();
            StageTimer tm(DPPO_STAGE_ELEMENTWISE, st);
            launch_stats_bound(t.part, groups, top_k, cv, tau, st);
            t.tau = tau; t.first = lead; t.count = -1;
        }
        gemm();
        StageTimer tm(DPPO_STAGE_ELEMENTWISE, st);
        launch_stats_join(t.part, group_rows(tile), Z, r.Vp, tokens, !gather, out, cv, st);
    }
    return check_launch("dppo_token_stats");
}

int dppo_token_stats_bwd(const dppo_head_shape* shape, const dppo_stats_grad_params* p, const void* H, const void* W,
                         const int32_t* ids, const int32_t* loss_pos, const float* lse, const float* entropy, const float* g_logp,
                         const float* g_lse, const float* g_entropy, void* dH, void* dW, int32_t* status, void* ws,
                         size_t ws_bytes, void* stream) {
    int rc = validate(shape, 0, true);
    if (rc != DPPO_OK) return rc;
    const dppo_head_shape& s = *shape;
    if (!p) return fail(DPPO_ERR_INVALID_ARG, "params is NULL");
    if (p->dW_dtype != F32 && p->dW_dtype != BF16) return fail(DPPO_ERR_UNSUPPORTED, "dW_dtype %d (0 = float32, 1 = bfloat16)", p->dW_dtype);
    const bool dw16 = p->dW_dtype == BF16;
    if (dw16 && (s.dtype != BF16 || p->accumulate_dW))
        return fail(DPPO_ERR_UNSUPPORTED, "a bfloat16 dW belongs to bfloat16 operands and is overwritten, not added to");
    if ((!dH && s.T > 0) || !dW || !W) return fail(DPPO_ERR_INVALID_ARG, "dH, dW and W must not be NULL");
    if (s.N > 0 && !g_logp && !g_lse && !g_entropy) return fail(DPPO_ERR_INVALID_ARG, "no incoming gradient");
    if (s.N > 0 && (!H || !lse)) return fail(DPPO_ERR_INVALID_ARG, "H and lse must not be NULL");
    if (s.N > 0 && g_logp && !ids) return fail(DPPO_ERR_INVALID_ARG, "g_logp needs the token ids");
    if (s.N > 0 && g_entropy && !entropy) return fail(DPPO_ERR_INVALID_ARG, "g_entropy needs the entropies of the forward pass");
    if (s.dtype == BF16 && (!aligned16(H) || !aligned16(W) || !aligned16(dH) || !aligned16(dW)))
        return fail(DPPO_ERR_INVALID_ARG, "H, W, dH and dW must be 16-byte aligned");
    if ((rc = check_workspace(ws)) != DPPO_OK) return rc;
    const int what = dw16 ? BACKWARD_BF16_DW : BACKWARD;
    if ((rc = check_least(s, 0, what, ws_bytes)) != DPPO_OK) return rc;
    int cus = DEFAULT_CUS;
    if (s.dtype == BF16 && ((rc = mfma_stats_setup(&cus)) != DPPO_OK || (rc = mfma_setup(nullptr)) != DPPO_OK)) return rc;
    Regions r;
    if ((rc = plan(s, 0, what, ws_bytes, cus, r)) != DPPO_OK) return rc;

    hipStream_t st = (hipStream_t)stream;
    char* w = reinterpret_cast<char*>(ws);
    {
        StageTimer tm(DPPO_STAGE_ELEMENTWISE, st);
        // dH is cleared beside the first chunk's gathering, in one launch; the status word before it
        launch_fill_zero(dH, s.N == 0 ? (size_t)s.T * r.row_bytes : 0, status, st);
        if (s.N == 0 && !p->accumulate_dW) launch_fill_zero(dW, (size_t)s.V * s.D * (dw16 ? 2 : 4), nullptr, st);
        if (s.N > 0 && s.dtype == BF16 && !r.direct_w) launch_transpose_w(W, s.V, s.D, r.Vp, w + r.o_wt, st);
    }
    const TokenArgs tokens{H, W, g_logp ? ids : nullptr, loss_pos, s.T, s.D, s.V, status};
    const StatsGrad grad{g_logp, g_lse, g_entropy, lse, entropy};
    int32_t* y = reinterpret_cast<int32_t*>(w + r.o_y);
    int32_t* rowc = reinterpret_cast<int32_t*>(w + r.o_rowc);
    void *Hc = w + r.o_hc, *G = w + r.o_z;
    const bool one_chunk = r.n_cp >= s.N;
    // bfloat16 dW of several chunks: summed in float32, rounded once at the end
    float* dw_sum = dw16 && !one_chunk ? reinterpret_cast<float*>(w + r.o_dwacc) : reinterpret_cast<float*>(dW);
    for (int64_t n0 = 0; n0 < s.N; n0 += r.n_cp) {
        const ChunkView cv = view(n0, s.N, r.n_cp);
        // dW sums over the chunk's tokens up to whole slices of its GEMM
        const int32_t n_sum = round_up32(cv.n_c, GEMM_B_BLOCK_K);
        const GatherRows rows{tokens, r.row_bytes, nullptr, r.small ? nullptr : Hc, y, rowc, nullptr, n0 == 0 ? dH : nullptr,
                              n0 == 0 ? (size_t)s.T * r.row_bytes : 0, s.dtype == BF16 ? w + r.o_hct : nullptr, n_sum,
                              r.small ? SMALL_BLOCK_ROWS : GEMM_B_BLOCK_ROWS};
        if (s.dtype == BF16) {
            StageTimer tm(DPPO_STAGE_ELEMENTWISE, st);
            launch_stats_gather(rows, cv, st);
        }
        StoreSpec oh{loss_pos ? dH : reinterpret_cast<char*>(dH) + (size_t)n0 * r.row_bytes, s.D, 0, loss_pos ? rowc : nullptr};
        StoreSpec ow{dw_sum, s.D, n0 == 0 && !p->accumulate_dW ? 0 : 1, nullptr};
        if (s.dtype == F32) {
            const float* Hf = reinterpret_cast<const float*>(Hc);
            float* Gf = reinterpret_cast<float*>(G);
            const float* A = reinterpret_cast<const float*>(H) + (loss_pos ? 0 : (size_t)n0 * s.D);
            launch_gemm_f32(GemmF32{A, s.D, 0, reinterpret_cast<const float*>(W), s.D, 0, cv.n_c, s.V, s.D, Gf, r.Vp, 0, nullptr, nullptr, 0,
                                    loss_pos ? loss_pos + n0 : nullptr, (int32_t)s.T}, cus, st);
            {
                StageTimer tm(DPPO_STAGE_GRAD_LOGITS, st);
                launch_stats_grad_f32(Gf, r.Vp, grad, rows, cv, st);
            }
            launch_gemm_f32(GemmF32{Gf, r.Vp, 0, reinterpret_cast<const float*>(W), s.D, 1, cv.n_c, s.D, s.V, reinterpret_cast<float*>(oh.C),
                                    oh.ldc, 0, oh.row_map, r.f32_parts > 1 ? reinterpret_cast<float*>(w + r.o_fpart) : nullptr,
                                    (int64_t)r.f32_parts * r.n_cp * s.D, nullptr, 0}, cus, st);
            launch_gemm_f32(GemmF32{Gf, r.Vp, 1, Hf, s.D, 1, s.V, s.D, cv.n_c, dw_sum, ow.ldc, ow.accumulate, nullptr, nullptr, 0, nullptr, 0},
                            cus, st);
            continue;
        }
        if (r.small) {
            const SmallGrad sg{W, s.V, s.D, H, loss_pos ? s.T : (int64_t)cv.n_c, loss_pos, cv, n_sum, round_up32(s.V, GEMM_B_BLOCK_K),
                               G, w + r.o_gt, w + r.o_hct, reinterpret_cast<float*>(w + r.o_dwpart)};
            {
                StageTimer tm(DPPO_STAGE_LOGITS_GEMM, st);
                launch_small_grad(sg, y, grad, st);
            }
            {
                StageTimer tm(DPPO_STAGE_DH_GEMM, st);
                launch_small_dh(sg, oh, cus, st);
            }
            StageTimer tm(DPPO_STAGE_DW_GEMM, st);
            launch_small_dw(sg, ow, dw16, cus, st);
            continue;
        }
        {
            StageTimer tm(DPPO_STAGE_LOGITS_GEMM, st);
            launch_mfma_stats_grad(W, s.V, s.D, Hc, cv, y, grad, G, r.Vp, st);
        }
        float* partial = reinterpret_cast<float*>(w + r.o_dwpart);
        {
            StageTimer tm(DPPO_STAGE_DH_GEMM, st);
            // partial tiles of dH: where dW is overwritten just behind, its memory holds more of them than the workspace
            float* dh_partial = partial;
            int64_t floats = (int64_t)(mfma_dw_partial_bytes() / 4);
            const int64_t dw_floats = (int64_t)s.V * s.D / (dw16 && one_chunk ? 2 : 1);
            if (!ow.accumulate && dw_floats > floats) { dh_partial = dw_sum; floats = dw_floats; }
            launch_mfma_dh(cus, G, r.Vp, r.direct_w ? nullptr : w + r.o_wt, W, s.V, cv.n_c, s.D, nullptr, oh, dh_partial, floats, st);
        }
        StageTimer tm(DPPO_STAGE_DW_GEMM, st);
        if (dw16 && one_chunk) launch_mfma_dw_bf16(cus, G, r.Vp, w + r.o_hct, n_sum, s.V, s.D, dW, partial, st);
        else launch_mfma_dw(cus, G, r.Vp, w + r.o_hct, n_sum, s.V, s.D, ow, partial, st);
    }
    if (dw16 && !one_chunk && s.N > 0) {
        StageTimer tm(DPPO_STAGE_ELEMENTWISE, st);
        launch_to_bf16(dw_sum, dW, (size_t)s.V * s.D, st);
    }
    return check_launch("dppo_token_stats_bwd");
}

int dppo_quantize_rows(int64_t rows, int32_t D, int32_t dtype, const void* X, int8_t* q, int64_t q_pitch, float* scale, void* stream) {
    if (rows < 0 || D <= 0) return fail(DPPO_ERR_SHAPE, "need rows >= 0 and D > 0 (rows=%lld D=%d)", (long long)rows, D);
    if (rows > 0x7fffffffLL) return fail(DPPO_ERR_UNSUPPORTED, "more than 2^31-1 rows");
    if (dtype != F32 && dtype != BF16) return fail(DPPO_ERR_UNSUPPORTED, "dtype %d (0 = float32, 1 = bfloat16)", dtype);
    if (q_pitch < D || q_pitch % I8_ROW != 0 || q_pitch > I8_D_MAX)
        return fail(DPPO_ERR_SHAPE, "q_pitch must be a multiple of %d in [D, %d] (%lld, D=%d)", I8_ROW, I8_D_MAX, (long long)q_pitch, D);
    if (rows == 0) return DPPO_OK;
    if (!X || !q || !scale) return fail(DPPO_ERR_INVALID_ARG, "a required array pointer is NULL");
    if (!aligned16(q)) return fail(DPPO_ERR_INVALID_ARG, "q must be 16-byte aligned");
    launch_quantize_rows(dtype, X, rows, D, q, q_pitch, scale, (hipStream_t)stream);
    return check_launch("dppo_quantize_rows");
}

int dppo_matmul_i8(int64_t T, int32_t V, int32_t D, const int8_t* X, const float* x_scale, const int8_t* W, const float* w_scale,
                   void* Y, int32_t out_dtype, void* stream) {
    const dppo_head_shape s{T, T, D, V, I8};
    int rc = validate(&s, 0, false);
    if (rc != DPPO_OK) return rc;
    if (out_dtype != F32 && out_dtype != BF16) return fail(DPPO_ERR_UNSUPPORTED, "out_dtype %d (0 = float32, 1 = bfloat16)", out_dtype);
    if (T == 0) return DPPO_OK;
    if (!X || !x_scale || !W || !w_scale || !Y) return fail(DPPO_ERR_INVALID_ARG, "a required array pointer is NULL");
    if (!aligned16(X) || !aligned16(W)) return fail(DPPO_ERR_INVALID_ARG, "X and W must be 16-byte aligned");
    int cus = 0;
    if ((rc = mfma_i8_setup(&cus)) != DPPO_OK) return rc;
    hipStream_t st = (hipStream_t)stream;
    StageTimer tm(DPPO_STAGE_LOGITS_GEMM, st);
    constexpr int64_t CHUNK = 32768;
    for (int64_t n0 = 0; n0 < T; n0 += CHUNK) {
        const int32_t n = (int32_t)(T - n0 < CHUNK ? T - n0 : CHUNK);
        LogitsOut g{logits_tile(n, V, D / 2, true), W, V, D / 2, X + (size_t)n0 * D, n, nullptr, n,
                    reinterpret_cast<char*>(Y) + (size_t)n0 * V * element_bytes(out_dtype), V};
        launch_logits_i8(g, OperandScales{w_scale, x_scale + n0, nullptr, n}, out_dtype == BF16, cus, st);
    }
    return check_launch("dppo_matmul_i8");
}

}  // extern "C"
