// Kernels around the logits GEMMs of dppo_token_stats and dppo_token_stats_bwd: softmax statistics and top alternatives of stored
// logits, gathering of rows, gradient entries of the float32 path.
#include <type_traits>

#include "api_internal.h"
#include "stats_internal.h"
#include "top_list.h"
#include "token_rows.h"

namespace dppo {
namespace {


// What one token's statistics and alternatives go to (any of the pointers may be NULL).
__device__ __forceinline__ void write_token(const StatsOut& o, int64_t n, const Stats& s, float target_logit) {
    const float log_sum = logf(s.sum), lse = s.m + log_sum;
    if (o.lse) o.lse[n] = lse;
    if (o.entropy) o.entropy[n] = log_sum - s.dev / s.sum;
    if (o.logp) o.logp[n] = target_logit - lse;
}
__device__ __forceinline__ void write_top(const StatsOut& o, int64_t n, const Stats& s, const TopList& top, int lane) {
    if (lane >= o.top_k) return;
    const float lse = s.m + logf(s.sum);
    o.top_ids[n * o.top_k + lane] = (int32_t)top_index(top.entry);
    o.top_logp[n * o.top_k + lane] = top_value(top.entry) - lse;
}

// ORs what is wrong with loss token i's position or target into *a.status.
__device__ __forceinline__ void report_token(const TokenArgs& a, int64_t i) {
    int64_t row;
    int32_t target;
    int flags = 0;
    if (a.ids) {
        flags = locate_token(a.ids, a.loss_pos, a.T, a.V, i, row, target);
    } else if (a.loss_pos) {
        row = a.loss_pos[i];
        if (row < 0 || row >= a.T) flags = DPPO_HEAD_BAD_POSITION;
    }
    if (flags != 0) atomicOr(a.status, flags);
}

// One workgroup per token and part of its row of stored logits (pitch a multiple of 256; columns from V on hold anything): one pass
// over the logits, which are bound by HBM or L2, 4 bytes each. Each wavefront keeps statistics per lane and one list of the
// top_k largest; a logit below the list's last entry costs a comparison of four logits' maximum. parts > 1 (few tokens): the
// workgroup's results go to `partial`, and join_parts_kernel puts the parts together.
constexpr int ROWS_THREADS = 256, ROWS_WAVES = ROWS_THREADS / 64, ROWS_UNROLL = 4;
template <bool TOP>
__global__ __launch_bounds__(ROWS_THREADS) void stats_rows_kernel(const float* __restrict__ Z, int64_t ldz, TokenArgs a, StatsOut o,
                                                                  ChunkView cv, PartialStats partial) {
    __shared__ Stats red[ROWS_WAVES];
    __shared__ uint64_t lists[TOP ? ROWS_WAVES : 1][PENDING4];
    const int n = blockIdx.x, part = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float NONE = -__builtin_inff();
    const float* z = Z + (size_t)n * ldz;
    const int vectors = (a.V + 3) / 4;
    const int lo = (int)((int64_t)vectors * part / partial.parts), hi = (int)((int64_t)vectors * (part + 1) / partial.parts);
    Stats s = no_stats();
    TopList top(lists[TOP ? wave : 0]);
    // (whole wavefronts walk the loop: the list needs every lane)
    for (int i0 = lo + wave * 64; i0 < hi; i0 += ROWS_THREADS * ROWS_UNROLL) {
        float x[ROWS_UNROLL][4], m4[ROWS_UNROLL];
#pragma unroll
        for (int u = 0; u < ROWS_UNROLL; ++u) {
            const int i = i0 + u * ROWS_THREADS + lane;
            float4 v = make_float4(NONE, NONE, NONE, NONE);
            if (i < hi) v = reinterpret_cast<const float4*>(z)[i];
            const float vv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int q = 0; q < 4; ++q) x[u][q] = i * 4 + q < a.V ? vv[q] : NONE;
        }
        float m = NONE;
#pragma unroll
        for (int u = 0; u < ROWS_UNROLL; ++u) {
            m4[u] = fmaxf(fmaxf(x[u][0], x[u][1]), fmaxf(x[u][2], x[u][3]));
            m = fmaxf(m, m4[u]);
        }
        const float ref = m == NONE ? 0.0f : m;
        Stats b{m, 0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < ROWS_UNROLL; ++u)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float d = x[u][q] - ref, e = exp_fast(d);
                b.sum += e;
                b.dev = fmaf(fmaxf(d, DEV_MIN), e, b.dev);
            }
        s = join(s, b);
        if (TOP) {
            // (k lanes' maxima of the first logits bound what the list begins with)
            if (i0 == lo + wave * 64) top.at_least(kth_of_lanes(m, o.top_k, lane));
#pragma unroll
            for (int u = 0; u < ROWS_UNROLL; ++u) {
                if (!__any(!(m4[u] < top.floor))) continue;
                const int i = i0 + u * ROWS_THREADS + lane;
                top.add4(x[u], i * 4, i < hi ? a.V : 0);
                top.take(o.top_k, lane, 63);
            }
        }
    }
    s = join_lanes<1>(s);
    if (lane == 0) red[wave] = s;
    if (TOP) {
        top.take(o.top_k, lane, 0);
        lists[wave][lane] = top.entry;
    }
    __syncthreads();
    if (wave != 0) return;
    for (int w = 1; w < ROWS_WAVES; ++w) s = join(s, red[w]);
    if (TOP) {
        for (int w = 1; w < ROWS_WAVES; ++w) top.merge(lists[w][lane], lane);
    }
    const int64_t gi = cv.n0 + n;
    if (partial.parts > 1) {
        const size_t at = (size_t)n * partial.parts + part;
        if (lane == 0) partial.stats[at] = make_float4(s.m, s.sum, s.dev, 0.0f);
        if (TOP && lane < o.top_k) partial.keys[at * o.top_k + lane] = top.entry;
        return;
    }
    float zy = 0.0f;
    if (a.ids) {
        int64_t row;
        int32_t target;
        locate_token(a.ids, a.loss_pos, a.T, a.V, gi, row, target);
        zy = z[target];
    }
    if (a.status != nullptr && lane == 0) report_token(a, gi);
    if (lane == 0) write_token(o, gi, s, zy);
    if (TOP) write_top(o, gi, s, top, lane);
}

// Puts the parts of a token's row together: one wavefront per token, a part's statistics per lane.
template <bool TOP>
__global__ __launch_bounds__(64) void join_parts_kernel(const float* __restrict__ Z, int64_t ldz, TokenArgs a, StatsOut o, ChunkView cv,
                                                        PartialStats partial) {
    const int n = blockIdx.x, lane = threadIdx.x;
    const size_t at = (size_t)n * partial.parts;
    Stats s = no_stats();
    for (int p = lane; p < partial.parts; p += 64) {
        const float4 v = partial.stats[at + p];
        s = join(s, Stats{v.x, v.y, v.z});
    }
    s = join_lanes<1>(s);
    __shared__ uint64_t pending[PENDING];
    TopList top(pending);
    if (TOP) {
        const int entries = partial.parts * o.top_k;
        for (int i = 0; i < entries; i += 64) {
            top.add(i + lane < entries ? partial.keys[at * o.top_k + i + lane] : 0);
            top.take(o.top_k, lane, i + 64 < entries ? 63 : 0);
        }
    }
    const int64_t gi = cv.n0 + n;
    float zy = 0.0f;
    if (a.ids) {
        int64_t row;
        int32_t target;
        locate_token(a.ids, a.loss_pos, a.T, a.V, gi, row, target);
        zy = Z[(size_t)n * ldz + target];
    }
    if (a.status != nullptr && lane == 0) report_token(a, gi);
    if (lane == 0) write_token(o, gi, s, zy);
    if (TOP) write_top(o, gi, s, top, lane);
}

// Joins the statistics of TOK tokens per workgroup over the groups of rows, and picks their top alternatives. The k largest logits of a
// token lie in the k groups with the largest maxima (in the order of maximum, then group: every group ahead of another one holds a
// logit that is ahead of all of the other's), so that of the stored logits only those groups are read: k / 2 KB of a row of V.
// The workgroup reads the statistics, neighbouring tokens side by side, the maxima stay in LDS; then up to 16 / TOK wavefronts per token
// list the groups, and after that their logits. Bound by latency up to some 2000 tokens, that of fetching its own code among it: both passes run
// the same instructions (V = 3000, 1 and 20 alternatives, 256 tokens: 10.9 -> 8.2 and 11.4 -> 10.1 us against a pass of its own each).
constexpr int JOIN_THREADS = 1024, JOIN_WAVES = JOIN_THREADS / 64, JOIN_MAXIMA = 10240, JOIN_UNROLL = 6;
template <int TOK, bool TOP>
__global__ __launch_bounds__(JOIN_THREADS) void stats_join_kernel(StatsPart part, int32_t rows, const float* __restrict__ Z, int64_t ldz,
                                                                  TokenArgs a, int look_up, StatsOut o, ChunkView cv) {
    constexpr int LANES = JOIN_THREADS / TOK, WPT = JOIN_WAVES / TOK;       // lanes and wavefronts per token
    constexpr int ROW = TOK + 1, BLOCK = JOIN_MAXIMA / TOK;                 // maxima in LDS: row pitch, groups of a block
    __shared__ float maxima[TOP ? BLOCK * ROW : 1];
    __shared__ Stats red[JOIN_WAVES][TOK];
    __shared__ Stats fin[TOK];
    __shared__ uint64_t pending[TOP ? JOIN_WAVES : 1][PENDING4];
    __shared__ uint64_t lists[TOP ? JOIN_WAVES : 1][TOP_MAX];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int tok = tid % TOK, n = blockIdx.x * TOK + tok;
    const int my_tok = wave / WPT, sub = wave % WPT, my_n = blockIdx.x * TOK + my_tok;   // of the wavefront's list
    const int groups = (a.V + rows - 1) / rows;
    Stats s = no_stats();
    auto load_block = [&](int b0, int b1) __attribute__((always_inline)) {
        if (n >= cv.n_c) return;
        for (int g0 = b0 + tid / TOK; g0 < b1; g0 += LANES * JOIN_UNROLL) {
            float2 sd[JOIN_UNROLL];
            float m[JOIN_UNROLL];
#pragma unroll
            for (int u = 0; u < JOIN_UNROLL; ++u) {
                const int g = g0 + u * LANES;
                if (g >= b1) break;
                m[u] = part.mx[part.at(g, n)];
                sd[u] = part.sd[part.at(g, n)];
            }
#pragma unroll
            for (int u = 0; u < JOIN_UNROLL; ++u) {
                const int g = g0 + u * LANES;
                if (g >= b1) break;
                s = join(s, Stats{m[u], sd[u].x, sd[u].y});
                if (TOP) maxima[(g - b0) * ROW + tok] = m[u];
            }
        }
    };
    auto finish_statistics = [&]() __attribute__((always_inline)) {
        s = join_lanes<TOK>(s);
        if (lane < TOK) red[wave][lane] = s;
        __syncthreads();
        if (wave != 0) return;
        s = no_stats();
        for (int w = lane / TOK; w < JOIN_WAVES; w += 64 / TOK) s = join(s, red[w][tok]);
        s = join_lanes<TOK>(s);
        if (lane >= TOK) return;
        if (TOP) fin[tok] = s;
        if (n < cv.n_c) {
            const int64_t gi = cv.n0 + n;
            if (look_up && a.status != nullptr) report_token(a, gi);
            write_token(o, gi, s, part.zy ? part.zy[n] : 0.0f);
        }
    };
    if (!TOP) {
        load_block(0, groups);
        finish_statistics();
        return;
    }
    // Two passes of the same code: the token's `used` wavefronts list its groups, block by block, then the logits of those that are ahead.
    TopList top(pending[TOP ? wave : 0]);
    const int per = 256 / rows, in = lane % (rows / 4), which = lane / (rows / 4);      // groups of a round of logits, rows / 4 lanes a group
    const float* z = Z + (size_t)my_n * ldz;
    constexpr int ROUNDS = 6;                    // rounds of logits whose loads are under way at once, one round a lane's float4
    float x[ROUNDS][4];
    int v0[ROUNDS];
    uint64_t group = 0;
    bool logits = false;
    int b0 = 0, b1 = 0, first = 0, end = 0, step = 0, used = 1;
    while (used < WPT && used * 128 < groups) used *= 2;
    while (true) {
        bool more = false;                       // a further block of groups
        if (!logits) {
            if (b0 > 0) __syncthreads();
            b1 = groups - b0 < BLOCK ? groups : b0 + BLOCK;
            load_block(b0, b1);
            __syncthreads();
            first = b0 + sub * 64; end = b1; step = used * 64;
            more = b1 < groups;
        }
        if (my_n >= cv.n_c || sub >= used) end = first;
        if constexpr (TOK == 1 || TOK == 16) {
            // Long lists: the lanes' own maxima bound what joins them, a quarter more than k instead of k (1 + log(groups / k)). (V = 151936, 20
            // alternatives: one token 17.8 -> 16.4 us, 8000 84 -> 78; with 4 and 8 tokens a workgroup the registers do not hold it as well.)
            if (!logits && b0 == 0 && end - first > 3 * step) {
                float m = -__builtin_inff();
                for (int g = first + lane; g < end; g += step) m = fmaxf(m, maxima[g * ROW + my_tok]);
                top.at_least(kth_of_lanes(m, o.top_k, lane));
            }
        }
        int ring = 0;
#pragma unroll 1
        for (int i = first;;) {
            const bool valid = i < end;
            if (valid && !logits) {
                const int g = i + lane;
                top.add(g < end ? top_key(maxima[(g - b0) * ROW + my_tok], (uint32_t)g) : 0);
            }
            if (valid && logits) {
                if (ring == 0) {
#pragma unroll
                    for (int u = 0; u < ROUNDS; ++u) {
                        const int at = i + u * step + which;
                        const uint32_t g = top_index((uint64_t)(uint32_t)__shfl((int)(uint32_t)group, at < end ? at : 0, 64));
                        v0[u] = at < end ? (int)g * rows + in * 4 : a.V;
                        if (v0[u] < a.V) *reinterpret_cast<float4*>(x[u]) = *reinterpret_cast<const float4*>(z + v0[u]);
                    }
                }
                ring = ring + 1 == ROUNDS ? 0 : ring + 1;
                const float m = fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3]));
                if (__any(v0[0] < a.V && !(m < top.floor))) top.add4(x[0], v0[0], a.V);
#pragma unroll
                for (int u = 0; u + 1 < ROUNDS; ++u) {
                    v0[u] = v0[u + 1];
#pragma unroll
                    for (int q = 0; q < 4; ++q) x[u][q] = x[u + 1][q];
                }
            }
            i += step;
            top.take(o.top_k, lane, i < end || more ? 63 : 0);
            if (i >= end) break;
        }
        if (more) {
            b0 += BLOCK;
            continue;
        }
        // the token's first wavefront ends with all of its lists joined
#pragma unroll 1
        for (int d = 1; d < used; d *= 2) {
            __syncthreads();
            if ((sub & (2 * d - 1)) == d) lists[wave][lane] = top.entry;
            __syncthreads();
            if ((sub & (2 * d - 1)) == 0) top.merge(lists[wave + d][lane], lane);
        }
        if (logits) break;
        if (sub == 0) lists[wave][lane] = top.entry;
        finish_statistics();                     // (with a barrier in it)
        group = lists[wave - sub][lane];
        top = TopList(pending[TOP ? wave : 0]);
        logits = true;
        first = sub * per;
        end = groups < o.top_k ? groups : o.top_k;
        // the k-th largest maximum: k logits are no smaller
        if (end == o.top_k) top.at_least(lane_value(group, end - 1));
        used = 1;
        while (used < WPT && used * per * 2 < end) used *= 2;
        step = used * per;
    }
    __syncthreads();
    if (sub == 0 && my_n < cv.n_c) write_top(o, cv.n0 + my_n, fin[my_tok], top, lane);
}

// tau[n]: one wavefront per token lists the maxima of the leading groups, read with neighbouring tokens side by side.
constexpr int BOUND_TOK = 16, BOUND_BLOCK = 640;
__global__ __launch_bounds__(1024) void stats_bound_kernel(StatsPart part, int32_t groups, int32_t top_k, int32_t n_c, float* __restrict__ tau) {
    __shared__ float maxima[BOUND_BLOCK * (BOUND_TOK + 1)];
    __shared__ uint64_t pending[16][PENDING];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int tok = tid % BOUND_TOK, n = blockIdx.x * BOUND_TOK + tok, my_n = blockIdx.x * BOUND_TOK + wave;
    TopList top(pending[wave]);
    for (int g0 = 0; g0 < groups; g0 += BOUND_BLOCK) {
        const int g1 = groups - g0 < BOUND_BLOCK ? groups : g0 + BOUND_BLOCK;
        if (g0 > 0) __syncthreads();
        if (n < n_c) {
            for (int g = g0 + tid / BOUND_TOK; g < g1; g += 1024 / BOUND_TOK) maxima[(g - g0) * (BOUND_TOK + 1) + tok] = part.mx[part.at(g, n)];
        }
        __syncthreads();
        for (int i = g0; i < g1; i += 64) {
            top.add(i + lane < g1 && my_n < n_c ? top_key(maxima[(i + lane - g0) * (BOUND_TOK + 1) + wave], (uint32_t)(i + lane)) : 0);
            top.take(top_k, lane, i + 64 < groups ? 63 : 0);
        }
    }
    if (lane == 0 && my_n < n_c) tau[my_n] = top_value(lane_value(top.entry, top_k - 1));
}

// Row of H of chunk token n, clamped (what is wrong with it is reported elsewhere).
__device__ __forceinline__ int64_t token_row(const TokenArgs& a, ChunkView cv, int n) {
    const int64_t row = a.loss_pos ? (int64_t)a.loss_pos[cv.n0 + n] : cv.n0 + n;
    return row < 0 ? 0 : row >= a.T ? a.T - 1 : row;
}
// 64 tokens x 64 columns of the transpose through LDS, 16-byte accesses on both sides.
__device__ void transpose_tokens(const GatherRows& g, ChunkView cv, int block, uint16_t (*tile)[64 + 2]) {
    const int D = g.tokens.D, r0 = block / (D / 64) * 64, c0 = block % (D / 64) * 64;
    const int vec = threadIdx.x & 7, line = threadIdx.x >> 3;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
        const int rr = line + pass * 32, r = r0 + rr;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r < cv.n_c) v = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(g.tokens.H) + (size_t)token_row(g.tokens, cv, r) * D + c0 + vec * 8);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            tile[rr][vec * 8 + 2 * k] = (uint16_t)(w[k] & 0xffffu);
            tile[rr][vec * 8 + 2 * k + 1] = (uint16_t)(w[k] >> 16);
        }
    }
    __syncthreads();
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
        const int cc = line + pass * 32, drow = c0 + cc;
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = (uint32_t)tile[vec * 8 + 2 * k][cc] | ((uint32_t)tile[vec * 8 + 2 * k + 1][cc] << 16);
        static_assert(GEMM_B_BLOCK_K == 64, "a 64-column tile = one block column");
        const size_t off = (((size_t)(drow / g.transpose_block) * (g.transpose_cols / GEMM_B_BLOCK_K) + r0 / GEMM_B_BLOCK_K) * g.transpose_block +
                            drow % g.transpose_block) * GEMM_B_BLOCK_K + vec * 8;
        *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(g.transpose) + off) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
// Workgroup `block` of `blocks`. The first gather, a wavefront per row of the chunk: target and (clamped) row of H of the token, a copy of the row
// (16-byte vectors, zero beyond n_c) and its scale, bound by HBM; the next transpose; the last clear.
struct GatherBlocks { unsigned gather, transpose, all; };
__device__ __forceinline__ void gather_rows(const GatherRows& g, ChunkView cv, unsigned block, const GatherBlocks& blocks, uint16_t (*tile)[64 + 2]) {
    if (block >= blocks.gather + blocks.transpose) {
        // (clear is 4-byte aligned, the words in front of and behind the vectors one by one)
        uint32_t* p = reinterpret_cast<uint32_t*>(g.clear);
        const unsigned first = blocks.gather + blocks.transpose;
        const size_t words = g.clear_bytes / 4, head = (size_t)(-(reinterpret_cast<intptr_t>(p) / 4) & 3), lead = head < words ? head : words;
        const size_t vectors = (words - lead) / 4, i0 = (size_t)(block - first) * 256 + threadIdx.x;
        uint4* v = reinterpret_cast<uint4*>(p + lead);
        for (size_t i = i0; i < vectors; i += (size_t)(blocks.all - first) * 256) v[i] = make_uint4(0, 0, 0, 0);
        if (i0 < lead) p[i0] = 0;
        if (lead + vectors * 4 + i0 < words) p[lead + vectors * 4 + i0] = 0;
        return;
    }
    if (block >= blocks.gather) {
        transpose_tokens(g, cv, (int)(block - blocks.gather), tile);
        return;
    }
    const int n = (int)block * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (n >= cv.n_cp) return;
    const bool valid = n < cv.n_c;
    int64_t row = 0;
    int32_t t = 0;
    if (valid) {
        int flags = 0;
        if (g.tokens.ids) {
            flags = locate_token(g.tokens.ids, g.tokens.loss_pos, g.tokens.T, g.tokens.V, cv.n0 + n, row, t);
        } else {
            row = g.tokens.loss_pos ? (int64_t)g.tokens.loss_pos[cv.n0 + n] : cv.n0 + n;
            if (row < 0 || row >= g.tokens.T) flags = DPPO_HEAD_BAD_POSITION;
            row = row < 0 ? 0 : row >= g.tokens.T ? g.tokens.T - 1 : row;
            t = -1;
        }
        if (flags != 0 && g.tokens.status != nullptr && lane == 0) atomicOr(g.tokens.status, flags);
    }
    if (lane == 0) {
        if (g.y) g.y[n] = t;
        if (g.rowc) g.rowc[n] = (int32_t)row;
        if (g.scale_out) g.scale_out[n] = valid ? g.scale[row] : 0.0f;
    }
    if (!g.out) return;
    if (g.row_bytes % 16 != 0 || reinterpret_cast<uintptr_t>(g.tokens.H) % 16 != 0) {      // float32 rows of any length and alignment
        const float* src = reinterpret_cast<const float*>(reinterpret_cast<const char*>(g.tokens.H) + (size_t)row * g.row_bytes);
        float* dst = reinterpret_cast<float*>(reinterpret_cast<char*>(g.out) + (size_t)n * g.row_bytes);
        for (int d = lane; d < (int)(g.row_bytes / 4); d += 64) dst[d] = valid ? src[d] : 0.0f;
        return;
    }
    const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(g.tokens.H) + (size_t)row * g.row_bytes);
    uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<char*>(g.out) + (size_t)n * g.row_bytes);
    constexpr int U = 8;
    const int vectors = (int)(g.row_bytes / 16);
    for (int c0 = lane; c0 < vectors; c0 += 64 * U) {
        uint4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * 64;
            x[u] = valid && c < vectors ? src[c] : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (c0 + u * 64 < vectors) dst[c0 + u * 64] = x[u];
    }
}

__global__ __launch_bounds__(256) void stats_gather_kernel(GatherRows g, ChunkView cv, GatherBlocks blocks) {
    __shared__ uint16_t tile[64][64 + 2];
    gather_rows(g, cv, blockIdx.x, blocks, tile);
}

// Gradient entries of the float32 path, in place over the stored logits: dz = p (c - g_ent (z - lse)) with
// c = g_lse - g_logp - g_ent entropy, the target's g_logp (1 - p) + p (g_lse - g_ent (z - lse + entropy)); 0 for V <= v < Vp. `parts` workgroups a
// token; those behind them gather what the two GEMMs after this need (a launch of its own costs the host 3 us).
__global__ __launch_bounds__(256) void stats_grad_kernel(float* __restrict__ ZG, int32_t V, int32_t Vp, StatsGrad g, ChunkView cv, unsigned parts,
                                                         GatherRows rows, GatherBlocks blocks) {
    const unsigned entries = (unsigned)cv.n_c * parts;
    if (blockIdx.x >= entries) {
        gather_rows(rows, cv, blockIdx.x - entries, blocks, nullptr);
        return;
    }
    const int n = (int)(blockIdx.x / parts), part = (int)(blockIdx.x % parts);
    const TokenGrad t = load_grad(g, cv.n0 + n);
    int32_t target = -1;
    if (rows.tokens.ids) {
        int64_t row;
        locate_token(rows.tokens.ids, rows.tokens.loss_pos, rows.tokens.T, rows.tokens.V, cv.n0 + n, row, target);
    }
    float4* z4 = reinterpret_cast<float4*>(ZG + (size_t)n * Vp);
    for (int i = part * 256 + threadIdx.x; i < Vp / 4; i += parts * 256) {
        const float4 z = z4[i];
        const float zz[4] = {z.x, z.y, z.z, z.w};
        float d[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int v = i * 4 + q;
            const float lp = zz[q] - t.lse;
            d[q] = v < V ? grad_entry(t, lp, expf(lp), v == target) : 0.0f;
        }
        z4[i] = make_float4(d[0], d[1], d[2], d[3]);
    }
}

__global__ __launch_bounds__(256) void to_bf16_kernel(const float4* __restrict__ src, uint2* __restrict__ dst, size_t vectors) {
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < vectors; i += (size_t)gridDim.x * 256) {
        const float4 v = src[i];
        const __bf16 b0 = (__bf16)v.x, b1 = (__bf16)v.y, b2 = (__bf16)v.z, b3 = (__bf16)v.w;
        const uint32_t lo = (uint32_t)__builtin_bit_cast(uint16_t, b0) | ((uint32_t)__builtin_bit_cast(uint16_t, b1) << 16);
        const uint32_t hi = (uint32_t)__builtin_bit_cast(uint16_t, b2) | ((uint32_t)__builtin_bit_cast(uint16_t, b3) << 16);
        dst[i] = make_uint2(lo, hi);
    }
}

}  // namespace

int stats_row_parts(int32_t n_c, int32_t V, int cus) {
    // enough workgroups for every compute unit to have four, none with fewer than 2048 logits
    const int64_t want = ceil_div((int64_t)4 * cus, n_c), most = V / 2048;
    return (int)(want < most ? want : most < 1 ? 1 : most);
}

void launch_stats_rows(const float* Z, int64_t ldz, const TokenArgs& a, const StatsOut& o, ChunkView cv, PartialStats partial, hipStream_t st) {
    const dim3 grid((unsigned)cv.n_c, (unsigned)partial.parts);
    const bool top = o.top_k > 0;
    if (top) stats_rows_kernel<true><<<grid, ROWS_THREADS, 0, st>>>(Z, ldz, a, o, cv, partial);
    else stats_rows_kernel<false><<<grid, ROWS_THREADS, 0, st>>>(Z, ldz, a, o, cv, partial);
    if (partial.parts == 1) return;
    if (top) join_parts_kernel<true><<<(unsigned)cv.n_c, 64, 0, st>>>(Z, ldz, a, o, cv, partial);
    else join_parts_kernel<false><<<(unsigned)cv.n_c, 64, 0, st>>>(Z, ldz, a, o, cv, partial);
}

void launch_stats_join(const StatsPart& part, int rows, const float* Z, int64_t ldz, const TokenArgs& a, bool look_up,
                       const StatsOut& o, ChunkView cv, hipStream_t st) {
    auto go = [&](auto tok) {
        constexpr int TOK = decltype(tok)::value;
        const unsigned blocks = (unsigned)ceil_div(cv.n_c, TOK);
        if (o.top_k > 0) stats_join_kernel<TOK, true><<<blocks, JOIN_THREADS, 0, st>>>(part, rows, Z, ldz, a, look_up, o, cv);
        else stats_join_kernel<TOK, false><<<blocks, JOIN_THREADS, 0, st>>>(part, rows, Z, ldz, a, look_up, o, cv);
    };
    switch (join_tokens(cv.n_c)) {
        case 1: go(std::integral_constant<int, 1>{}); break;
        case 4: go(std::integral_constant<int, 4>{}); break;
        case 8: go(std::integral_constant<int, 8>{}); break;
        default: go(std::integral_constant<int, 16>{});
    }
}

void launch_stats_bound(const StatsPart& part, int32_t groups, int32_t top_k, ChunkView cv, float* tau, hipStream_t st) {
    stats_bound_kernel<<<(unsigned)ceil_div(cv.n_c, BOUND_TOK), 1024, 0, st>>>(part, groups, top_k, cv.n_c, tau);
}

static GatherBlocks gather_blocks(const GatherRows& g, ChunkView cv) {
    GatherBlocks b;
    b.gather = (unsigned)ceil_div(cv.n_cp, 4);
    b.transpose = g.transpose ? (unsigned)(g.tokens.D / 64 * (g.transpose_cols / 64)) : 0;
    const int64_t fill = ceil_div((int64_t)g.clear_bytes, 16 * 256 * 4);
    b.all = b.gather + b.transpose + (unsigned)(fill < 4096 ? fill : 4096);
    return b;
}

void launch_stats_gather(const GatherRows& g, ChunkView cv, hipStream_t st) {
    const GatherBlocks b = gather_blocks(g, cv);
    stats_gather_kernel<<<b.all, 256, 0, st>>>(g, cv, b);
}

void launch_stats_grad_f32(float* ZG, int32_t Vp, const StatsGrad& g, const GatherRows& rows, ChunkView cv, hipStream_t st) {
    const GatherBlocks b = gather_blocks(rows, cv);
    int parts = (int)ceil_div(Vp / 4, 256);
    if (parts > 64) parts = 64;
    stats_grad_kernel<<<(unsigned)cv.n_c * (unsigned)parts + b.all, 256, 0, st>>>(ZG, rows.tokens.V, Vp, g, cv, (unsigned)parts, rows, b);
}

void launch_to_bf16(const float* src, void* dst, size_t n, hipStream_t st) {
    const size_t vectors = n / 4;
    size_t blocks = (vectors + 255) / 256;
    if (blocks > 16384) blocks = 16384;
    if (blocks == 0) return;
    to_bf16_kernel<<<(unsigned)blocks, 256, 0, st>>>(reinterpret_cast<const float4*>(src), reinterpret_cast<uint2*>(dst), vectors);
}

}  // namespace dppo
