// Kernels around the logits GEMMs of dppo_token_stats and dppo_token_stats_bwd: softmax statistics and top alternatives of stored
// logits, gathering of rows, gradient entries of the float32 path.
#include "stats_internal.h"
#include "top_list.h"
#include "token_rows.h"

namespace dppo {
namespace {

// Statistics of a set of logits against its maximum m: sum = sum exp(z - m), dev = sum (z - m) exp(z - m). With them
// lse = m + log(sum) and the entropy -sum p log p = log(sum) - dev / sum, in which nothing of the size of the logits cancels.
struct Stats { float m, sum, dev; };

// exp() is 0 in 32 bits below -104: differences are cut at -150 where they are multiplied by it, so that a logit at -infinity (or
// at the type's lowest value, whose difference overflows) adds 0 and not 0 * infinity.
constexpr float DEV_MIN = -150.0f;

__device__ __forceinline__ Stats no_stats() { return Stats{-__builtin_inff(), 0.0f, 0.0f}; }
__device__ __forceinline__ Stats join(const Stats& a, const Stats& b) {
    const float m = fmaxf(a.m, b.m), ref = m == -__builtin_inff() ? 0.0f : m;
    const float da = a.m - ref, db = b.m - ref, ea = expf(da), eb = expf(db);
    return Stats{m, a.sum * ea + b.sum * eb,
                 ea * (a.dev + fmaxf(da, DEV_MIN) * a.sum) + eb * (b.dev + fmaxf(db, DEV_MIN) * b.sum)};
}
__device__ __forceinline__ Stats join_lanes(Stats s) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1)
        s = join(s, Stats{__shfl_xor(s.m, off, 64), __shfl_xor(s.sum, off, 64), __shfl_xor(s.dev, off, 64)});
    return s;
}

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

// One workgroup per token and part of its row of stored logits (pitch a multiple of 256; columns from V on hold anything): one pass
// over the logits, which are bound by HBM or L2, 4 bytes each. Each wavefront keeps statistics per lane and one list of the
// top_k largest; a logit below the list's last entry costs a comparison of four logits' maximum. parts > 1 (few tokens): the
// workgroup's results go to `partial`, and join_parts_kernel puts the parts together.
constexpr int ROWS_THREADS = 256, ROWS_WAVES = ROWS_THREADS / 64, ROWS_UNROLL = 4;
template <bool TOP>
__global__ __launch_bounds__(ROWS_THREADS) void stats_rows_kernel(const float* __restrict__ Z, int64_t ldz, TokenArgs a, StatsOut o,
                                                                  ChunkView cv, PartialStats partial) {
    __shared__ Stats red[ROWS_WAVES];
    __shared__ uint64_t lists[ROWS_WAVES][TOP_MAX];
    const int n = blockIdx.x, part = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float NONE = -__builtin_inff();
    const float* z = Z + (size_t)n * ldz;
    const int vectors = (a.V + 3) / 4;
    const int lo = (int)((int64_t)vectors * part / partial.parts), hi = (int)((int64_t)vectors * (part + 1) / partial.parts);
    Stats s = no_stats();
    TopList top;
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
                const float d = x[u][q] - ref, e = expf(d);
                b.sum += e;
                b.dev = fmaf(fmaxf(d, DEV_MIN), e, b.dev);
            }
        s = join(s, b);
        if (TOP) {
#pragma unroll
            for (int u = 0; u < ROWS_UNROLL; ++u) {
                if (!__any(!(m4[u] < top.floor))) continue;
                const int i = i0 + u * ROWS_THREADS + lane;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    top.offer(i < hi && i * 4 + q < a.V ? top_key(x[u][q], (uint32_t)(i * 4 + q)) : 0, o.top_k);
            }
        }
    }
    s = join_lanes(s);
    if (lane == 0) red[wave] = s;
    if (TOP) lists[wave][lane] = top.entry;
    __syncthreads();
    if (wave != 0) return;
    for (int w = 1; w < ROWS_WAVES; ++w) s = join(s, red[w]);
    if (TOP) {
        for (int w = 1; w < ROWS_WAVES; ++w) top.offer(lists[w][lane], o.top_k);
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
        const int flags = locate_token(a.ids, a.loss_pos, a.T, a.V, gi, row, target);
        if (flags != 0 && a.status != nullptr && lane == 0) atomicOr(a.status, flags);
        zy = z[target];
    } else if (a.loss_pos && a.status != nullptr && lane == 0) {
        const int64_t row = a.loss_pos[gi];
        if (row < 0 || row >= a.T) atomicOr(a.status, DPPO_HEAD_BAD_POSITION);
    }
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
    s = join_lanes(s);
    TopList top;
    if (TOP) {
        const int entries = partial.parts * o.top_k;
        for (int i = 0; i < entries; i += 64) top.offer(i + lane < entries ? partial.keys[at * o.top_k + i + lane] : 0, o.top_k);
    }
    const int64_t gi = cv.n0 + n;
    float zy = 0.0f;
    if (a.ids) {
        int64_t row;
        int32_t target;
        const int flags = locate_token(a.ids, a.loss_pos, a.T, a.V, gi, row, target);
        if (flags != 0 && a.status != nullptr && lane == 0) atomicOr(a.status, flags);
        zy = Z[(size_t)n * ldz + target];
    } else if (a.loss_pos && a.status != nullptr && lane == 0) {
        const int64_t row = a.loss_pos[gi];
        if (row < 0 || row >= a.T) atomicOr(a.status, DPPO_HEAD_BAD_POSITION);
    }
    if (lane == 0) write_token(o, gi, s, zy);
    if (TOP) write_top(o, gi, s, top, lane);
}

// A wavefront per row of the chunk: target and (clamped) row of H of the token, a copy of the row (16-byte vectors, zero beyond
// n_c) and its scale. Bound by HBM.
__global__ __launch_bounds__(256) void stats_gather_kernel(GatherRows g, ChunkView cv) {
    const int n = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
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

// Gradient entries of the float32 path, in place over the stored logits: dz = p (c - g_ent (z - lse)) with
// c = g_lse - g_logp - g_ent entropy, the target's g_logp (1 - p) + p (g_lse - g_ent (z - lse + entropy)); 0 for V <= v < Vp.
__global__ __launch_bounds__(256) void stats_grad_kernel(float* __restrict__ ZG, int32_t V, int32_t Vp, const int32_t* __restrict__ y,
                                                         StatsGrad g, ChunkView cv) {
    const int n = blockIdx.x;
    const TokenGrad t = load_grad(g, cv.n0 + n);
    const int target = y[n];
    float4* row = reinterpret_cast<float4*>(ZG + (size_t)n * Vp);
    for (int i = blockIdx.y * 256 + threadIdx.x; i < Vp / 4; i += gridDim.y * 256) {
        const float4 z = row[i];
        const float zz[4] = {z.x, z.y, z.z, z.w};
        float d[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int v = i * 4 + q;
            const float lp = zz[q] - t.lse;
            d[q] = v < V ? grad_entry(t, lp, expf(lp), v == target) : 0.0f;
        }
        row[i] = make_float4(d[0], d[1], d[2], d[3]);
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

void launch_stats_gather(const GatherRows& g, ChunkView cv, hipStream_t st) {
    stats_gather_kernel<<<(unsigned)ceil_div(cv.n_cp, 4), 256, 0, st>>>(g, cv);
}

void launch_stats_grad_f32(float* ZG, int32_t V, int32_t Vp, const int32_t* y, const StatsGrad& g, ChunkView cv, hipStream_t st) {
    int by = (int)ceil_div(Vp / 4, 256);
    if (by > 64) by = 64;
    stats_grad_kernel<<<dim3((unsigned)cv.n_c, (unsigned)by), 256, 0, st>>>(ZG, V, Vp, y, g, cv);
}

void launch_to_bf16(const float* src, void* dst, size_t n, hipStream_t st) {
    const size_t vectors = n / 4;
    size_t blocks = (vectors + 255) / 256;
    if (blocks > 16384) blocks = 16384;
    if (blocks == 0) return;
    to_bf16_kernel<<<(unsigned)blocks, 256, 0, st>>>(reinterpret_cast<const float4*>(src), reinterpret_cast<uint2*>(dst), vectors);
}

}  // namespace dppo
