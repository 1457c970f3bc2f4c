// Rows brought to 8 bits with one scale each: scale = max|x| * (1 / 127), q = x / scale rounded to the nearest integer (ties to even).
#include "stats_internal.h"

namespace dppo {
namespace {

// One wavefront per row, which it reads twice: the second time from its registers (rows of up to 64 * U vectors of 8) or from L2.
// Bound by HBM: read once, written once at half (a quarter) of the size.
__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        x[2 * k] = __uint_as_float(w[k] << 16);
        x[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ float load1(const float* p) { return *p; }

template <class E>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const E* __restrict__ X, int64_t rows, int32_t D, int8_t* __restrict__ Q,
                                                            int64_t pitch, float* __restrict__ scale_out, int vec) {
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (r >= rows) return;
    const E* x = X + (size_t)r * D;
    int8_t* q = Q + (size_t)r * pitch;
    const int groups = (int)(pitch / 8);
    auto load = [&](int g, float (&v)[8]) {
        if (vec && g * 8 + 8 <= D) { load8(x + g * 8, v); return; }
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = g * 8 + k < D ? load1(x + g * 8 + k) : 0.0f;
    };
    // |x| as an integer orders like |x|, with infinity and NaN on top
    uint32_t top = 0;
    for (int g = lane; g < groups; g += 64) {
        float v[8];
        load(g, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t b = __float_as_uint(v[k]) & 0x7fffffffu;
            top = b > top ? b : top;
        }
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)top, off, 64);
        top = o > top ? o : top;
    }
    const bool finite = top < 0x7f800000u;
    const float scale = __uint_as_float(top) * (1.0f / 127.0f);
    // (a scale of 0: every value is 0, or too small for a quotient to be stored)
    const bool some = finite && scale > 0.0f;
    if (lane == 0) scale_out[r] = finite ? scale : __builtin_nanf("");
    for (int g = lane; g < groups; g += 64) {
        float v[8];
        load(g, v);
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float t = fminf(fmaxf(rintf(__fdiv_rn(v[k], scale)), -127.0f), 127.0f);
            const int i = some ? (int)t : 0;
            w[k / 4] |= ((uint32_t)i & 0xffu) << (8 * (k % 4));
        }
        *reinterpret_cast<uint2*>(q + g * 8) = make_uint2(w[0], w[1]);
    }
}

}  // namespace

void launch_quantize_rows(int dtype, const void* X, int64_t rows, int32_t D, int8_t* q, int64_t pitch, float* scale, hipStream_t st) {
    const unsigned blocks = (unsigned)ceil_div(rows, 4);
    const int vec = (size_t)D * (dtype == 1 ? 2 : 4) % 16 == 0 && reinterpret_cast<uintptr_t>(X) % 16 == 0;
    if (dtype == 1) quantize_rows_kernel<uint16_t><<<blocks, 256, 0, st>>>(reinterpret_cast<const uint16_t*>(X), rows, D, q, pitch, scale, vec);
    else quantize_rows_kernel<float><<<blocks, 256, 0, st>>>(reinterpret_cast<const float*>(X), rows, D, q, pitch, scale, vec);
}

}  // namespace dppo
