// Rows brought to 8 bits with one scale each: scale = max|x| * (1 / 127), q = x / scale rounded to the nearest integer (ties to even).
#include <type_traits>

#include "stats_internal.h"

namespace dppo {
namespace {

// Eight neighbouring elements of a row: one or two loads of 16 bytes, aligned or not (rows of any length follow each other).
struct __attribute__((packed, aligned(2))) Raw16 { uint32_t w[4]; };
struct __attribute__((packed, aligned(4))) Raw32 { float w[8]; };
__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
    const Raw16 v = *reinterpret_cast<const Raw16*>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        x[2 * k] = __uint_as_float(v.w[k] << 16);
        x[2 * k + 1] = __uint_as_float(v.w[k] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
    const Raw32 v = *reinterpret_cast<const Raw32*>(p);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = v.w[k];
}
__device__ __forceinline__ float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ float load1(const float* p) { return *p; }

// Eight quotients as bytes. x * (1 / scale) is within 2^-22 of the correctly rounded quotient's value, relative (2 roundings against 1, of
// values up to 127: 4e-5): where no product comes that near to the middle between two integers, both round to the same integer,
// and adding 1.5 * 2^23 does it, to even. The others (one product in 5000) and scales whose reciprocal is no ordinary number take the
// division.
constexpr float ROUND_MAGIC = 12582912.0f, MIDDLE = 0.4999f;
__device__ __forceinline__ uint2 quantize8(const float (&x)[8], float scale, float inverse, bool divide) {
    uint32_t bits[8];
    float off = divide ? 1.0f : 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float t = x[k] * inverse, m = t + ROUND_MAGIC;
        bits[k] = __float_as_uint(m);
        off = fmaxf(off, fabsf(t - (m - ROUND_MAGIC)));
    }
    if (!(off < MIDDLE)) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            bits[k] = (uint32_t)(int)fminf(fmaxf(rintf(__fdiv_rn(x[k], scale)), -127.0f), 127.0f);
    }
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        // byte 0 of each: v_perm_b32 takes bytes 0 to 3 from its second operand, 4 to 7 from its first
        const uint32_t lo = __builtin_amdgcn_perm(bits[4 * h + 1], bits[4 * h], 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(bits[4 * h + 3], bits[4 * h + 2], 0x04000c0cu);
        w[h] = lo | hi;
    }
    return make_uint2(w[0], w[1]);
}

// WPR wavefronts per row. Rows of up to 512 NV WPR elements stay in the registers between the two looks at them (all loads in flight at once),
// longer ones (NV 0) are read again from L2. Bound by HBM: read once, written once at half (a quarter) of the size.
template <class E, int NV, int WPR>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const E* __restrict__ X, int64_t rows, int32_t D, int8_t* __restrict__ Q,
                                                            int64_t pitch, float* __restrict__ scale_out) {
    __shared__ uint32_t tops[WPR];
    const int wave = threadIdx.x >> 6, lane = (WPR > 1 ? wave * 64 : 0) + (threadIdx.x & 63);      // of the row's lanes
    const int64_t r = WPR > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
    if (r >= rows) return;
    constexpr int LANES = 64 * WPR;
    const E* x = X + (size_t)r * D;
    int8_t* q = Q + (size_t)r * pitch;
    const int groups = (int)(pitch / 8);
    auto load = [&](int g, float (&v)[8]) __attribute__((always_inline)) {
        if (g * 8 + 8 <= D) { load8(x + g * 8, v); return; }
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = g * 8 + k < D ? load1(x + g * 8 + k) : 0.0f;
    };
    // |x| as an integer orders like |x|, with infinity and NaN on top
    uint32_t top = 0;
    auto look = [&](const float (&v)[8]) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t b = __float_as_uint(v[k]) & 0x7fffffffu;
            top = b > top ? b : top;
        }
    };
    float v[NV > 0 ? NV : 1][8];
    if constexpr (NV > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int g = i * LANES + lane;
            if (g < groups) {
                load(g, v[i]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[i][k] = 0.0f;
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) look(v[i]);
    } else {
        for (int g = lane; g < groups; g += LANES) {
            load(g, v[0]);
            look(v[0]);
        }
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)top, off, 64);
        top = o > top ? o : top;
    }
    if constexpr (WPR > 1) {
        if ((threadIdx.x & 63) == 0) tops[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WPR; ++w) top = tops[w] > top ? tops[w] : top;
    }
    const bool finite = top < 0x7f800000u;
    const float scale = __uint_as_float(top) * (1.0f / 127.0f);
    // (a scale of 0: every value is 0, or too small for a quotient to be stored)
    const bool some = finite && scale > 0.0f;
    const bool divide = !(scale > 0x1p-120f && scale < 0x1p120f);
    const float inverse = divide ? 0.0f : __fdiv_rn(1.0f, scale);
    if (lane == 0) scale_out[r] = finite ? scale : __builtin_nanf("");
    auto store = [&](int g, const float (&x8)[8]) __attribute__((always_inline)) {
        const uint2 w = some ? quantize8(x8, scale, inverse, divide) : make_uint2(0, 0);
        *reinterpret_cast<uint2*>(q + g * 8) = w;
    };
    if constexpr (NV > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * LANES + lane < groups) store(i * LANES + lane, v[i]);
    } else {
        for (int g = lane; g < groups; g += LANES) {
            load(g, v[0]);
            store(g, v[0]);
        }
    }
}

constexpr int64_t FEW_ROWS = 2048, MANY_ROWS = 16384;
template <class E>
void launch(const E* X, int64_t rows, int32_t D, int8_t* q, int64_t pitch, float* scale, hipStream_t st) {
    auto go = [&](auto nv, auto wpr) {
        constexpr int WPR = decltype(wpr)::value;
        // (a launch of 2^32 threads or more runs what is left of their number in 32 bits, and reports nothing)
        constexpr int64_t MOST = (int64_t)(1 << 23) * (4 / WPR);
        for (int64_t r0 = 0; r0 < rows; r0 += MOST) {
            const int64_t n = rows - r0 < MOST ? rows - r0 : MOST;
            quantize_rows_kernel<E, decltype(nv)::value, WPR><<<(unsigned)ceil_div(n, 4 / WPR), 256, 0, st>>>(
                X + (size_t)r0 * D, n, D, q + (size_t)r0 * pitch, pitch, scale + r0);
        }
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 4> four;
    // A workgroup per row, its loads and divisions in a quarter of the time, where rows are long or few. us, a wavefront / a workgroup per row,
    // bfloat16: D = 4096, 1024 rows 6.8 / 4.9, 4096 14.0 / 11.8, 151936 332 / 314; 3200, 151936 282 / 275; 2560, 1024 5.0 / 4.0, 8192 16.3 / 14.6,
    // 32768 42.9 / 44.1, 151936 215 / 243; 2048, 2048 5.5 / 5.1, 4096 7.4 / 8.0; 1024, 2048 4.0 / 4.0, 4096 4.9 / 6.0. Many long rows
    // of bfloat16 that begin off 16-byte addresses stay with a wavefront each: 3001, 8192 19.7 / 17.3, 16384 31.0 / 29.6, 32768 66 / 71, 151936 277 / 314;
    // 4095, 16384 45 / 43, 151936 453 / 481. float32: 4096, 4096 15.6 / 13.5, 151936 547 / 538; 4095, 151936 582 / 539; 2048, 2048 5.2 / 5.2, 4096 7.6 / 8.7.
    const bool many = sizeof(E) == 2 && D % 8 != 0 && rows > MANY_ROWS;
    if ((rows <= FEW_ROWS && pitch > 512) || (pitch > 2560 && !many) || pitch > 4096) {
        if (pitch <= 2048) go(std::integral_constant<int, 1>{}, four);
        else if (pitch <= 4096) go(std::integral_constant<int, 2>{}, four);
        else if (pitch <= 8192) go(std::integral_constant<int, 4>{}, four);
        else if (pitch <= 16384) go(std::integral_constant<int, 8>{}, four);
        else go(std::integral_constant<int, 0>{}, four);
    } else if (pitch <= 512) go(std::integral_constant<int, 1>{}, one);
    else if (pitch <= 1024) go(std::integral_constant<int, 2>{}, one);
    else if (pitch <= 2048) go(std::integral_constant<int, 4>{}, one);
    else if (pitch <= 2560) go(std::integral_constant<int, 5>{}, one);     // (with registers for 4096 elements 151936 rows of 2176 take 207 us, not 174)
    else go(std::integral_constant<int, 8>{}, one);
}

}  // namespace

void launch_quantize_rows(int dtype, const void* X, int64_t rows, int32_t D, int8_t* q, int64_t pitch, float* scale, hipStream_t st) {
    if (dtype == 1) launch(reinterpret_cast<const uint16_t*>(X), rows, D, q, pitch, scale, st);
    else launch(reinterpret_cast<const float*>(X), rows, D, q, pitch, scale, st);
}

}  // namespace dppo
