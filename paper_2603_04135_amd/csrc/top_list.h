// The k largest (value, index) pairs of a stream, held by one wavefront: entry i, in descending order, in lane i.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dppo {

constexpr int TOP_MAX = 64;     // one entry per lane

// One whole number per logit that orders like the logit and, among equal ones, like the lower index: the float's bits made
// monotone in the high word, the index's complement in the low one. -0 counts as +0; NaN ranks below everything (high word 1);
// 0 stands for "no entry".
__device__ __forceinline__ uint64_t top_key(float z, uint32_t index) {
    const uint32_t b = __float_as_uint(z + 0.0f);
    const uint32_t o = (b >> 31) ? ~b : b | 0x80000000u;
    return ((uint64_t)(z == z ? o : 1u) << 32) | (uint32_t)~index;
}
__device__ __forceinline__ uint32_t top_index(uint64_t key) { return ~(uint32_t)key; }
__device__ __forceinline__ float top_value(uint64_t key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return o <= 1u ? __builtin_nanf("") : __uint_as_float((o >> 31) ? o & 0x7fffffffu : ~o);
}

__device__ __forceinline__ uint64_t lane_value(uint64_t v, int lane) {
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)v, lane), hi = __builtin_amdgcn_readlane((uint32_t)(v >> 32), lane);
    return ((uint64_t)hi << 32) | lo;
}

struct TopList {
    uint64_t entry = 0;       // this lane's
    uint64_t least = 0;       // entry k - 1: what a newcomer has to exceed
    float floor = -__builtin_inff();   // the same as a logit: a lower one need not be looked at (-infinity while there are not k)

    // All lanes: lane l's key joins the list if it exceeds `least`.
    __device__ __forceinline__ void offer(uint64_t key, int k) {
        uint64_t hits = __ballot(key > least);
        if (hits == 0) return;
        do {
            const int l = __builtin_ctzll(hits);
            hits &= hits - 1;
            insert(lane_value(key, l));
        } while (hits);
        settle(k);
    }
    // A sorted insertion: whoever is smaller moves one lane up.
    __device__ __forceinline__ void insert(uint64_t key) {
        // wave_shr:1, lane 0 receives all ones
        const uint32_t lo = __builtin_amdgcn_update_dpp(0xffffffffu, (uint32_t)entry, 0x138, 0xf, 0xf, false);
        const uint32_t hi = __builtin_amdgcn_update_dpp(0xffffffffu, (uint32_t)(entry >> 32), 0x138, 0xf, 0xf, false);
        const uint64_t before = ((uint64_t)hi << 32) | lo;
        entry = entry > key ? entry : before > key ? key : before;
    }
    __device__ __forceinline__ void settle(int k) {
        least = lane_value(entry, k - 1);
        floor = (uint32_t)(least >> 32) <= 1u ? -__builtin_inff() : top_value(least);
    }
};

}  // namespace dppo
