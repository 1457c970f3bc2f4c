// The k largest (value, index) pairs of a stream, held by one wavefront: entry i, in descending order, in lane i.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lanes.h"

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
constexpr uint32_t MINUS_INFINITY = 0x007fffffu;       // high word of -infinity's key
__device__ __forceinline__ uint32_t top_index(uint64_t key) { return ~(uint32_t)key; }
__device__ __forceinline__ float top_value(uint64_t key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return o <= 1u ? __builtin_nanf("") : __uint_as_float((o >> 31) ? o & 0x7fffffffu : ~o);
}

__device__ __forceinline__ uint64_t lane_value(uint64_t v, int lane) {
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)v, lane), hi = __builtin_amdgcn_readlane((uint32_t)(v >> 32), lane);
    return ((uint64_t)hi << 32) | lo;
}

// Of a pair of lanes X apart, the one with the lower number (bit BIT clear) keeps the larger key.
template <int X, int BIT>
__device__ __forceinline__ uint64_t exchange(uint64_t v, int lane) {
    const uint64_t o = xor_lane<X>(v);
    return ((lane & BIT) == 0) == (o > v) ? o : v;
}
// A sequence that falls and then rises (or is such a one's rotation) in descending order: 2 N lanes, N the first distance.
template <int N>
__device__ __forceinline__ uint64_t settle_bitonic(uint64_t v, int lane) {
    v = exchange<N, N>(v, lane);
    if constexpr (N > 1) v = settle_bitonic<N / 2>(v, lane);
    return v;
}
// 64 keys in descending order: sorted runs of N are mirrored against each other to runs of 2 N.
template <int N = 1>
__device__ __forceinline__ uint64_t sort_lanes(uint64_t v, int lane) {
    v = exchange<2 * N - 1, N>(v, lane);
    if constexpr (N > 1) v = settle_bitonic<N / 2>(v, lane);
    if constexpr (N < 32) v = sort_lanes<2 * N>(v, lane);
    return v;
}

// The k-th largest of the lanes' logits (NaN: the lane has none): a bound that k logits reach.
__device__ __forceinline__ uint64_t kth_of_lanes(float z, int k, int lane) {
    return lane_value(sort_lanes(top_key(z, 0) >> 32, lane), k - 1) << 32;
}

// Newcomers that beat the list's last entry gather in LDS (`pending`, of this wavefront) and are sorted and merged by 64, and what is left at
// the end: some 10 instructions for 64 on offer and 250 a merge, against 20 for each that is inserted by itself.
constexpr int PENDING = 128, PENDING4 = 320;     // keys of a buffer: up to 63 that wait, and one or four new ones a lane
struct TopList {
    uint64_t* pending;
    int waiting = 0;
    uint64_t entry = 0;       // this lane's
    uint64_t least = 0;       // entry k - 1 (or a bound below it that is known from elsewhere): what a newcomer has to exceed
    float floor = -__builtin_inff();   // the same as a logit: a lower one need not be looked at (-infinity while there are not k)

    __device__ __forceinline__ explicit TopList(uint64_t* lds) : pending(lds) {}
    // All lanes: lane l's key waits if it exceeds `least`.
    __device__ __forceinline__ void add(uint64_t key) {
        const bool hit = key > least;
        const uint64_t hits = __ballot(hit);
        if (hits == 0) return;
        if (hit) pending[waiting + __builtin_amdgcn_mbcnt_hi((uint32_t)(hits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hits, 0))] = key;
        waiting += __builtin_popcountll(hits);
    }
    // Takes in those that wait, 64 at a time, until no more than `keep` are left.
    __device__ __forceinline__ void take(int k, int lane, int keep) {
#pragma unroll 1
        while (waiting > keep) {
            const int n = waiting < 64 ? waiting : 64;
            waiting -= n;
            // (the wavefront's own LDS accesses stay in order; the compiler has to leave them so)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const uint64_t key = lane < n ? pending[waiting + lane] : 0;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            merge(sort_lanes(key, lane), lane);
            settle(k);
        }
    }
    // The lane's logits x[0 .. 3] of indices v to v + 3, those below V.
    __device__ __forceinline__ void add4(const float (&x)[4], int v, int V) {
#pragma unroll
        for (int q = 0; q < 4; ++q) add(v + q < V ? top_key(x[q], (uint32_t)(v + q)) : 0);
    }
    // Joins keys in descending order: the larger of each mirrored pair are the 64 largest, in bitonic order.
    __device__ __forceinline__ void merge(uint64_t sorted, int lane) {
        const uint64_t o = xor_lane<63>(sorted);
        entry = settle_bitonic<32>(entry > o ? entry : o, lane);
    }
    __device__ __forceinline__ void settle(int k) {
        const uint64_t last = lane_value(entry, k - 1);
        least = last > least ? last : least;
        floor = (uint32_t)(least >> 32) <= 1u ? -__builtin_inff() : top_value(least);
    }
    // Only keys whose value is at least `key`'s will be wanted: k of those on offer reach it. (A bound of -infinity shuts out nothing: it
    // may be the maximum of a group of NaN.)
    __device__ __forceinline__ void at_least(uint64_t key) {
        if ((uint32_t)(key >> 32) <= MINUS_INFINITY) return;
        least = (key >> 32 << 32) - 1;
        floor = top_value(key);
    }
};

}  // namespace dppo
