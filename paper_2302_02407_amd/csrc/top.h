// Selecting a row's largest elements: places in their order, what a work group sets aside, and a way for any row.
#ifndef HE_TOP_H
#define HE_TOP_H

#include "plain.h"

// Ordered like the numbers: NaN above infinity, -0 with +0
__device__ __forceinline__ uint32_t order_key(float z) {
    const uint32_t b = __builtin_bit_cast(uint32_t, z == 0.0f ? 0.0f : z);
    return z != z ? 0xffffffffu : b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float value_of(uint32_t key) {
    return key == 0xffffffffu ? NAN : __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
__device__ __forceinline__ u64 place_of(float z, uint32_t i) { return (u64)order_key(z) << 32 | (uint32_t)~i; }

// An element's place in the order is one number of 64 bits, its key above the complement of its index, all different.

template <int THREADS, int ROOM_ = THREADS == 1024 ? 1024 : THREADS == 64 ? 64 : 512> struct TopShared {
    static constexpr int ROOM = ROOM_, KEEP = 512;
    uint4 aside[ROOM];                         // 16 bytes of the row each, and which
    uint32_t which[ROOM];                      // index of the first of its elements, and above 24 bits how many are another's
    u64 keep[KEEP], more, last;                // last: the k-th place
    uint32_t bins[256];
    int32_t tw[2][THREADS / 64];
    float room[THREADS / 64];
    uint32_t digit, left, got, kept;
};

// A value that at least r * full of the work group's lanes have reached: of every wavefront below `full` the r-th largest of its lanes' `high`, and of these
// the smallest; -infinity for r above 64.  tw: a slot a wavefront.  A barrier.
template <int WAVES> __device__ __forceinline__ float reached_by_all(float high, uint32_t r, uint32_t full, uint32_t lane, uint32_t wave, int32_t* tw) {
    int32_t w = ordered(high), best = INT32_MIN;
    if (r <= 64)
        for (uint32_t i = 0; i < r; i++) {
            best = wave_max(w);
            if (lane == (uint32_t)__builtin_ctzll(__ballot(w == best))) w = INT32_MIN;
        }
    if (lane == 0) tw[wave] = wave < full ? best : INT32_MAX;
    __syncthreads();
    const int32_t all = __builtin_amdgcn_readfirstlane(row_min(tw[lane % WAVES]));
    return r <= 64 ? fmaxf(unordered(all), -INFINITY) : -INFINITY;           // no NaN: lanes that have run out
}

// The k-th largest place of n elements, whose indices begin at `offset`, and in s.keep, in any order, the k places from it on; others(v) is called for every
// other element.  They are read as often as it takes: a digit of 8 bits at a time is found from the counts of that digit among the elements that agree with the
// digits before.
template <class T, int THREADS, int ROOM, class F> __device__ __forceinline__ u64 exact_keep(const typename T::raw* z, uint32_t n, uint32_t k, uint32_t offset, TopShared<THREADS, ROOM>& s, F&& others) {
    const uint32_t t = threadIdx.x;
    u64 prefix = 0;
    uint32_t want = k;                         // how many of the elements that agree with `prefix` are still wanted
    for (int shift = 56; shift >= 0; shift -= 8) {
        __syncthreads();
        for (uint32_t i = t; i < 256; i += THREADS) s.bins[i] = 0;
        __syncthreads();
        for (uint32_t i = t; i < n; i += THREADS) {
            const u64 c = place_of(to_float<T>(z[i]), offset + i);
            if (shift == 56 || c >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&s.bins[(uint32_t)(c >> shift) & 255], 1u);
        }
        __syncthreads();
        if (t == 0) {
            uint32_t left = want, d = 255;
            while (s.bins[d] < left) left -= s.bins[d--];
            s.digit = d;
            s.left = left;
        }
        __syncthreads();
        prefix |= (u64)s.digit << shift;
        want = s.left;
    }
    if (t == 0) s.got = 0;
    __syncthreads();
    for (uint32_t i = t; i < n; i += THREADS) {
        const float v = to_float<T>(z[i]);
        const u64 c = place_of(v, offset + i);
        if (c >= prefix) s.keep[atomicAdd(&s.got, 1u)] = c;                  // exactly k
        else others(v);
    }
    __syncthreads();
    return prefix;
}

#endif
