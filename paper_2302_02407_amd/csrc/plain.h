// Plaintext numbers (the operators of a teacher's head and a student's loss): element types, conversions and reductions over a
// wavefront or a work group.  Everything is computed in 32 bits; an element is rounded once, to nearest even, when it is stored.
#ifndef HE_PLAIN_H
#define HE_PLAIN_H

#include "he_internal.h"

#define HE_LOG2E 1.44269504088896340736f
#define HE_LN2 0.69314718055994530942f

struct f32_t { using raw = uint32_t; };
struct bf16_t { using raw = uint16_t; };
struct f16_t { using raw = uint16_t; };

template <class T> __device__ __forceinline__ float to_float(typename T::raw r);
template <> __device__ __forceinline__ float to_float<f32_t>(uint32_t r) { return __builtin_bit_cast(float, r); }
template <> __device__ __forceinline__ float to_float<bf16_t>(uint16_t r) { return __builtin_bit_cast(float, (uint32_t)r << 16); }
template <> __device__ __forceinline__ float to_float<f16_t>(uint16_t r) { return (float)__builtin_bit_cast(_Float16, r); }
template <class T> __device__ __forceinline__ typename T::raw from_float(float v);
template <> __device__ __forceinline__ uint32_t from_float<f32_t>(float v) { return __builtin_bit_cast(uint32_t, v); }
template <> __device__ __forceinline__ uint16_t from_float<bf16_t>(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
template <> __device__ __forceinline__ uint16_t from_float<f16_t>(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }   // v_exp_f32: 1 ulp, -inf -> 0

template <class F> __device__ __forceinline__ float wave_reduce(float v, F f) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v = f(v, __shfl_xor(v, o));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) { return wave_reduce(v, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ float wave_max(float v) { return wave_reduce(v, [](float a, float b) { return fmaxf(a, b); }); }

// Over a work group of WAVES wavefronts: every thread gets the result, in a fixed order.  `room`: WAVES floats that nothing else uses
// between the two barriers.
template <int WAVES, class F> __device__ __forceinline__ float group_reduce(float v, float* room, F f) {
    v = wave_reduce(v, f);
    if (WAVES == 1) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    v = room[0];
#pragma unroll
    for (int i = 1; i < WAVES; i++) v = f(v, room[i]);
    return v;
}
template <int WAVES> __device__ __forceinline__ float group_sum(float v, float* room) { return group_reduce<WAVES>(v, room, [](float a, float b) { return a + b; }); }
template <int WAVES> __device__ __forceinline__ float group_max(float v, float* room) { return group_reduce<WAVES>(v, room, [](float a, float b) { return fmaxf(a, b); }); }

// Sixteen bytes of a row that starts anywhere its elements may: N numbers from p on, of which `left` are the row's; the others are `fill`
template <class T> struct Vec {
    using raw = typename T::raw;
    static constexpr int N = 16 / sizeof(raw);
    raw r[N];
    __device__ __forceinline__ void load(const raw* p, uint32_t left, float fill) {
        if (left >= (uint32_t)N) __builtin_memcpy(r, p, 16);
        else
#pragma unroll
            for (int i = 0; i < N; i++) r[i] = (uint32_t)i < left ? p[i] : from_float<T>(fill);
    }
    __device__ __forceinline__ void store(raw* p, uint32_t left) const {
        if (left >= (uint32_t)N) __builtin_memcpy(p, r, 16);
        else
#pragma unroll
            for (int i = 0; i < N; i++)
                if ((uint32_t)i < left) p[i] = r[i];
    }
    __device__ __forceinline__ float operator[](int i) const { return to_float<T>(r[i]); }
};

// Maximum over a wavefront, the same in all lanes: within rows of 16 lanes by rotations, then over the four rows
template <int CTRL> __device__ __forceinline__ float rotated(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float lane_value(float v, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }
__device__ __forceinline__ float wave_max_dpp(float v) {
    v = fmaxf(v, rotated<0x128>(v));      // row_ror:8, 4, 2, 1
    v = fmaxf(v, rotated<0x124>(v));
    v = fmaxf(v, rotated<0x122>(v));
    v = fmaxf(v, rotated<0x121>(v));
    return fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)), fmaxf(lane_value(v, 32), lane_value(v, 48)));
}

// Calls f with the type of `dtype` (an he_dtype that has been checked)
template <class F> static inline void with_dtype(int32_t dtype, F&& f) {
    if (dtype == HE_F32) f(f32_t{});
    else if (dtype == HE_BF16) f(bf16_t{});
    else f(f16_t{});
}
static inline uint32_t dtype_bytes(int32_t dtype) { return dtype == HE_F32 ? 4 : 2; }
static inline bool dtype_known(int32_t dtype) { return dtype == HE_F32 || dtype == HE_BF16 || dtype == HE_F16; }
// Whether [a, a + na) and [b, b + nb) share a byte
static inline bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
    return a && b && na && nb && (const char*)a < (const char*)b + nb && (const char*)b < (const char*)a + na;
}
// Bytes from the first to past the last element of `rows` rows of `cols` elements, `ld` elements apart
static inline uint64_t span(uint64_t rows, uint64_t cols, uint64_t ld, uint64_t size) { return rows && cols ? ((rows - 1) * ld + cols) * size : 0; }
// Rows of `cols` elements, ld apart: they do not overlap, and no offset of HE_ROWS_MAX of them leaves 64 bits
static inline bool ld_fits(uint64_t ld, uint64_t cols) { return ld >= cols && ld <= (1u << 28); }
#define HE_ROWS_MAX (1u << 21)     // a work group of at most 1024 threads a row: a launch's threads stay below 2^32
#define HE_VOCAB_MAX (1u << 20)
// Kernel arguments have been checked; what can still fail is the launch
#define HE_LAUNCHED(ctx) HE_HIP(ctx, hipGetLastError())

#endif
