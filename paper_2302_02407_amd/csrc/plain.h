// Plaintext numbers (the operators of a teacher's head and a student's loss): element types, conversions and reductions over a
// wavefront or a work group.  Everything is computed in 32 bits; an element is rounded once, to nearest even, when it is stored.
#ifndef HE_PLAIN_H
#define HE_PLAIN_H

#include <type_traits>

#include "checks.h"
#include "he_internal.h"

#define HE_LOG2E 1.44269504088896340736f
#define HE_LN2 0.69314718055994530942f
// A logit z with z or z / tau at -2^126 or below, such as the lowest number of its type in a masked place, counts as -infinity in a sum of
// exponentials: from there on log2(e) / tau times z need not be a number any more.
#define HE_MASKED -0x1p126f
__device__ __forceinline__ float masked_from(float tau) { return HE_MASKED * fminf(1.0f, tau); }

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

// What the lanes of a wavefront have written to LDS is there for its other lanes after this
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Reductions over a wavefront, the same in all lanes: rotations within rows of 16 lanes, then the four rows' results as scalars.  (The
// maximum of integers takes an instruction a step; of floats two more make a signalling NaN a quiet one.)
template <int CTRL> __device__ __forceinline__ int32_t rotated(int32_t v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true); }   // 0x120 + n: row_ror:n
// Maximum, minimum over each row of 16 lanes
__device__ __forceinline__ int32_t row_max(int32_t v) {
    v = max(v, rotated<0x128>(v));
    v = max(v, rotated<0x124>(v));
    v = max(v, rotated<0x122>(v));
    return max(v, rotated<0x121>(v));
}
__device__ __forceinline__ int32_t row_min(int32_t v) {
    v = min(v, rotated<0x128>(v));
    v = min(v, rotated<0x124>(v));
    v = min(v, rotated<0x122>(v));
    return min(v, rotated<0x121>(v));
}
__device__ __forceinline__ int32_t wave_max(int32_t v) {
    v = row_max(v);
    return max(max(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)), max(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}
template <class F> __device__ __forceinline__ float wave_reduce(float v, F f) {
    const auto bits = [](float x) { return __builtin_bit_cast(int32_t, x); };
    const auto number = [](int32_t x) { return __builtin_bit_cast(float, x); };
    v = f(v, number(rotated<0x128>(bits(v))));
    v = f(v, number(rotated<0x124>(bits(v))));
    v = f(v, number(rotated<0x122>(bits(v))));
    v = f(v, number(rotated<0x121>(bits(v))));
    const auto row = [&](int lane) { return number(__builtin_amdgcn_readlane(bits(v), lane)); };
    return f(f(row(0), row(16)), f(row(32), row(48)));
}
__device__ __forceinline__ float wave_sum(float v) { return wave_reduce(v, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ float wave_max(float v) { return wave_reduce(v, [](float a, float b) { return fmaxf(a, b); }); }

// Over each row of 16 lanes
__device__ __forceinline__ float row_sum(float v) {
    const auto turned = [&](auto ctrl) { return __builtin_bit_cast(float, rotated<decltype(ctrl)::value>(__builtin_bit_cast(int32_t, v))); };
    v += turned(std::integral_constant<int, 0x128>{});
    v += turned(std::integral_constant<int, 0x124>{});
    v += turned(std::integral_constant<int, 0x122>{});
    return v + turned(std::integral_constant<int, 0x121>{});
}

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

// Two sums at once; `room`: 2 * WAVES floats.  WAVES = 0: over rows of 16 lanes
template <int WAVES> __device__ __forceinline__ void group_sum2(float& x, float& y, float* room) {
    if constexpr (WAVES == 0) {
        x = row_sum(x);
        y = row_sum(y);
        return;
    }
    x = wave_sum(x);
    y = wave_sum(y);
    if (WAVES == 1) return;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        room[threadIdx.x >> 6] = x;
        room[WAVES + (threadIdx.x >> 6)] = y;
    }
    __syncthreads();
    x = room[0];
    y = room[WAVES];
#pragma unroll
    for (int i = 1; i < WAVES; i++) {
        x += room[i];
        y += room[WAVES + i];
    }
}

// Sixteen bytes of a row, which may start anywhere its elements may
template <class T> struct Vec {
    using raw = typename T::raw;
    static constexpr int N = 16 / sizeof(raw);
    uint32_t w[4];
    __device__ __forceinline__ void load(const raw* p) { __builtin_memcpy(w, p, 16); }
    __device__ __forceinline__ void store(raw* p) const { __builtin_memcpy(p, w, 16); }
    // What is not read again soon: it leaves the cache to what is
    __device__ __forceinline__ void store_past(raw* p) const {
        typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
        __builtin_nontemporal_store(u4{w[0], w[1], w[2], w[3]}, (u4*)p);
    }
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (N == 4) return __builtin_bit_cast(float, w[i]);
        else if constexpr (__is_same(T, bf16_t)) return __builtin_bit_cast(float, i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else return (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i / 2] >> 16 * (i & 1)));
    }
    __device__ __forceinline__ void set(const float* v) {
        if constexpr (N == 4)
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] = __builtin_bit_cast(uint32_t, v[i]);
        else
#pragma unroll
            for (int i = 0; i < 4; i++) {
                typedef float f2 __attribute__((ext_vector_type(2)));
                const f2 p = {v[2 * i], v[2 * i + 1]};
                if constexpr (__is_same(T, bf16_t)) {
                    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
                    w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, b2));
                } else {
                    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
                    w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, h2));
                }
            }
    }
    __device__ __forceinline__ void set(int i, float v) {
        const raw r = from_float<T>(v);
        if constexpr (N == 4) w[i] = r;
        else w[i / 2] = i & 1 ? (w[i / 2] & 0xffffu) | (uint32_t)r << 16 : (w[i / 2] & 0xffff0000u) | r;
    }
};

// Eight elements of a row, as numbers
template <class T> struct Eight {
    using raw = typename T::raw;
    static constexpr int VECS = 8 / Vec<T>::N;
    Vec<T> v[VECS];
    __device__ __forceinline__ void load(const raw* p) {
#pragma unroll
        for (int i = 0; i < VECS; i++) v[i].load(p + i * Vec<T>::N);
    }
    __device__ __forceinline__ void store(raw* p) const {
#pragma unroll
        for (int i = 0; i < VECS; i++) v[i].store(p + i * Vec<T>::N);
    }
    __device__ __forceinline__ float operator[](int i) const { return v[i / Vec<T>::N][i % Vec<T>::N]; }
    __device__ __forceinline__ void set(const float* x) {
#pragma unroll
        for (int i = 0; i < VECS; i++) v[i].set(x + i * Vec<T>::N);
    }
};

// Eight elements from `at` on of a row of n, zeros for those that are not there; and those of them that are there written
template <class T> __device__ __forceinline__ void load8(const typename T::raw* p, uint32_t at, uint32_t n, float* x) {
    if (at + 8 <= n) {
        Eight<T> v;
        v.load(p + at);
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = v[i];
    } else
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = at + i < n ? to_float<T>(p[at + i]) : 0.0f;
}
template <class T> __device__ __forceinline__ void store8(typename T::raw* p, uint32_t at, uint32_t n, const float* x) {
    if (at + 8 <= n) {
        Eight<T> v;
        v.set(x);
        v.store(p + at);
    } else
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (at + i < n) p[at + i] = from_float<T>(x[i]);
}

// A row of n >= N elements in pieces of 16 bytes, without a branch on the way to a load: piece v starts at base(v), the last one, and any
// past it, where it still lies in the row.  The elements of those that belong to the piece before, or to nothing, are those below
// v * N.
template <class T> struct Row {
    using raw = typename T::raw;
    static constexpr uint32_t N = Vec<T>::N;
    const raw* p;
    uint32_t n;
    __device__ __forceinline__ uint32_t pieces() const { return (n + N - 1) / N; }
    __device__ __forceinline__ uint32_t base(uint32_t v) const { return min(v * N, n - N); }
    __device__ __forceinline__ Vec<T> load(uint32_t v) const {
        Vec<T> x;
        x.load(p + base(v));
        return x;
    }
    // Piece v of a row that is written: all of it, or of a last one what is its own
    __device__ __forceinline__ void store(raw* to, uint32_t v, const Vec<T>& x, bool past_cache) const {
        const uint32_t at = base(v), past = v * N - at;
        if (past == 0) {
            if (past_cache) x.store_past(to + at);
            else x.store(to + at);
        } else
#pragma unroll
            for (uint32_t i = 0; i < N; i++)
                if (i >= past) to[at + i] = from_float<T>(x[i]);
    }
};
// The same of a row of fewer than N elements: piece 0 with -infinity after them
template <class T> struct ShortRow {
    using raw = typename T::raw;
    static constexpr uint32_t N = Vec<T>::N;
    const raw* p;
    uint32_t n;
    __device__ __forceinline__ uint32_t pieces() const { return 1; }
    __device__ __forceinline__ uint32_t base(uint32_t) const { return 0; }
    __device__ __forceinline__ Vec<T> load(uint32_t) const {
        float x[N];
#pragma unroll
        for (uint32_t i = 0; i < N; i++) x[i] = i < n ? to_float<T>(p[i]) : -INFINITY;
        Vec<T> v;
        v.set(x);
        return v;
    }
    __device__ __forceinline__ void store(raw* to, uint32_t v, const Vec<T>& x, bool) const {
#pragma unroll
        for (uint32_t i = 0; i < N; i++)
            if (v == 0 && i < n) to[i] = from_float<T>(x[i]);
    }
};

// Which tile a work group owns.  Work groups go to the 8 dies in turn and each die has a cache of its own, so die x takes the x-th
// eighth of the tiles, in stripes of 8 tiles of the second operand: its 32 compute units then work on about 8 x 4 tiles at a time, which read
// 12 strips instead of 33.
__device__ __forceinline__ void tile_in_order(uint32_t t, uint32_t tiles_n, uint32_t tiles_m, uint32_t& n, uint32_t& m) {
    const uint32_t stripe = t / (8 * tiles_n), high = min(8u, tiles_m - 8 * stripe), r = t - stripe * 8 * tiles_n;
    m = 8 * stripe + r % high;
    n = r / high;
}
__device__ __forceinline__ bool tile_of(uint32_t tiles_n, uint32_t tiles_m, uint32_t& n, uint32_t& m) {
    const uint32_t all = tiles_n * tiles_m, each = (all + 7) / 8, t = blockIdx.x % 8 * each + blockIdx.x / 8;
    if (blockIdx.x / 8 >= each || t >= all) return false;
    tile_in_order(t, tiles_n, tiles_m, n, m);
    return true;
}

// Numbers as integers in their order, and back (NaN lies beyond the infinity of its sign)
__device__ __forceinline__ int32_t ordered(float v) {
    const int32_t b = __builtin_bit_cast(int32_t, v);
    return b ^ (b >> 31 & 0x7fffffff);
}
__device__ __forceinline__ float unordered(int32_t k) { return __builtin_bit_cast(float, k ^ (k >> 31 & 0x7fffffff)); }

// Calls f with the type of `dtype` (an he_dtype that has been checked)
template <class F> static inline void with_dtype(int32_t dtype, F&& f) {
    if (dtype == HE_F32) f(f32_t{});
    else if (dtype == HE_BF16) f(bf16_t{});
    else f(f16_t{});
}
// Kernel arguments have been checked; what can still fail is the launch
#define HE_LAUNCHED(ctx) HE_HIP(ctx, hipGetLastError())

// The context's GPU is the current one while this lives
class OnDevice {
    int was_ = -1;

public:
    hipError_t status;
    explicit OnDevice(const he_ctx* ctx) {
        int now = -1;
        status = hipGetDevice(&now);
        if (status != hipSuccess || now == ctx->device) return;
        status = hipSetDevice(ctx->device);
        if (status == hipSuccess) was_ = now;
    }
    ~OnDevice() {
        if (was_ >= 0) (void)hipSetDevice(was_);
    }
    OnDevice(const OnDevice&) = delete;
};
// What an operator with a check of its plan (checks.h) does first
#define HE_REFUSE(ctx, name, why)                                                    \
    do {                                                                             \
        if (const char* why__ = (why)) return he_fail(ctx, HE_ERR_BADARG, "%s: %s", name, why__); \
    } while (0)

#endif
