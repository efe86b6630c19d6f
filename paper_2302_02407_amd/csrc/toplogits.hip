// The k largest logits of a row in order, and the log-sum-exp of the others.
#include "top.h"

struct TopArgs {
    const void* z;
    float* values;
    int32_t* index;
    float* rest;
    u64 ld_z;
    uint32_t vocab, k;
    float tau;
};

// A sum times a power of two: what is beside nothing is nothing, also where it had become infinite
__device__ __forceinline__ float times_power(float sum, float exponent) {
    const float f = exp2_fast(exponent);
    return f > 0.0f || sum != sum ? sum * f : 0.0f;
}

// d_rest of a row, whose k-th place is `last` and whose largest other logit that counts is `most`, by reading it once more
template <class T, int THREADS> __device__ __forceinline__ void rest_of(const TopArgs& a, TopShared<THREADS>& s, u64 row, u64 last, float most) {
    const typename T::raw* z = (const typename T::raw*)a.z + row * a.ld_z;
    const float c = HE_LOG2E / a.tau, low = masked_from(a.tau), at = most == -INFINITY ? 0.0f : most;
    float sum = 0;
    for (uint32_t i = threadIdx.x; i < a.vocab; i += THREADS) {
        const float v = to_float<T>(z[i]);
        if (place_of(v, i) < last && !(v <= low)) sum += v >= -low ? INFINITY : exp2_fast((v - at) * c);
    }
    sum = group_sum<THREADS / 64>(sum, s.room);
    if (threadIdx.x == 0) a.rest[row] = at >= -low ? sum : logf(sum) + at / a.tau;
}

// A row by reading it as often as it takes; the rest is summed against its own maximum.  For rows with so many equal elements, or elements in such an
// order, that setting aside (below) has not enough room, and for rows with NaN.
template <class T, int THREADS> __device__ __forceinline__ void exact_row(const TopArgs& a, TopShared<THREADS>& s, u64 row) {
    using raw = typename T::raw;
    const raw* z = (const raw*)a.z + row * a.ld_z;
    const uint32_t t = threadIdx.x;
    const float low = masked_from(a.tau);
    float most = -INFINITY;
    const u64 prefix = exact_keep<T>(z, a.vocab, a.k, 0, s, [&](float v) {
        if (!(v <= low)) most = fmaxf(most, v);
    });
    most = group_max<THREADS / 64>(most, s.room);
    for (uint32_t i0 = t; i0 < a.k; i0 += THREADS) {
        const u64 c = s.keep[i0];
        uint32_t place = 0;
        for (uint32_t j = 0; j < a.k; j++) place += s.keep[j] > c;
        const uint32_t i = ~(uint32_t)c;
        a.values[row * a.k + place] = to_float<T>(z[i]);
        a.index[row * a.k + place] = (int32_t)i;
    }
    if (a.rest) rest_of<T, THREADS>(a, s, row, prefix, most);
}

// One row a work group, read once, 16 bytes a lane at a time.  Pieces of 16 bytes with an element that reaches a threshold are set aside in
// LDS, the elements of the others go into their lane's sum against its running maximum.  The threshold is one that at least k
// elements reach: every wavefront has r = ceil(k / wavefronts) lanes whose largest element so far reaches its r-th largest lane's, and the
// smallest of those over the wavefronts is it.  It is taken anew after 0, 2, 6, 14 ... turns, so that of a row in no particular order a
// few times k (1 + ln(turns)) pieces are set aside, and once more at the end.  Of the elements that reach the last one each counts how
// many come before it: the first k are the result, in order.  The others join the sum as whole multiples of 2^-44 of the rest's largest
// term, in any order the same number.  A term's exponent is one multiply-add, c z - R with R = c times the running maximum; the rounding of R
// stays in it, 2^-25 of R, which is that of the result (its size is R ln 2) as long as it is a factor of at most 2^(1/2): up to R = 2^24.  Beyond, a lane's
// sum may be off by any factor; it counts for nothing beside a rest below that, and a rest beyond it (of nothing but masks at -1e9, say) is
// summed anew from differences.  An element of -infinity can only be among the first k if its index is below k: of the first k
// elements at most as many are larger as there are larger ones at all.
//
// 2048 x 131072 bf16, k = 64: 144 us (3.7 TB/s), 87% of its cycles vector instructions: about 17 for an element, of which 8 are the sum's (one
// exponential among them) and the rest maxima, thresholds and what is set aside.  As ten passes of a digit it took 3.1 ms.
template <class T, int THREADS> __global__ __launch_bounds__(THREADS, THREADS == 1024 ? 8 : 4) void top_logits_kernel(TopArgs a) {
    using raw = typename T::raw;
    constexpr int N = Vec<T>::N, WAVES = THREADS / 64, ROOM = TopShared<THREADS>::ROOM, KEEP = TopShared<THREADS>::KEEP;
    __shared__ TopShared<THREADS> s;
    const u64 row = blockIdx.x;
    const raw* z = (const raw*)a.z + row * a.ld_z;
    const uint32_t t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    if (a.vocab < (uint32_t)N) return exact_row<T, THREADS>(a, s, row);
    const Row<T> in{z, a.vocab};
    const uint32_t vecs = in.pieces(), turns = (vecs + THREADS - 1) / THREADS;
    const uint32_t full = max(1u, min((uint32_t)WAVES, vecs / 64)), r = (a.k + full - 1) / full;      // a lane without a piece counts as -infinity
    const float c = HE_LOG2E / a.tau, low = masked_from(a.tau);
    if (t == 0) s.got = s.kept = 0, s.more = 0;
    float m = low, sum = 0, high = -INFINITY, least = -INFINITY;
    auto raise = [&](int32_t* tw) {
        least = reached_by_all<WAVES>(high, r, full, lane, wave, tw);
    };
    auto turn = [&](uint32_t p, Vec<T>& buf) {           // two buffers in turn, each refilled as soon as it is taken
        const uint32_t v = p * THREADS + t;
        const uint32_t base = in.base(v), past = v * N - base;       // elements of it that are another piece's
        Vec<T> x = buf;
        buf = in.load(v + 2 * THREADS);
        float e[N];
#pragma unroll
        for (int i = 0; i < N; i++) e[i] = x[i];
        if (past)
#pragma unroll
            for (int i = 0; i < N; i++)
                if ((uint32_t)i < past) x.set(i, e[i] = -INFINITY);
        float mx = e[0];
#pragma unroll
        for (int i = 1; i < N; i++) mx = fmaxf(mx, e[i]);
        high = fmaxf(high, mx);
        if (((p + 1) & (p + 2)) == 0) raise(s.tw[__builtin_ctz(p + 2) & 1]);
        if (!(mx < least) && (mx != -INFINITY || base < a.k)) {
            const uint32_t to = atomicAdd(&s.got, 1u);
            if (to < ROOM) {
                s.aside[to] = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
                s.which[to] = base | min(past, 15u) << 24;
            }
        } else {
            if (mx > m) {
                sum = times_power(sum, (m - mx) * c);
                m = mx;
            }
            const float mc = m == low ? 0.0f : m * c;      // nothing that counts so far
#pragma unroll
            for (int i = 0; i < N; i++) sum += exp2_fast(fmaf(e[i], c, -mc));
        }
    };
    Vec<T> one = in.load(t), two = in.load(THREADS + t);
    for (uint32_t p = 0; p < turns; p += 2) {
        turn(p, one);
        if (p + 1 < turns) turn(p + 1, two);
    }
    __syncthreads();                                     // all is set aside, and the slots of tw have been read
    const uint32_t got = s.got;
    if (got > ROOM || __syncthreads_or(sum != sum)) return exact_row<T, THREADS>(a, s, row);
    raise(s.tw[0]);
    float most = m;
    for (uint32_t i = t; i < got * N; i += THREADS) {
        const float v = to_float<T>(((const raw*)s.aside)[i]);
        const uint32_t which = s.which[i / N], at = (which & 0xffffff) + i % N;
        if (!(v < least) && i % N >= which >> 24) {
            const uint32_t to = atomicAdd(&s.kept, 1u);
            if (to < KEEP) s.keep[to] = place_of(v, at);
        } else most = fmaxf(most, v);
    }
    __syncthreads();
    const uint32_t kept = s.kept;
    if (kept > KEEP) return exact_row<T, THREADS>(a, s, row);
    constexpr int Q = KEEP > THREADS ? KEEP / THREADS : 1;
    u64 over[Q];                                         // what this thread looks after and is not among the first k, 0: nothing
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const uint32_t i = q * THREADS + t;
        over[q] = 0;
        if (i >= kept) continue;
        const u64 mine = s.keep[i];
        uint32_t place = 0;
        for (uint32_t j = 0; j < kept; j++) place += s.keep[j] > mine;
        if (place < a.k) {
            const uint32_t at = ~(uint32_t)mine;
            a.values[row * a.k + place] = to_float<T>(z[at]);          // as it stands there: -0, the NaN's bits
            a.index[row * a.k + place] = (int32_t)at;
            if (place == a.k - 1) s.last = mine;
        } else {
            over[q] = mine;
            most = fmaxf(most, value_of((uint32_t)(mine >> 32)));
        }
    }
    if (!a.rest) return;
    bool lost = false;                                   // a NaN among the rest
    most = group_max<WAVES>(most, s.room);
    if (most > low && fabsf(most) * c >= 0x1p24f) {
        __syncthreads();                                 // `last` is there
        return rest_of<T, THREADS>(a, s, row, s.last, most);
    }
    u64 more = 0;
    auto add = [&](float v) {
        lost = lost || v != v;
        if (!(v <= low) && most < -low) more += (u64)(exp2_fast((v - most) * c) * 0x1p44f);
    };
    for (uint32_t i = t; i < got * N; i += THREADS) {
        const float v = to_float<T>(((const raw*)s.aside)[i]);
        if (v < least) add(v);
    }
#pragma unroll
    for (int q = 0; q < Q; q++)
        if (over[q]) add(value_of((uint32_t)(over[q] >> 32)));
    if (more) atomicAdd((unsigned long long*)&s.more, (unsigned long long)more);
    sum = group_sum<WAVES>(!(most < -low) ? 0.0f : times_power(sum, (m - most) * c), s.room);
    lost = __syncthreads_or(lost);
    if (t == 0) a.rest[row] = lost ? NAN : most >= -low ? INFINITY : logf(sum + (float)s.more * 0x1p-44f) + most / a.tau;
}

extern "C" int32_t he_top_logits(he_ctx* ctx, const he_top_plan* p) {
    return he_guard(ctx, "he_top_logits: host allocation failed", [&]() -> int32_t {
    if (!ctx) return HE_ERR_BADARG;
    if (!p) return he_fail(ctx, HE_ERR_BADARG, "he_top_logits: null plan");
    if (!dtype_known(p->dtype)) return he_fail(ctx, HE_ERR_BADARG, "he_top_logits: unknown type %d", p->dtype);
    if (p->vocab == 0 || p->vocab > HE_VOCAB_MAX) return he_fail(ctx, HE_ERR_BADARG, "he_top_logits: %u logits outside 1..2^20", p->vocab);
    if (p->k == 0 || p->k > HE_TOP_MAX || p->k > p->vocab) return he_fail(ctx, HE_ERR_BADARG, "he_top_logits: k = %u outside 1..min(vocab, %d)", p->k, HE_TOP_MAX);
    if (!tau_fits(p->tau)) return he_fail(ctx, HE_ERR_BADARG, "he_top_logits: the temperature is not a number from 2^-60 to 2^60");
    if (p->rows > HE_ROWS_MAX) return he_fail(ctx, HE_ERR_BADARG, "he_top_logits: more than 2^21 rows");
    if (p->rows == 0) return HE_OK;
    if (!p->d_z || !p->d_values || !p->d_index) return he_fail(ctx, HE_ERR_BADARG, "he_top_logits: null argument");
    if (!ld_fits(p->ld_z, p->vocab)) return he_fail(ctx, HE_ERR_BADARG, "he_top_logits: ld_z is below the row's length or above 2^28");
    const uint32_t es = dtype_bytes(p->dtype);
    if ((uintptr_t)p->d_z & (es - 1) || ((uintptr_t)p->d_values | (uintptr_t)p->d_index | (uintptr_t)p->d_rest) & 3)
        return he_fail(ctx, HE_ERR_BADARG, "he_top_logits: a pointer is not aligned to its elements");
    const uint64_t nz = span(p->rows, p->vocab, p->ld_z, es), nk = (uint64_t)p->rows * p->k * 4, nr = (uint64_t)p->rows * 4;
    if (overlap(p->d_z, nz, p->d_values, nk) || overlap(p->d_z, nz, p->d_index, nk) || overlap(p->d_z, nz, p->d_rest, nr) ||
        overlap(p->d_values, nk, p->d_index, nk) || overlap(p->d_values, nk, p->d_rest, nr) || overlap(p->d_index, nk, p->d_rest, nr))
        return he_fail(ctx, HE_ERR_BADARG, "he_top_logits: an output overlaps the logits or another output");
    const TopArgs a = {p->d_z, p->d_values, p->d_index, p->d_rest, p->ld_z, p->vocab, p->k, p->tau};
    with_dtype(p->dtype, [&](auto t) {
        using T = decltype(t);
        // Rows of at most a piece a lane go to one wavefront (4000 x 500 bf16, k = 20: 15 us, by four 83; 3090 x 48, k of a few: 6.7 and 14), unless most of a
        // row's elements are candidates, which four put in order sooner (256 x 500, k = 100: 21 us, by one 62).  Slow among those of four:
        // elements of 16 bits, 513 to 1023 of them, and k above some 30.  One wavefront's lanes are full then, so a threshold takes k maxima one
        // after another (256 x 1000, k = 64: 68 us); above 64 none is taken, all of the row stays, more than there is room for, and it is read
        // ten times (k = 128: 64 us; f32, which there is room for: 24).
        const uint64_t bytes = (uint64_t)p->vocab * es;
        if (bytes > 32768) top_logits_kernel<T, 1024><<<p->rows, 1024, 0, ctx->stream>>>(a);
        else if (bytes <= 1024 && (p->k <= 32 || p->vocab <= 128)) top_logits_kernel<T, 64><<<p->rows, 64, 0, ctx->stream>>>(a);
        else top_logits_kernel<T, 256><<<p->rows, 256, 0, ctx->stream>>>(a);
    });
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}
