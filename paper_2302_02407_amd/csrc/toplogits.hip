// The k largest logits of a row in order, and the log-sum-exp of the others.
#include "plain.h"

struct TopArgs {
    const void* z;
    float* values;
    int32_t* index;
    float* rest;
    u64 ld_z;
    uint32_t vocab, k;
    float tau;
};

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

template <int THREADS> struct TopShared {
    static constexpr int ROOM = 2048;          // elements that can be set aside
    u64 found[ROOM];
    float dropped[ROOM];
    uint32_t bins[256];
    float tw[2][THREADS / 64], room[THREADS / 64];
    uint32_t digit, left, got;
};

// A row by reading it as often as it takes: the k-th largest place is found a digit of 8 bits at a time, from the row's counts of that digit
// among the elements that agree with the digits before; then the elements from it on are gathered and the rest is summed against its own
// maximum.  For rows with so many equal elements, or elements in such an order, that setting aside (below) has not enough room, and for rows
// with NaN.
template <class T, int THREADS> __device__ __forceinline__ void exact_row(const TopArgs& a, TopShared<THREADS>& s, u64 row) {
    using raw = typename T::raw;
    const raw* z = (const raw*)a.z + row * a.ld_z;
    const uint32_t t = threadIdx.x;
    u64 prefix = 0;
    uint32_t want = a.k;                       // how many of the elements that agree with `prefix` are still wanted
    for (int shift = 56; shift >= 0; shift -= 8) {
        __syncthreads();
        if (t < 256) s.bins[t] = 0;
        __syncthreads();
        for (uint32_t i = t; i < a.vocab; i += THREADS) {
            const u64 c = place_of(to_float<T>(z[i]), i);
            if (shift == 56 || c >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&s.bins[(uint32_t)(c >> shift) & 255], 1u);
        }
        __syncthreads();
        if (t == 0) {
            uint32_t n = want, d = 255;
            while (s.bins[d] < n) n -= s.bins[d--];
            s.digit = d;
            s.left = n;
        }
        __syncthreads();
        prefix |= (u64)s.digit << shift;
        want = s.left;
    }
    if (t == 0) s.got = 0;
    __syncthreads();
    float most = -INFINITY;
    for (uint32_t i = t; i < a.vocab; i += THREADS) {
        const float v = to_float<T>(z[i]);
        const u64 c = place_of(v, i);
        if (c >= prefix) s.found[atomicAdd(&s.got, 1u)] = c;    // exactly k
        else most = fmaxf(most, v);
    }
    most = group_max<THREADS / 64>(most, s.room);
    __syncthreads();
    if (t < a.k) {
        const u64 c = s.found[t];
        uint32_t place = 0;
        for (uint32_t j = 0; j < a.k; j++) place += s.found[j] > c;
        const uint32_t i = ~(uint32_t)c;
        a.values[row * a.k + place] = to_float<T>(z[i]);
        a.index[row * a.k + place] = (int32_t)i;
    }
    if (!a.rest) return;
    const float scale = HE_LOG2E / a.tau, at = most == -INFINITY ? 0.0f : most;
    float sum = 0;
    for (uint32_t i = t; i < a.vocab; i += THREADS) {
        const float v = to_float<T>(z[i]);
        if (place_of(v, i) < prefix) sum += v == INFINITY ? INFINITY : exp2_fast((v - at) * scale);
    }
    sum = group_sum<THREADS / 64>(sum, s.room);
    if (t == 0) a.rest[row] = at == INFINITY ? sum : logf(sum) + at / a.tau;
}

// One row a work group, read once, 16 bytes a lane at a time.  Elements from a threshold on are set aside in LDS, the others go into their
// lane's sum against its running maximum.  The threshold is one that at least k elements reach: every wavefront has r = ceil(k / wavefronts)
// lanes whose largest element so far reaches its r-th largest lane's, and the smallest of those over the wavefronts is it.  It is taken
// anew after 0, 1, 2, 4, 8 ... pieces of the row, so that of a row in no particular order some k (1 + ln(pieces)) elements are set
// aside.  At the end each of them counts how many of them come before it: the first k are the result, in order, the others join the
// sum, by their place in that order so that the same row gives the same bits.  An element of -infinity can only be among the
// first k if its index is below k: of the first k elements at most as many are larger as there are larger ones at all.
template <class T, int THREADS> __global__ __launch_bounds__(THREADS, THREADS == 1024 ? 8 : 4) void top_logits_kernel(TopArgs a) {
    using raw = typename T::raw;
    constexpr int N = Vec<T>::N, WAVES = THREADS / 64, ROOM = TopShared<THREADS>::ROOM;
    __shared__ TopShared<THREADS> s;
    const u64 row = blockIdx.x;
    const raw* z = (const raw*)a.z + row * a.ld_z;
    const uint32_t t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const uint32_t vecs = (a.vocab + N - 1) / N, pieces = (vecs + THREADS - 1) / THREADS;
    const uint32_t full = min((uint32_t)WAVES, vecs / 64), r = full ? (a.k + full - 1) / full : 65;
    const float c = HE_LOG2E / a.tau;
    auto load = [&](uint32_t v) {
        Vec<T> x;
        const uint32_t at = v * N;
        x.load(z + at, at < a.vocab ? a.vocab - at : 0, -INFINITY);
        return x;
    };
    if (t == 0) s.got = 0;
    float m = -3e38f, sum = 0, high = -INFINITY, least = -INFINITY;
    Vec<T> next = load(t);
    for (uint32_t p = 0; p < pieces; p++) {
        const Vec<T> x = next;
        if (p + 1 < pieces) next = load((p + 1) * THREADS + t);
        float e[N];
#pragma unroll
        for (int i = 0; i < N; i++) e[i] = x[i];
        float mx = e[0];
#pragma unroll
        for (int i = 1; i < N; i++) mx = fmaxf(mx, e[i]);
        high = fmaxf(high, mx);
        if ((p & (p - 1)) == 0) {
            float w = high, best = -INFINITY;
            if (r <= 64)
                for (uint32_t i = 0; i < r; i++) {
                    best = wave_max_dpp(w);
                    const uint64_t who = __ballot(w == best);
                    if (lane == (uint32_t)__builtin_ctzll(who | 1ull << 63)) w = -INFINITY;
                }
            float* tw = s.tw[p ? __builtin_ctz(p) + 1 & 1 : 0];
            if (lane == 0) tw[wave] = wave < full ? best : INFINITY;
            __syncthreads();
            least = tw[0];
#pragma unroll
            for (int i = 1; i < WAVES; i++) least = fminf(least, tw[i]);
            if (r > 64) least = -INFINITY;
        }
        if (__any(!(mx < least))) {
            const uint32_t at = (p * THREADS + t) * N;
#pragma unroll
            for (int i = 0; i < N; i++)
                if (!(e[i] < least)) {
                    if (e[i] != -INFINITY || at + i < a.k) {
                        const uint32_t to = atomicAdd(&s.got, 1u);
                        if (to < ROOM) s.found[to] = place_of(e[i], at + i);
                    }
                    e[i] = -INFINITY;
                }
            mx = e[0];
#pragma unroll
            for (int i = 1; i < N; i++) mx = fmaxf(mx, e[i]);
        }
        if (__any(mx > m)) {
            const float to = fmaxf(m, mx);
            sum *= exp2_fast((m - to) * c);
            m = to;
        }
        const float mc = m == -3e38f ? 0.0f : m * c;     // nothing but -infinity so far
#pragma unroll
        for (int i = 0; i < N; i++) sum += exp2_fast(fmaf(e[i], c, -mc));
    }
    __syncthreads();
    const uint32_t got = s.got;
    if (got > ROOM || __syncthreads_or(sum != sum)) return exact_row<T, THREADS>(a, s, row);
    for (uint32_t i = t; i < got; i += THREADS) {
        const u64 mine = s.found[i];
        uint32_t place = 0;
        for (uint32_t j = 0; j < got; j++) place += s.found[j] > mine;
        const float v = value_of((uint32_t)(mine >> 32));
        if (place < a.k) {
            a.values[row * a.k + place] = to_float<T>(z[~(uint32_t)mine]);      // as it stands there: -0, the NaN's bits
            a.index[row * a.k + place] = (int32_t)~(uint32_t)mine;
        }
        s.dropped[place] = v;
    }
    if (!a.rest) return;
    __syncthreads();
    for (uint32_t i = a.k + t; i < got; i += THREADS) {
        const float v = s.dropped[i], to = fmaxf(m, v);
        sum = sum * exp2_fast((m - to) * c) + (v == INFINITY ? INFINITY : v == -INFINITY ? 0.0f : exp2_fast((v - to) * c));
        m = to;
    }
    const float most = group_max<WAVES>(m, s.room);
    sum = group_sum<WAVES>(sum == 0.0f ? 0.0f : most == INFINITY ? sum : sum * exp2_fast((m - most) * c), s.room);
    if (t == 0) a.rest[row] = most == INFINITY ? INFINITY : logf(sum) + most / a.tau;
}

extern "C" int32_t he_top_logits(he_ctx* ctx, const he_top_plan* p) {
    return he_guard(ctx, "he_top_logits: host allocation failed", [&]() -> int32_t {
    if (!ctx) return HE_ERR_BADARG;
    if (!p) return he_fail(ctx, HE_ERR_BADARG, "he_top_logits: null plan");
    if (!dtype_known(p->dtype)) return he_fail(ctx, HE_ERR_BADARG, "he_top_logits: unknown type %d", p->dtype);
    if (p->vocab == 0 || p->vocab > HE_VOCAB_MAX) return he_fail(ctx, HE_ERR_BADARG, "he_top_logits: %u logits outside 1..2^20", p->vocab);
    if (p->k == 0 || p->k > HE_TOP_MAX || p->k > p->vocab) return he_fail(ctx, HE_ERR_BADARG, "he_top_logits: k = %u outside 1..min(vocab, %d)", p->k, HE_TOP_MAX);
    if (!(p->tau > 0.0f) || p->tau == INFINITY) return he_fail(ctx, HE_ERR_BADARG, "he_top_logits: the temperature is not a positive number");
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
        if ((uint64_t)p->vocab * es > 32768) top_logits_kernel<T, 1024><<<p->rows, 1024, 0, ctx->stream>>>(a);
        else top_logits_kernel<T, 256><<<p->rows, 256, 0, ctx->stream>>>(a);
    });
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}
