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

// One row a work group.  An element's place in the order is one number of 64 bits, its key above the complement of its index, all
// different; the k-th largest is found a digit of 8 bits at a time, from the row's counts of that digit among the elements that
// agree with the digits before.  Then the elements from it on are gathered and put in order by counting for each how many are
// larger, and the rest is summed against its own maximum.
template <class T> __global__ __launch_bounds__(256) void top_logits_kernel(TopArgs a) {
    using raw = typename T::raw;
    __shared__ uint32_t bins[256];
    __shared__ u64 found[HE_TOP_MAX];
    __shared__ float room[4];
    __shared__ uint32_t digit, left, got;
    const u64 row = blockIdx.x;
    const raw* z = (const raw*)a.z + row * a.ld_z;
    const uint32_t t = threadIdx.x;
    u64 prefix = 0;
    uint32_t want = a.k;                       // how many of the elements that agree with `prefix` are still wanted
    for (int shift = 56; shift >= 0; shift -= 8) {
        bins[t] = 0;
        __syncthreads();
        for (uint32_t i = t; i < a.vocab; i += 256) {
            const u64 c = (u64)order_key(to_float<T>(z[i])) << 32 | (uint32_t)~i;
            if (shift == 56 || c >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&bins[(uint32_t)(c >> shift) & 255], 1u);
        }
        __syncthreads();
        if (t == 0) {
            uint32_t n = want, d = 255;
            while (bins[d] < n) n -= bins[d--];
            digit = d;
            left = n;
        }
        __syncthreads();
        prefix |= (u64)digit << shift;
        want = left;
        __syncthreads();
    }
    if (t == 0) got = 0;
    __syncthreads();
    float most = -INFINITY;
    for (uint32_t i = t; i < a.vocab; i += 256) {
        const float v = to_float<T>(z[i]);
        const u64 c = (u64)order_key(v) << 32 | (uint32_t)~i;
        if (c >= prefix) found[atomicAdd(&got, 1u)] = c;    // exactly k
        else most = fmaxf(most, v);
    }
    most = group_max<4>(most, room);
    __syncthreads();
    if (t < a.k) {
        const u64 c = found[t];
        uint32_t place = 0;
        for (uint32_t j = 0; j < a.k; j++) place += found[j] > c;
        const uint32_t i = ~(uint32_t)c;
        a.values[row * a.k + place] = to_float<T>(z[i]);
        a.index[row * a.k + place] = (int32_t)i;
    }
    if (!a.rest) return;
    const float scale = HE_LOG2E / a.tau, at = most == -INFINITY ? 0.0f : most;
    float sum = 0;
    for (uint32_t i = t; i < a.vocab; i += 256) {
        const float v = to_float<T>(z[i]);
        if (((u64)order_key(v) << 32 | (uint32_t)~i) < prefix) sum += exp2_fast((v - at) * scale);
    }
    sum = group_sum<4>(sum, room);
    if (t == 0) a.rest[row] = logf(sum) + at / a.tau;
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
    with_dtype(p->dtype, [&](auto t) { top_logits_kernel<decltype(t)><<<p->rows, 256, 0, ctx->stream>>>(a); });
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}
