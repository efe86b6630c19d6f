// Log probabilities of given tokens, entropy and alternatives of rows of logits, and their gradient.
//
// With c = log2(e) / tau, M the largest logit that counts and e_i = 2^(c (z_i - M)): S = sum e_i and Q = sum e_i (z_i - M) c, so that
// log p_i = (z_i - M) / tau - ln S and the entropy is ln S - ln 2 Q / S, two terms of one sign.
#include "plain.h"

struct LogprobArgs {
    const void* z;
    const int32_t* tokens;
    float *logp, *entropy, *values;
    const int32_t* index;
    float4* stats;
    u64 ld_z;
    uint32_t vocab, k;
    float tau;
};

struct Totals {
    float ref, sum, less;          // M, S, Q; M is masked_from(tau) where there is no term
};
__device__ __forceinline__ float weight_of(float d) { return d < -200.0f ? 0.0f : exp2_fast(d); }
// Sums against another reference, which is not below theirs
__device__ __forceinline__ Totals against(const Totals& t, float ref, float c) {
    const float d = t.ref == ref ? 0.0f : (t.ref - ref) * c, f = weight_of(d);
    return {ref, f == 0.0f ? 0.0f : t.sum * f, f == 0.0f ? 0.0f : (t.less + t.sum * d) * f};
}

// A row a work group
template <class T> __global__ __launch_bounds__(256) void logprobs_kernel(LogprobArgs a) {
    using raw = typename T::raw;
    __shared__ float room[8];
    const u64 row = blockIdx.x;
    const raw* z = (const raw*)a.z + row * a.ld_z;
    const float c = HE_LOG2E / a.tau, low = masked_from(a.tau);
    Totals t = {low, 0, 0};
    bool none = false;                                    // a logit that leaves no distribution
    for (uint32_t i = threadIdx.x; i < a.vocab; i += 256) {
        const float v = to_float<T>(z[i]);
        if (v <= low) continue;
        if (!(v < -low)) none = true;
        if (v > t.ref) t = against(t, v, c);
        const float d = (v - t.ref) * c, e = weight_of(d);
        t.sum += e;
        if (e != 0.0f) t.less += e * d;
    }
    none = __syncthreads_or(none);
    const float ref = group_max<4>(t.ref, room);
    t = against(t, ref, c);
    group_sum2<4>(t.sum, t.less, room);
    const float log_sum = logf(t.sum), entropy = none ? NAN : t.sum == 0.0f ? 0.0f : log_sum - HE_LN2 * t.less / t.sum;
    auto log_of = [&](float v) { return none ? NAN : v <= low ? -INFINITY : (v - ref) / a.tau - log_sum; };
    if (threadIdx.x == 0) {
        if (a.logp) {
            const int32_t at = a.tokens[row];
            a.logp[row] = (uint32_t)at < a.vocab ? log_of(to_float<T>(z[at])) : 0.0f;
        }
        if (a.entropy) a.entropy[row] = entropy;
        if (a.stats) a.stats[row] = {none ? NAN : t.sum == 0.0f ? 0.0f : ref, none ? NAN : t.sum, entropy, 0};
    }
    for (uint32_t i = threadIdx.x; i < a.k; i += 256) a.values[row * a.k + i] = log_of(to_float<T>(z[a.index[row * a.k + i]]));
}

extern "C" int32_t he_work_token_logprobs(const he_ctx* ctx, const he_logprobs_plan* p, uint64_t* h_bytes) {
    return he_guard(ctx, "he_work_token_logprobs: host allocation failed", [&]() -> int32_t {
    if (!ctx || !h_bytes) return HE_ERR_BADARG;
    HE_REFUSE(const_cast<he_ctx*>(ctx), "he_work_token_logprobs", refuse_logprobs(p, true));
    *h_bytes = logprobs_work(p);
    return HE_OK;
    });
}

extern "C" int32_t he_token_logprobs(he_ctx* ctx, const he_logprobs_plan* p) {
    return he_guard(ctx, "he_token_logprobs: host allocation failed", [&]() -> int32_t {
    if (!ctx) return HE_ERR_BADARG;
    HE_REFUSE(ctx, "he_token_logprobs", refuse_logprobs(p));
    if (p->rows == 0) return HE_OK;
    const OnDevice device(ctx);
    HE_HIP(ctx, device.status);
    if (p->k) {
        const he_top_plan top = {p->rows, p->vocab, p->k, p->dtype, p->tau, p->d_z, p->ld_z, p->d_values, p->d_index, nullptr};
        const int32_t rc = he_top_logits(ctx, &top);
        if (rc != HE_OK) return rc;
    }
    const LogprobArgs a = {p->d_z, p->d_tokens, p->d_logp, p->d_entropy, p->d_values, p->d_index, (float4*)p->d_stats, p->ld_z, p->vocab, p->k, p->tau};
    with_dtype(p->dtype, [&](auto t) { logprobs_kernel<decltype(t)><<<p->rows, 256, 0, ctx->stream>>>(a); });
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}

// ---- gradient

struct LogprobGradArgs {
    const void* z;
    const int32_t* tokens;
    const float4* stats;
    const float *logp_weights, *entropy_weights;
    void* grad;
    u64 ld_z, ld_grad;
    uint32_t vocab;
    float tau;
};

// A row a work group: of x = (z - M) c it is p (A + B x) with two numbers a row, and the token's own term.
template <class T> __global__ __launch_bounds__(256) void logprobs_grad_kernel(LogprobGradArgs a) {
    using raw = typename T::raw;
    const u64 row = blockIdx.x;
    const raw* z = (const raw*)a.z + row * a.ld_z;
    raw* grad = (raw*)a.grad + row * a.ld_grad;
    const float c = HE_LOG2E / a.tau, low = masked_from(a.tau);
    const float4 stats = a.stats[row];
    const int32_t token = a.tokens ? a.tokens[row] : -1;
    float wl = a.logp_weights && (uint32_t)token < a.vocab ? a.logp_weights[row] : 0.0f;
    if (wl != 0.0f && to_float<T>(z[token]) <= low) wl = 0.0f;
    const float wh = a.entropy_weights ? a.entropy_weights[row] : 0.0f;
    __syncthreads();                                      // the token's logit has been read, where the gradient lies over it
    const bool zero = (wl == 0.0f && wh == 0.0f) || stats.y == 0.0f;
    const float by = 1.0f / (stats.y * a.tau);
    const float A = -(wl + wh * (stats.z - logf(stats.y))) * by, B = -wh * HE_LN2 * by;
    for (uint32_t i = threadIdx.x; i < a.vocab; i += 256) {
        const float v = to_float<T>(z[i]), d = (v - stats.x) * c, e = weight_of(d);
        float y = v <= low || e == 0.0f ? 0.0f : e * fmaf(B, d, A);
        if ((int32_t)i == token) y += wl / a.tau;
        grad[i] = from_float<T>(zero ? 0.0f : y);
    }
}

extern "C" int32_t he_token_logprobs_grad(he_ctx* ctx, const he_logprobs_grad_plan* p) {
    return he_guard(ctx, "he_token_logprobs_grad: host allocation failed", [&]() -> int32_t {
    if (!ctx) return HE_ERR_BADARG;
    HE_REFUSE(ctx, "he_token_logprobs_grad", refuse_logprobs_grad(p));
    if (p->rows == 0) return HE_OK;
    const OnDevice device(ctx);
    HE_HIP(ctx, device.status);
    const LogprobGradArgs a = {p->d_z, p->d_tokens, (const float4*)p->d_stats, p->d_logp_weights, p->d_entropy_weights, p->d_grad, p->ld_z, p->ld_grad, p->vocab, p->tau};
    with_dtype(p->dtype, [&](auto t) { logprobs_grad_kernel<decltype(t)><<<p->rows, 256, 0, ctx->stream>>>(a); });
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}
