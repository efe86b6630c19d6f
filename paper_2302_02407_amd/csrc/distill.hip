// Distillation loss against a teacher's top logits, mixed with the label's cross entropy, and its gradient.
//
// Of a row's logits z the indices that the teacher names are few: they and the label are handled one a thread, and the pass over the
// row sums the others against their own maximum m: S = sum exp((z - m)/tau), S1 = sum exp(z - m).  The rest's probability then keeps
// its relative accuracy however small it is.  With the sums over all, Z and Z1 (against the same m), the gradient at an index that
// the teacher does not name is
//   exp((z - m)/tau) * (1 - alpha) tau (1/Z - P_rest/S) + exp(z - m) * alpha/Z1,
// two factors a row.  Where no rest is given (P_rest = 0) nothing has to be told apart and the pass sums over all.
#include "plain.h"

struct DistillArgs {
    const void* z;
    const float *values, *rest, *weights;
    const int32_t *index, *labels;
    float *loss, *stats;
    void* grad;
    u64 ld_z, ld_grad;
    uint32_t vocab, k;
    float tau, alpha;
};

// What a row's threads share
struct RowShared {
    float t[HE_TOP_MAX], zt[HE_TOP_MAX], p[HE_TOP_MAX];   // the teacher's value / tau, the student's logit, the teacher's probability
    int32_t at[HE_TOP_MAX];                               // index, -1: not there
    float room[16];
};

// Maximum and sums over the indices that the teacher names: thread j < k holds entry j
struct Named {
    bool live;        // entry j is there and the first with its index
    float z;          // student's logit
};

// LOSS: writes the loss (and the statistics); GRAD: writes the gradient.  GRAD alone takes m, S, S1 from the statistics.
template <class T, bool LOSS, bool GRAD, bool REST> __global__ __launch_bounds__(256) void distill_kernel(DistillArgs a) {
    using raw = typename T::raw;
    __shared__ RowShared s;
    extern __shared__ uint32_t named[];                   // REST: a bit for each index that the teacher names
    const u64 row = blockIdx.x;
    const uint32_t t = threadIdx.x;
    const raw* z = (const raw*)a.z + row * a.ld_z;
    raw* grad = (raw*)a.grad + row * a.ld_grad;
    const int32_t label = a.labels ? a.labels[row] : 0;
    const float weight = GRAD ? a.weights[row] : 0.0f;
    if (a.labels && label < 0) {
        if (LOSS && t == 0) a.loss[row] = 0;
        if (LOSS && a.stats && t < 4) a.stats[row * 4 + t] = 0;
        if (GRAD) for (uint32_t i = t; i < a.vocab; i += 256) grad[i] = 0;
        return;
    }
    const float inv_tau = 1.0f / a.tau, c = HE_LOG2E / a.tau;
    const uint32_t words = (a.vocab + 31) / 32;
    if (REST) for (uint32_t i = t; i < words; i += 256) named[i] = 0;
    float tv = -INFINITY, zt = -INFINITY;
    int32_t at = -1;
    if (t < a.k) {
        at = a.index[row * a.k + t];
        if (at < 0 || (uint32_t)at >= a.vocab) at = -1;
        if (at >= 0) {
            tv = a.values[row * a.k + t] / a.tau;
            zt = to_float<T>(z[at]);
        }
        s.at[t] = at;
        s.t[t] = tv;
        s.zt[t] = zt;
    }
    __syncthreads();
    bool first = at >= 0;                                 // the first entry with its index
    if (t < a.k && at >= 0) {
        for (uint32_t j = 0; j < t; j++) first = first && s.at[j] != at;
        if (REST) atomicOr(&named[at >> 5], 1u << (at & 31));
    }
    // the teacher: P_j, P_rest
    const float tr = REST ? a.rest[row] : -INFINITY;
    const float tm = fmaxf(group_max<4>(tv, s.room), tr), tm0 = tm == -INFINITY ? 0.0f : tm;
    const float et = exp2_fast((tv - tm0) * HE_LOG2E), er = exp2_fast((tr - tm0) * HE_LOG2E);
    const float ttop = group_sum<4>(et, s.room), tall = ttop + er;
    const bool taught = !(tall == 0.0f);
    const float p = taught ? et / tall : 0.0f, pr = taught ? er / tall : 0.0f;
    if (t < a.k) s.p[t] = p;
    __syncthreads();
    const bool kl_on = taught && a.alpha < 1.0f, ce_on = a.alpha > 0.0f && a.labels && (uint32_t)label < a.vocab;
    const float zl = ce_on ? to_float<T>(z[label]) : 0.0f;
    // the student's indices that are not named (all of them without a rest)
    float m, S, S1;
    if (LOSS) {
        m = -INFINITY;
        for (uint32_t i = t; i < a.vocab; i += 256)
            if (!REST || !(named[i >> 5] >> (i & 31) & 1)) m = fmaxf(m, to_float<T>(z[i]));
        m = group_max<4>(m, s.room);
    } else {
        m = a.stats[row * 4];
        S = a.stats[row * 4 + 1];
        S1 = a.stats[row * 4 + 2];
    }
    const float m0 = m == -INFINITY ? 0.0f : m;
    if (LOSS) {
        S = S1 = 0;
        for (uint32_t i = t; i < a.vocab; i += 256)
            if (!REST || !(named[i >> 5] >> (i & 31) & 1)) {
                const float d = to_float<T>(z[i]) - m0;
                S += exp2_fast(d * c);
                S1 += exp2_fast(d * HE_LOG2E);
            }
        S = group_sum<4>(S, s.room);
        S1 = group_sum<4>(S1, s.room);
    }
    // all: against M, the larger of the two maxima
    const float mt = group_max<4>(REST ? zt : -INFINITY, s.room), M = fmaxf(m, mt), M0 = M == -INFINITY ? 0.0f : M;
    const float top = group_sum<4>(REST && first ? exp2_fast((zt - M0) * c) : 0.0f, s.room);
    const float top1 = group_sum<4>(REST && first ? exp2_fast((zt - M0) * HE_LOG2E) : 0.0f, s.room);
    const float down = exp2_fast((m0 - M0) * c), down1 = exp2_fast((m0 - M0) * HE_LOG2E);
    const float Z = top + S * down, Z1 = top1 + S1 * down1;
    const bool dead = Z == 0.0f;                          // nothing but -infinity
    if (LOSS) {
        const float term = p > 0.0f ? p * ((tv - tm0 - logf(tall)) - ((zt - M0) * inv_tau - logf(Z))) : 0.0f;
        float kl = group_sum<4>(term, s.room);
        if (t == 0) {
            if (REST && pr > 0.0f) {
                const float lp = er >= ttop ? -log1pf(ttop / er) : tr - tm0 - logf(tall);
                const float lq = S * down >= top ? -log1pf(top / (S * down)) : (m0 - M0) * inv_tau + logf(S) - logf(Z);
                kl += pr * (lp - lq);
            }
            float loss = 0;
            if (kl_on && !dead) loss = (1.0f - a.alpha) * a.tau * a.tau * kl;
            if (ce_on && !dead) loss += a.alpha * (logf(Z1) - (zl - M0));
            a.loss[row] = loss;
            if (a.stats) {
                a.stats[row * 4] = m;
                a.stats[row * 4 + 1] = S;
                a.stats[row * 4 + 2] = S1;
                a.stats[row * 4 + 3] = 0;
            }
        }
    }
    if (GRAD) {
        const float wk = kl_on && !dead ? weight * (1.0f - a.alpha) * a.tau : 0.0f, wc = ce_on && !dead ? weight * a.alpha : 0.0f;
        const float fk = dead ? 0.0f : wk * (down / Z - (S > 0.0f ? pr / S : 0.0f)), fc = dead ? 0.0f : wc * (down1 / Z1);
        for (uint32_t i = t; i < a.vocab; i += 256) {
            const float d = to_float<T>(z[i]) - m0;
            const float g = (fk != 0.0f ? fk * exp2_fast(d * c) : 0.0f) + (fc != 0.0f ? fc * exp2_fast(d * HE_LOG2E) : 0.0f);
            grad[i] = from_float<T>(g);
        }
        __syncthreads();
        // the named indices and the label, each by one thread
        if (t < a.k && first) {
            float q = 0;
            for (uint32_t j = 0; j < a.k; j++) q += s.at[j] == at ? s.p[j] : 0.0f;
            float g = dead ? 0.0f : wk * (exp2_fast((zt - M0) * c) / Z - q) + wc * (exp2_fast((zt - M0) * HE_LOG2E) / Z1);
            if (ce_on && at == label) g -= wc;
            grad[at] = from_float<T>(g);
        }
        if (ce_on && t == 255) {
            bool alone = true;
            for (uint32_t j = 0; j < a.k; j++) alone = alone && s.at[j] != label;
            if (alone && !dead) {
                const float d = zl - m0;
                grad[label] = from_float<T>((fk != 0.0f ? fk * exp2_fast(d * c) : 0.0f) + fc * exp2_fast(d * HE_LOG2E) - wc);
            }
        }
    }
}

static int32_t check(he_ctx* ctx, const he_distill_plan* p, const char* who) {
    if (!p) return he_fail(ctx, HE_ERR_BADARG, "%s: null plan", who);
    if (!dtype_known(p->dtype)) return he_fail(ctx, HE_ERR_BADARG, "%s: unknown type %d", who, p->dtype);
    if (p->vocab == 0 || p->vocab > HE_VOCAB_MAX) return he_fail(ctx, HE_ERR_BADARG, "%s: %u logits outside 1..2^20", who, p->vocab);
    if (p->k == 0 || p->k > HE_TOP_MAX) return he_fail(ctx, HE_ERR_BADARG, "%s: k = %u outside 1..%d", who, p->k, HE_TOP_MAX);
    if (!(p->tau > 0.0f) || p->tau == INFINITY) return he_fail(ctx, HE_ERR_BADARG, "%s: the temperature is not a positive number", who);
    if (!(p->alpha >= 0.0f && p->alpha <= 1.0f)) return he_fail(ctx, HE_ERR_BADARG, "%s: alpha outside 0..1", who);
    if (p->rows > HE_ROWS_MAX) return he_fail(ctx, HE_ERR_BADARG, "%s: more than 2^21 rows", who);
    if (p->alpha > 0.0f && !p->d_labels && p->rows) return he_fail(ctx, HE_ERR_BADARG, "%s: alpha without labels", who);
    return HE_OK;
}

// Operands of a call with rows in it; outputs: the gradient, or the loss and what is given beside it
static int32_t check_operands(he_ctx* ctx, const he_distill_plan* p, const char* who, bool loss) {
    const uint32_t es = dtype_bytes(p->dtype);
    const bool grad = !loss || p->d_grad;
    if (!p->d_z || !p->d_values || !p->d_index || (loss ? !p->d_loss : !p->d_stats || !p->d_grad) || (grad && !p->d_row_weights))
        return he_fail(ctx, HE_ERR_BADARG, "%s: null argument", who);
    if (!ld_fits(p->ld_z, p->vocab) || (grad && !ld_fits(p->ld_grad, p->vocab))) return he_fail(ctx, HE_ERR_BADARG, "%s: an ld is below the row's length or above 2^28", who);
    if (((uintptr_t)p->d_z | (grad ? (uintptr_t)p->d_grad : 0)) & (es - 1) ||
        ((uintptr_t)p->d_values | (uintptr_t)p->d_index | (uintptr_t)p->d_rest | (uintptr_t)p->d_labels | (uintptr_t)p->d_stats |
         (loss ? (uintptr_t)p->d_loss : 0) | (grad ? (uintptr_t)p->d_row_weights : 0)) & 3)
        return he_fail(ctx, HE_ERR_BADARG, "%s: a pointer is not aligned to its elements", who);
    const uint64_t nk = (uint64_t)p->rows * p->k * 4, nr = (uint64_t)p->rows * 4;
    const void* stats_in = loss ? nullptr : p->d_stats;
    const struct { const void* d; uint64_t n; } in[7] = {{p->d_z, span(p->rows, p->vocab, p->ld_z, es)}, {p->d_values, nk}, {p->d_index, nk}, {p->d_rest, nr},
                                                         {p->d_labels, nr}, {grad ? p->d_row_weights : nullptr, nr}, {stats_in, 4 * nr}},
        out[3] = {{grad ? p->d_grad : nullptr, grad ? span(p->rows, p->vocab, p->ld_grad, es) : 0}, {loss ? p->d_loss : nullptr, nr}, {loss ? p->d_stats : nullptr, 4 * nr}};
    for (int o = 0; o < 3; o++) {
        for (int i = 0; i < 7; i++)
            if (!(o == 0 && i == 0 && p->d_grad == p->d_z && p->ld_grad == p->ld_z) && overlap(out[o].d, out[o].n, in[i].d, in[i].n))
                return he_fail(ctx, HE_ERR_BADARG, "%s: an output overlaps an input", who);
        for (int i = 0; i < o; i++)
            if (overlap(out[o].d, out[o].n, out[i].d, out[i].n)) return he_fail(ctx, HE_ERR_BADARG, "%s: two outputs overlap", who);
    }
    return HE_OK;
}

template <bool LOSS, bool GRAD> static void launch(he_ctx* ctx, const he_distill_plan* p) {
    const DistillArgs a = {p->d_z, p->d_values, p->d_rest, p->d_row_weights, p->d_index, p->d_labels, p->d_loss, p->d_stats, p->d_grad, p->ld_z, p->ld_grad,
                           p->vocab, p->k, p->tau, p->alpha};
    const uint32_t lds = p->d_rest ? (p->vocab + 31) / 32 * 4 : 0;
    with_dtype(p->dtype, [&](auto t) {
        using T = decltype(t);
        if (p->d_rest) distill_kernel<T, LOSS, GRAD, true><<<p->rows, 256, lds, ctx->stream>>>(a);
        else distill_kernel<T, LOSS, GRAD, false><<<p->rows, 256, 0, ctx->stream>>>(a);
    });
}

extern "C" int32_t he_distill_loss(he_ctx* ctx, const he_distill_plan* p) {
    return he_guard(ctx, "he_distill_loss: host allocation failed", [&]() -> int32_t {
    if (!ctx) return HE_ERR_BADARG;
    int32_t rc = check(ctx, p, "he_distill_loss");
    if (rc != HE_OK || p->rows == 0) return rc;
    if ((rc = check_operands(ctx, p, "he_distill_loss", true)) != HE_OK) return rc;
    if (p->d_grad) launch<true, true>(ctx, p);
    else launch<true, false>(ctx, p);
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}

extern "C" int32_t he_distill_grad(he_ctx* ctx, const he_distill_plan* p) {
    return he_guard(ctx, "he_distill_grad: host allocation failed", [&]() -> int32_t {
    if (!ctx) return HE_ERR_BADARG;
    int32_t rc = check(ctx, p, "he_distill_grad");
    if (rc != HE_OK || p->rows == 0) return rc;
    if ((rc = check_operands(ctx, p, "he_distill_grad", false)) != HE_OK) return rc;
    launch<false, true>(ctx, p);
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}
