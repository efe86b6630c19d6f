// Distillation loss against a teacher's top logits, mixed with the label's cross entropy, and its gradient.
//
// Of a row's logits z the indices that the teacher names are few: they and the label are handled apart, and the pass over the row
// sums the others.  The rest's probability then keeps its relative accuracy however small it is.  With c = log2(e) / tau all sums are of
// 2^(c (z - R)) for a reference R that is one of the row's logits, the largest: the difference comes first, so that its rounding is one of
// the difference, and the largest term is 1, whatever size the logits are.  (c z - R with R near c times the largest, one multiply-add, leaves
// the rounding of R in the exponent: past 2^7 from logits of 2^32 on, where the sum is 0 or infinite.)  With S the sum over the indices that
// are not named, Z over all, and S1, Z1 the same at temperature 1, the gradient at an index that is not named is
//   2^(c (z - R)) * (1 - alpha) tau (1/Z - P_rest/S) + 2^(log2(e) (z - R)) * alpha/Z1,
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

// Sums of a row's exponentials against a logit: value * 2^(c ref), and at temperature 1.  Without a term: ref = masked_from(tau), below
// any logit that counts.
struct Sums {
    float ref, value, value1;
};
struct Scale {
    float c, low;
    bool two;                       // there is a sum at temperature 1, and it is another
    __device__ __forceinline__ float number(float ref) const { return ref == low ? 0.0f : ref; }    // masked logits have no power against 0
    __device__ __forceinline__ float power(float d) const { return exp2_fast(d * c); }
    __device__ __forceinline__ float power1(float d) const { return exp2_fast(d * HE_LOG2E); }
};
__device__ __forceinline__ void raise(Sums& s, float ref, const Scale& scale) {
    if (ref > s.ref) {
        s.value *= scale.power(s.ref - ref);
        if (scale.two) s.value1 *= scale.power1(s.ref - ref);
        s.ref = ref;
    }
}
// Over a wavefront, then over the work group (a barrier before `w` is used again is the caller's)
__device__ __forceinline__ Sums wave_total(Sums s, const Scale& scale) {
    const float r = wave_max(s.ref);
    return {r, wave_sum(s.value * scale.power(s.ref - r)), scale.two ? wave_sum(s.value1 * scale.power1(s.ref - r)) : 0.0f};
}
template <int WAVES> __device__ __forceinline__ Sums total_of(const Sums* w, const Scale& scale, uint32_t lane) {
    return wave_total(lane < WAVES ? w[lane] : Sums{scale.low, 0, 0}, scale);
}

// What a row's threads share
template <int WAVES> struct RowShared {
    int32_t at[HE_TOP_MAX];         // the teacher's indices, -1: not there
    struct Entry {
        float t, z, p;              // value / tau, the student's logit, probability
        int32_t first;              // there, and the first with its index
    } entry[HE_TOP_MAX];
    float label_z;
    float teacher[5];               // P_rest, log of the sum over all (against the largest), log P_rest, the largest, whether anything is there
    int32_t put_at[HE_TOP_MAX + 1]; // where the gradient is written last, -1: nowhere; the label at the end
    float put[HE_TOP_MAX + 1];
    Sums part[WAVES];
    float factor[3];                // R and the factors of the two powers
    int32_t none;                   // neither term is there
};

// The teacher's entries of a row and what goes with them, by one wavefront, entry lane + 64 u; in LDS until the sums are there
template <class T, int WAVES> __device__ __forceinline__ void named_entries(const DistillArgs& a, RowShared<WAVES>& s, u64 row, const typename T::raw* z, uint32_t lane) {
    int32_t at[2];
    float t[2], zt[2], x[2];
#pragma unroll
    for (int u = 0; u < 2; u++) {
        const uint32_t j = lane + 64 * u;
        at[u] = -1;
        t[u] = zt[u] = -INFINITY;
        if (j < a.k) {
            const int32_t i = a.index[row * a.k + j];
            if (i >= 0 && (uint32_t)i < a.vocab) {
                at[u] = i;
                t[u] = a.values[row * a.k + j] / a.tau;
                zt[u] = to_float<T>(z[i]);
            }
        }
        s.at[j] = at[u];
    }
    const float r = a.rest ? a.rest[row] : -INFINITY, high = fmaxf(wave_max(fmaxf(t[0], t[1])), r), most = high == -INFINITY ? 0.0f : high;
#pragma unroll
    for (int u = 0; u < 2; u++) x[u] = exp2_fast((t[u] - most) * HE_LOG2E);
    const float xr = exp2_fast((r - most) * HE_LOG2E), top = wave_sum(x[0] + x[1]), all = top + xr, all_log = logf(all);
    const bool any = !(all == 0.0f);
    wave_sync();
#pragma unroll
    for (int u = 0; u < 2; u++) {
        const uint32_t j = lane + 64 * u;
        bool first = at[u] >= 0;
        if (first)
            for (uint32_t i = 0; i < j; i++)
                if (s.at[i] == at[u]) first = false;
        s.entry[j] = {t[u], zt[u], any ? x[u] / all : 0.0f, first};
    }
    if (lane == 0) {
        s.teacher[0] = any ? xr / all : 0.0f;
        s.teacher[1] = all_log;
        s.teacher[2] = xr >= top ? -log1pf(top / xr) : r - most - all_log;     // where the rest has nearly all, what it lacks
        s.teacher[3] = most;
        s.teacher[4] = any ? 1.0f : 0.0f;
    }
    wave_sync();
}

// One row a work group.  LOSS: writes the loss (and the statistics); GRAD: writes the gradient; REST: the rest counts as one outcome.
// GRAD alone takes the sums from the statistics.  16 bytes a lane at a time, sums against each lane's running reference.  Loss and gradient
// together need the row twice: V pieces a lane stay in registers between (16 of them: 64 of 128 registers; with 512 threads a work group 128
// KiB, two work groups to a compute unit, one of which reads or writes while the other adds up), what is beyond is read again, backwards,
// so that the caches still have some of it (of the half that is read again a fifth in the die's own, counted), and the gradient of long rows
// is written past them.
//
// 4096 x 131072 bf16, both: 473 us (4.5 TB/s of one read and one write); 467 when an exponent was one multiply-add (above).  With that, nothing
// kept 529 us, without its second pass going backwards past the caches 483; all of the row kept, one work group of 1024 threads to a compute
// unit, 680: nothing runs beside its sums.  4096 x 50021: 243 us (236 then, with nothing kept 283); 8192 x 10000, too short for it to
// matter: 94 us (92 then, with 16 pieces kept, fewer work groups at a time, 138).
template <class T, class R_, int THREADS, int V, bool LOSS, bool GRAD, bool REST> __global__ __launch_bounds__(THREADS, THREADS == 1024 && V == 0 ? 8 : 4) void distill_kernel(DistillArgs a) {
    using raw = typename T::raw;
    constexpr int N = Vec<T>::N, WAVES = THREADS / 64;
    __shared__ RowShared<WAVES> s;
    extern __shared__ uint32_t named[];                   // REST: a bit for each index that the teacher names
    const u64 row = blockIdx.x;
    const uint32_t t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const raw* z = (const raw*)a.z + row * a.ld_z;
    raw* grad = (raw*)a.grad + row * a.ld_grad;
    const R_ in{z, a.vocab};
    const uint32_t turns = (in.pieces() + THREADS - 1) / THREADS;
    const int32_t label = a.labels ? a.labels[row] : 0;
    auto no_gradient = [&]() {
        for (uint32_t p = 0; p < turns; p++) in.store(grad, p * THREADS + t, Vec<T>{{0, 0, 0, 0}}, false);
    };
    if (a.labels && label < 0) {
        if (LOSS && t == 0) a.loss[row] = 0;
        if (LOSS && a.stats && t < 4) a.stats[row * 4 + t] = 0;
        if (GRAD) no_gradient();
        return;
    }
    const uint32_t words = (a.vocab + 31) / 32;
    const bool ce_on = a.alpha > 0.0f && a.labels && (uint32_t)label < a.vocab;
    const Scale scale = {HE_LOG2E / a.tau, masked_from(a.tau), ce_on && a.tau != 1.0f};
    const uint32_t kept = min(turns, (uint32_t)V), read = turns - kept;
    Vec<T> one, other, row_[V ? V : 1];
    auto at = [&](uint32_t p, bool back) { return (kept + (back ? (p < read ? read - 1 - p : 0) : p)) * THREADS + t; };
    auto begin = [&](bool back) {
        one = in.load(at(0, back));
        other = in.load(at(1, back));
    };
    // f(number, piece) for all of the row: what is kept and what is read, two buffers in turn, each refilled as soon as it is taken; or
    // backwards
    auto keep = [&](auto&& f, int p) {
        if ((uint32_t)p >= turns) return;
        f(p * THREADS + t, row_[p]);
        // what comes of it now is not kept for the next time: two numbers of 16 bits take one register here, two there
        asm volatile("" : "+v"(row_[p].w[0]), "+v"(row_[p].w[1]), "+v"(row_[p].w[2]), "+v"(row_[p].w[3]));
    };
    auto each = [&](auto&& f, bool back) {
        if (!back)
#pragma unroll
            for (int p = 0; p < V; p++) keep(f, p);
        for (uint32_t p = 0; p < read; p += 2) {
            const Vec<T> x = one;
            one = in.load(at(p + 2, back));
            f(at(p, back), x);
            if (p + 1 >= read) break;
            const Vec<T> y = other;
            other = in.load(at(p + 3, back));
            f(at(p + 1, back), y);
        }
        if (back)
#pragma unroll
            for (int p = V - 1; p >= 0; p--) keep(f, p);
    };
#pragma unroll
    for (int p = 0; p < V; p++)
        if ((uint32_t)p < turns) row_[p] = in.load(p * THREADS + t);
    begin(false);
    if (REST && LOSS) {
        for (uint32_t i = t; i < words; i += THREADS) named[i] = 0;
        __syncthreads();
    }
    if (wave == 0) {
        named_entries<T, WAVES>(a, s, row, z, lane);
        if (REST && LOSS)
#pragma unroll
            for (int u = 0; u < 2; u++)
                if (const int32_t at = s.at[lane + 64 * u]; at >= 0) atomicOr(&named[at >> 5], 1u << (at & 31));
        if (lane == 0 && ce_on) s.label_z = to_float<T>(z[label]);
        wave_sync();                                      // where no sums are taken, no barrier lies between this and its other lanes' reading
    }
    Sums S = {scale.low, 0, 0};
    if (LOSS) {
        if (REST) __syncthreads();
        each([&](uint32_t v, const Vec<T>& piece) {
            const uint32_t base = in.base(v), past = v * N - base;
            float x[N];
#pragma unroll
            for (int i = 0; i < N; i++) x[i] = piece[i];
            uint32_t out = 0;
            if (REST) {
                out = named[base >> 5] >> (base & 31);
                if (past && (base & 31) > 32 - N && (base >> 5) + 1 < words) out |= named[(base >> 5) + 1] << (32 - (base & 31));   // across two words
            }
            out &= (1u << N) - 1;
            if (past) out |= (1u << min(past, (uint32_t)N)) - 1;
            if (out)
#pragma unroll
                for (int i = 0; i < N; i++)
                    if (out >> i & 1) x[i] = -INFINITY;
            float most = x[0];
#pragma unroll
            for (int i = 1; i < N; i++) most = fmaxf(most, x[i]);
            raise(S, most, scale);
            const float R = scale.number(S.ref);
#pragma unroll
            for (int i = 0; i < N; i++) S.value += scale.power(x[i] - R);
            if (scale.two)
#pragma unroll
                for (int i = 0; i < N; i++) S.value1 += scale.power1(x[i] - R);
        }, false);
        if (GRAD) begin(true);                            // on their way while the sums are joined
        S = wave_total(S, scale);
        if (lane == 0) s.part[wave] = S;
        __syncthreads();
    }
    if (wave == 0) {
        if (LOSS) S = total_of<WAVES>(s.part, scale, lane);
        else S = {a.stats[row * 4], a.stats[row * 4 + 1], a.stats[row * 4 + 2]};
        if (!scale.two) S.value1 = S.value;
        struct {
            int32_t at[2];
            float t[2], z[2], p[2];
            bool first[2];
        } e;
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const auto& n = s.entry[lane + 64 * u];
            e.at[u] = s.at[lane + 64 * u];
            e.t[u] = n.t;
            e.z[u] = n.z;
            e.p[u] = n.p;
            e.first[u] = n.first;
        }
        const float rest = s.teacher[0], all_log = s.teacher[1], rest_log = s.teacher[2], teacher_most = s.teacher[3], zl = ce_on ? s.label_z : 0.0f;
        // all: against the larger of the reference and the named logits' largest
        const auto power1 = [&](float d) { return scale.two ? scale.power1(d) : scale.power(d); };
        const float zt = fmaxf(REST && e.first[0] ? e.z[0] : -INFINITY, REST && e.first[1] ? e.z[1] : -INFINITY), M = fmaxf(S.ref, wave_max(zt)), R = scale.number(M);
        float x[2], x1[2];
#pragma unroll
        for (int u = 0; u < 2; u++) {
            x[u] = e.at[u] >= 0 ? scale.power(e.z[u] - R) : 0.0f;
            x1[u] = e.at[u] >= 0 ? power1(e.z[u] - R) : 0.0f;
        }
        const float top = wave_sum(REST ? (e.first[0] ? x[0] : 0.0f) + (e.first[1] ? x[1] : 0.0f) : 0.0f);
        const float top1 = wave_sum(REST ? (e.first[0] ? x1[0] : 0.0f) + (e.first[1] ? x1[1] : 0.0f) : 0.0f);
        const float down = scale.power(S.ref - M), down1 = power1(S.ref - M), others = S.value * down;
        const float Z = top + others, Z1 = top1 + S.value1 * down1;
        const bool dead = Z == 0.0f;                      // nothing but -infinity
        const bool kl_on = s.teacher[4] != 0.0f && a.alpha < 1.0f && !dead, ce = ce_on && !dead;
        if (LOSS) {
            // tau times the divergence, so that a logit's distance from the largest stands as it is.  What has no probability is left out; a
            // probability that is not a number, a teacher's that is not finite, makes the loss one that is none.
            const float log_z = logf(Z);
            float term = 0;
#pragma unroll
            for (int u = 0; u < 2; u++)
                if (e.p[u] != 0.0f) term += e.p[u] * (a.tau * (e.t[u] - teacher_most - all_log + log_z) - (e.z[u] - R));
            float kl = wave_sum(term);
            if (REST && rest != 0.0f) {
                const float lq = others >= top ? -a.tau * log1pf(top / others) : scale.number(S.ref) - R + a.tau * (logf(S.value) - log_z);
                kl += rest * (a.tau * rest_log - lq);
            }
            if (lane == 0) {
                float loss = kl_on ? (1.0f - a.alpha) * a.tau * kl : 0.0f;
                if (ce) loss += a.alpha * (logf(Z1) - (zl - R));
                a.loss[row] = loss;
                if (a.stats) {
                    a.stats[row * 4] = S.ref;
                    a.stats[row * 4 + 1] = S.value;
                    a.stats[row * 4 + 2] = S.value1;
                    a.stats[row * 4 + 3] = 0;
                }
            }
        }
        if (GRAD) {
            // a term that is not there adds nothing, though what it would be made of need not be a number
            const float weight = a.weights[row], wk = weight * (1.0f - a.alpha) * a.tau, wc = ce ? weight * a.alpha : 0.0f;
            const float fk = kl_on ? wk * (down / Z - (S.value > 0.0f ? rest / S.value : 0.0f)) : 0.0f, fc = ce ? wc * (down1 / Z1) : 0.0f;
            const float own = scale.number(S.ref), label_power = ce ? power1(zl - own) : 0.0f, label_power_k = ce ? scale.power(zl - own) : 0.0f;
            const bool alone = __all(e.at[0] != label && e.at[1] != label);
            if (lane == 0) {
                s.none = !kl_on && !ce;
                s.factor[0] = own;
                s.factor[1] = scale.two ? fk : fk + fc;   // one temperature: one power
                s.factor[2] = fc;
                s.put_at[HE_TOP_MAX] = ce && alone ? label : -1;
                s.put[HE_TOP_MAX] = (fk != 0.0f ? fk * label_power_k : 0.0f) + fc * label_power - wc;
            }
            // what stands at the named indices, and at the label's if it is none of them, is written once all else is
#pragma unroll
            for (int u = 0; u < 2; u++) {
                const uint32_t j = lane + 64 * u;
                float q = 0;
                if (e.first[u])
                    for (uint32_t i = 0; i < a.k; i++) q += s.at[i] == e.at[u] ? s.entry[i].p : 0.0f;
                float g = (kl_on ? wk * (x[u] / Z - q) : 0.0f) + (ce ? wc * (x1[u] / Z1) : 0.0f);
                if (ce && e.at[u] == label) g -= wc;
                s.put_at[j] = e.first[u] ? e.at[u] : -1;
                s.put[j] = g;
            }
        }
    }
    if (!GRAD) return;
    __syncthreads();
    if (s.none) return no_gradient();
    const float R = s.factor[0], fk = s.factor[1], fc = s.factor[2];
    each([&](uint32_t v, const Vec<T>& x) {
        float y[N];
#pragma unroll
        for (int i = 0; i < N; i++) y[i] = fk * scale.power(x[i] - R);
        if (scale.two)
#pragma unroll
            for (int i = 0; i < N; i++) y[i] = fmaf(fc, scale.power1(x[i] - R), y[i]);
        Vec<T> g;
        g.set(y);
        in.store(grad, v, g, THREADS > 256);
    }, LOSS);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // every wavefront's pieces are in memory before single elements of them are written anew
    __syncthreads();
    for (uint32_t i = t; i <= HE_TOP_MAX; i += THREADS)
        if (s.put_at[i] >= 0) grad[s.put_at[i]] = from_float<T>(s.put[i]);
}

static int32_t check(he_ctx* ctx, const he_distill_plan* p, const char* who) {
    if (!p) return he_fail(ctx, HE_ERR_BADARG, "%s: null plan", who);
    if (!dtype_known(p->dtype)) return he_fail(ctx, HE_ERR_BADARG, "%s: unknown type %d", who, p->dtype);
    if (p->vocab == 0 || p->vocab > HE_VOCAB_MAX) return he_fail(ctx, HE_ERR_BADARG, "%s: %u logits outside 1..2^20", who, p->vocab);
    if (p->k == 0 || p->k > HE_TOP_MAX) return he_fail(ctx, HE_ERR_BADARG, "%s: k = %u outside 1..%d", who, p->k, HE_TOP_MAX);
    if (!tau_fits(p->tau)) return he_fail(ctx, HE_ERR_BADARG, "%s: the temperature is not a number from 2^-60 to 2^60", who);
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

template <class R> struct Of { using type = R; };
template <bool LOSS, bool GRAD> static void launch(he_ctx* ctx, const he_distill_plan* p) {
    const DistillArgs a = {p->d_z, p->d_values, p->d_rest, p->d_row_weights, p->d_index, p->d_labels, p->d_loss, p->d_stats, p->d_grad, p->ld_z, p->ld_grad,
                           p->vocab, p->k, p->tau, p->alpha};
    const uint32_t lds = p->d_rest && LOSS ? (p->vocab + 31) / 32 * 4 : 0;
    with_dtype(p->dtype, [&](auto t) {
        using T = decltype(t);
        auto go = [&](auto threads, auto pieces, auto row) {
            constexpr int THREADS = decltype(threads)::value, V = decltype(pieces)::value;
            using R = typename decltype(row)::type;
            if (p->d_rest) distill_kernel<T, R, THREADS, V, LOSS, GRAD, true><<<p->rows, THREADS, lds, ctx->stream>>>(a);
            else distill_kernel<T, R, THREADS, V, LOSS, GRAD, false><<<p->rows, THREADS, 0, ctx->stream>>>(a);
        };
        using std::integral_constant;
        const uint64_t bytes = (uint64_t)p->vocab * dtype_bytes(p->dtype);
        // A row of at most one piece a lane by one wavefront, where several have only barriers more; up to four pieces a lane, with the four a
        // work group had otherwise, once there are rows for every wavefront slot to have one.  Loss and gradient in one call, one
        // wavefront and four: 6171 x 56 bf16 14.6 and 25.9 us, 4000 x 1000 f32 16.9 and 22.2, 256 x 1000 8.7 and 8.0.  (1024 lies between: four
        // wavefronts to each of 256 compute units; it was not measured.)
        const bool many = p->rows >= 1024;
        if (p->vocab < (uint32_t)Vec<T>::N) go(integral_constant<int, 64>{}, integral_constant<int, 0>{}, Of<ShortRow<T>>{});
        else if constexpr (LOSS && GRAD) {
            if (bytes <= 1024) go(integral_constant<int, 64>{}, integral_constant<int, 1>{}, Of<Row<T>>{});
            else if (bytes <= 4096 && many) go(integral_constant<int, 64>{}, integral_constant<int, 4>{}, Of<Row<T>>{});
            else if (bytes <= 4096) go(integral_constant<int, 256>{}, integral_constant<int, 1>{}, Of<Row<T>>{});
            else if (bytes <= 16384) go(integral_constant<int, 256>{}, integral_constant<int, 4>{}, Of<Row<T>>{});
            else if (bytes <= 32768) go(integral_constant<int, 256>{}, integral_constant<int, 0>{}, Of<Row<T>>{});
            else if (bytes <= 65536) go(integral_constant<int, 256>{}, integral_constant<int, 16>{}, Of<Row<T>>{});
            else go(integral_constant<int, 512>{}, integral_constant<int, 16>{}, Of<Row<T>>{});
        } else if (bytes > 32768) go(integral_constant<int, 1024>{}, integral_constant<int, 0>{}, Of<Row<T>>{});
        else if (bytes <= (many ? 4096 : 1024)) go(integral_constant<int, 64>{}, integral_constant<int, 0>{}, Of<Row<T>>{});
        else go(integral_constant<int, 256>{}, integral_constant<int, 0>{}, Of<Row<T>>{});
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
