// Log probabilities of given tokens, entropy and alternatives of rows of logits, and their gradient.
//
// With c = log2(e) / tau, M the largest logit that counts and e_i = 2^(c (z_i - M)): S = sum e_i and Q = sum e_i (z_i - M) c, so that
// log p_i = (z_i - M) / tau - ln S and the entropy is ln S - ln 2 Q / S, two terms of one sign.
#include "top.h"

struct LogprobArgs {
    const void* z;
    const int32_t* tokens;
    float *logp, *entropy, *values;
    int32_t* index;
    float4* stats;
    u64 ld_z;
    uint32_t vocab, k;
    float tau;
    uint32_t parts, len;           // a row's parts and how many elements each of them has (the last: what is left)
    u64* places;                   // [rows][parts][k], in order
    float4* totals;                // [rows][parts]
};

struct Totals {
    float ref, sum, less;          // M, S, Q; M is masked_from(tau) where there is no term
};
// Masked logits have no power against 0; and a power below 2^-1000 is as good as that one, which an infinite difference is not in Q
__device__ __forceinline__ float reference(float ref, float low) { return ref == low ? 0.0f : ref; }
#define LEAST_POWER -1000.0f
// Sums against another reference, which is not below theirs
__device__ __forceinline__ Totals against(const Totals& t, float ref, float c) {
    const float d = t.ref == ref ? 0.0f : fmaxf((t.ref - ref) * c, LEAST_POWER), f = exp2_fast(d);
    return {ref, f == 0.0f && t.sum == t.sum ? 0.0f : t.sum * f, f == 0.0f ? 0.0f : fmaf(t.sum, d, t.less) * f};
}

// What a row's totals say: S is a NaN where there is no distribution
struct Distribution {
    float ref, sum, log_sum, entropy, low, tau;
    bool none;
    __device__ __forceinline__ Distribution(const Totals& t, float low_, float tau_) : ref(reference(t.ref, low_)), sum(t.sum), low(low_), tau(tau_) {
        none = sum != sum || t.ref >= -low_;
        log_sum = logf(sum);
        entropy = none ? NAN : sum == 0.0f ? 0.0f : log_sum - HE_LN2 * t.less / sum;
        if (none) sum = NAN;
    }
    __device__ __forceinline__ float log_of(float v) const { return none ? NAN : v <= low ? -INFINITY : (v - ref) / tau - log_sum; }
    __device__ __forceinline__ float4 stats() const { return {none ? NAN : sum == 0.0f ? 0.0f : ref, sum, entropy, 0}; }
};

// The token's own and the row's numbers, by one thread
template <class T> __device__ __forceinline__ void write_row(const LogprobArgs& a, u64 row, const Distribution& d) {
    if (a.logp) {
        const int32_t at = a.tokens[row];
        a.logp[row] = (uint32_t)at < a.vocab ? d.log_of(to_float<T>(((const typename T::raw*)a.z)[row * a.ld_z + at])) : 0.0f;
    }
    if (a.entropy) a.entropy[row] = d.entropy;
    if (a.stats) a.stats[row] = d.stats();
}

// One row, or a part of one, a work group, read once, 16 bytes a lane at a time: every element into its lane's sums against the lane's running maximum,
// (z - M) c by a difference and a product, so that logits of any size lose nothing.  TOP: pieces with an element that reaches a threshold are also set
// aside, as top_logits_kernel does (toplogits.hip); what is set aside only has to be put in order, the sums have it already.  HELD: a row of at most four pieces a
// lane stays in registers, and one threshold, taken when it is all there, says which elements are put in order.
//
// 2048 x 131072 bf16, k = 8: 106 us (5.0 TB/s of one reading), vector instructions 96% of its cycles under the counters, 13.4 an element, one exponential among them;
// as two passes, order and sums, 413.  8192 x 500, k = 30, 20 us, without HELD 30.
template <class T, int THREADS, int ROOM, bool HELD, bool PARTED> __global__ __launch_bounds__(THREADS, 4) void logprobs_kernel(LogprobArgs a) {
    using raw = typename T::raw;
    constexpr int N = Vec<T>::N, WAVES = THREADS / 64;
    constexpr bool TOP = ROOM != 0;
    __shared__ std::conditional_t<TOP, TopShared<THREADS, TOP ? ROOM : 1>, char> shared;
    __shared__ float room[2 * WAVES];
    const u64 row = PARTED ? blockIdx.y : blockIdx.x;
    const uint32_t part = PARTED ? blockIdx.x : 0, from = PARTED ? part * a.len : 0, n = PARTED ? min(a.len, a.vocab - from) : a.vocab;
    const raw* z = (const raw*)a.z + row * a.ld_z + from;
    const uint32_t t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const Row<T> in{z, n};
    const uint32_t vecs = in.pieces(), turns = (vecs + THREADS - 1) / THREADS;
    const uint32_t full = max(1u, min((uint32_t)WAVES, vecs / 64)), r = (a.k + full - 1) / full;      // a lane without a piece counts as -infinity
    const float c = HE_LOG2E / a.tau, low = masked_from(a.tau);
    if constexpr (TOP)
        if (t == 0) shared.got = shared.kept = 0;
    Totals s = {low, 0, 0};
    float high = -INFINITY, least = -INFINITY;
    auto turn = [&](uint32_t p, Vec<T>& buf) {           // two buffers in turn, each refilled as soon as it is taken
        const uint32_t v = p * THREADS + t;
        const uint32_t base = in.base(v), past = v * N - base;       // elements of it that are another piece's
        Vec<T> x = buf;
        if (!HELD) buf = in.load(v + 2 * THREADS);
        float e[N];
#pragma unroll
        for (int i = 0; i < N; i++) e[i] = x[i];
        if (past)
#pragma unroll
            for (int i = 0; i < N; i++)
                if ((uint32_t)i < past) {
                    if (TOP && !HELD) x.set(i, -INFINITY);
                    e[i] = -INFINITY;
                }
        float mx = e[0];
#pragma unroll
        for (int i = 1; i < N; i++) mx = fmaxf(mx, e[i]);
        if constexpr (TOP) high = fmaxf(high, mx);
        if constexpr (TOP && !HELD) {
            if (((p + 1) & (p + 2)) == 0) least = reached_by_all<WAVES>(high, r, full, lane, wave, shared.tw[__builtin_ctz(p + 2) & 1]);
            if (!(mx < least) && (mx != -INFINITY || base < a.k)) {
                const uint32_t to = atomicAdd(&shared.got, 1u);
                if (to < ROOM) {
                    shared.aside[to] = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
                    shared.which[to] = base | min(past, 15u) << 24;
                }
            }
        }
        if (mx > s.ref) s = against(s, mx, c);
        const float ref = reference(s.ref, low);
#pragma unroll
        for (int i = 0; i < N; i++) {
            const float d = (e[i] - ref) * c, f = exp2_fast(d);
            s.sum += f;
            s.less = fmaf(f, fmaxf(d, LEAST_POWER), s.less);
        }
    };
    Vec<T> held[HELD ? 4 : 2];
    if constexpr (HELD) {
#pragma unroll
        for (uint32_t p = 0; p < 4; p++)
            if (p < turns) held[p] = in.load(p * THREADS + t);
#pragma unroll
        for (uint32_t p = 0; p < 4; p++)
            if (p < turns) turn(p, held[p]);
    } else {
        held[0] = in.load(t);
        held[1] = in.load(THREADS + t);
        for (uint32_t p = 0; p < turns; p += 2) {
            turn(p, held[0]);
            if (p + 1 < turns) turn(p + 1, held[1]);
        }
    }
    const float ref = group_max<WAVES>(s.ref, room);
    s = against(s, ref, c);
    group_sum2<WAVES>(s.sum, s.less, room);
    const Distribution d(s, low, a.tau);
    if (t == 0) {
        if (PARTED) a.totals[row * a.parts + part] = {s.ref, s.sum, s.less, 0};
        else write_row<T>(a, row, d);
    }
    if constexpr (TOP) {
        __syncthreads();                                 // all is set aside, and the slots of tw have been read
        const uint32_t got = HELD ? 0 : shared.got;
        uint32_t kept = 0;
        bool exact = got > ROOM || d.sum != d.sum;       // a NaN stands above every number, and a threshold does not see it
        if (!exact) {
            least = reached_by_all<WAVES>(high, r, full, lane, wave, shared.tw[0]);
            if constexpr (HELD)
#pragma unroll
                for (uint32_t p = 0; p < 4; p++) {
                    if (p >= turns) break;
                    const uint32_t piece = p * THREADS + t, base = in.base(piece), past = piece * N - base;
#pragma unroll
                    for (uint32_t i = 0; i < (uint32_t)N; i++)
                        if (const float v = held[p][i]; !(v < least) && i >= past && (v != -INFINITY || base + i < a.k)) {
                            const uint32_t to = atomicAdd(&shared.kept, 1u);
                            if (to < shared.KEEP) shared.keep[to] = place_of(v, from + base + i);
                        }
                }
            for (uint32_t i = t; i < got * N; i += THREADS) {
                const float v = to_float<T>(((const raw*)shared.aside)[i]);
                const uint32_t which = shared.which[i / N], at = (which & 0xffffff) + i % N;
                if (!(v < least) && i % N >= which >> 24) {
                    const uint32_t to = atomicAdd(&shared.kept, 1u);
                    if (to < shared.KEEP) shared.keep[to] = place_of(v, from + at);
                }
            }
            __syncthreads();
            kept = shared.kept;
            exact = kept > shared.KEEP;
        }
        if (exact) {
            exact_keep<T>(z, n, a.k, from, shared, [](float) {});
            kept = a.k;
        }
        for (uint32_t i = t; i < kept; i += THREADS) {
            const u64 mine = shared.keep[i];
            uint32_t place = 0;
            for (uint32_t j = 0; j < kept; j++) place += shared.keep[j] > mine;
            if (place >= a.k) continue;
            if (PARTED) a.places[(row * a.parts + part) * a.k + place] = mine;
            else {
                a.values[row * a.k + place] = d.log_of(value_of((uint32_t)(mine >> 32)));
                a.index[row * a.k + place] = (int32_t)~(uint32_t)mine;
            }
        }
    }
}

// The parts of a row, joined by a work group: totals, and of the parts' places those that can be among the first k.  Every part has its own first k in order, so
// with r = ceil(k / parts) the smallest of the parts' r-th places is one that k places reach, and so is any part's k-th.  1 x 131072 bf16, k = 20: 6.6 us for the parts and 5.3
// for this.
template <class T> __global__ __launch_bounds__(256) void logprobs_join_kernel(LogprobArgs a) {
    __shared__ u64 keep[HE_JOIN_PARTS * HE_TOP_MAX], bound[2];
    __shared__ uint32_t kept;
    const u64 row = blockIdx.x;
    const uint32_t t = threadIdx.x, lane = t & 63;
    const float c = HE_LOG2E / a.tau, low = masked_from(a.tau);
    const u64* places = a.places + row * a.parts * a.k;
    if (t == 0) kept = 0;
    // every wavefront joins the totals for itself, in order of the parts
    const float4 x = lane < a.parts ? a.totals[row * a.parts + lane] : float4{low, 0, 0, 0};
    const float ref = wave_max(x.x);
    Totals s = against({x.x, x.y, x.z}, ref, c);
    s.sum = wave_sum(s.sum);
    s.less = wave_sum(s.less);
    const Distribution d(s, low, a.tau);
    if (t == 0) write_row<T>(a, row, d);
    if (a.k == 0) return;
    if (t < 64) {
        const uint32_t r = (a.k + a.parts - 1) / a.parts;
        u64 all = lane < a.parts ? places[lane * a.k + r - 1] : ~0ull, any = lane < a.parts ? places[lane * a.k + a.k - 1] : 0;
        for (int i = 32; i; i >>= 1) {
            const u64 p = __shfl_xor(all, i), q = __shfl_xor(any, i);
            all = p < all ? p : all;
            any = q > any ? q : any;
        }
        if (t == 0) bound[0] = all > any ? all : any;
    }
    __syncthreads();
    const u64 least = bound[0];
    for (uint32_t i = t; i < a.parts * a.k; i += 256)
        if (const u64 p = places[i]; p >= least) keep[atomicAdd(&kept, 1u)] = p;
    __syncthreads();
    const uint32_t n = kept;
    for (uint32_t i = t; i < n; i += 256) {
        const u64 mine = keep[i];
        uint32_t place = 0;
        for (uint32_t j = 0; j < n; j++) place += keep[j] > mine;
        if (place >= a.k) continue;
        a.values[row * a.k + place] = d.log_of(value_of((uint32_t)(mine >> 32)));
        a.index[row * a.k + place] = (int32_t)~(uint32_t)mine;
    }
}

// Rows of fewer elements than 16 bytes have, a thread each: of so few every one counts how many come before it
template <class T> __global__ __launch_bounds__(256) void logprobs_short_kernel(LogprobArgs a, uint32_t rows) {
    using raw = typename T::raw;
    const u64 row = (u64)blockIdx.x * 256 + threadIdx.x;
    if (row >= rows) return;
    const raw* z = (const raw*)a.z + row * a.ld_z;
    constexpr uint32_t N = Vec<T>::N;
    const float c = HE_LOG2E / a.tau, low = masked_from(a.tau);
    float e[N];
    Totals s = {low, 0, 0};
#pragma unroll
    for (uint32_t i = 0; i < N; i++) {
        e[i] = i < a.vocab ? to_float<T>(z[i]) : -INFINITY;
        s.ref = fmaxf(s.ref, e[i]);
    }
    const float ref = reference(s.ref, low);
#pragma unroll
    for (uint32_t i = 0; i < N; i++) {
        const float d = (e[i] - ref) * c, f = exp2_fast(d);
        s.sum += f;
        s.less = fmaf(f, fmaxf(d, LEAST_POWER), s.less);
    }
    const Distribution d(s, low, a.tau);
    write_row<T>(a, row, d);
#pragma unroll
    for (uint32_t i = 0; i < N; i++) {
        uint32_t place = 0;
#pragma unroll
        for (uint32_t j = 0; j < N; j++) place += j < a.vocab && place_of(e[j], j) > place_of(e[i], i);
        if (i < a.vocab && place < a.k) {
            a.values[row * a.k + place] = d.log_of(e[i]);
            a.index[row * a.k + place] = (int32_t)i;
        }
    }
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
    const LogprobCut cut = logprobs_cut(p->rows, p->vocab, p->dtype);
    const LogprobArgs a = {p->d_z, p->d_tokens, p->d_logp, p->d_entropy, p->d_values, p->d_index, (float4*)p->d_stats, p->ld_z, p->vocab, p->k, p->tau,
                           cut.parts, cut.len, (u64*)p->d_work + 2 * (uint64_t)p->rows * cut.parts, (float4*)p->d_work};
    with_dtype(p->dtype, [&](auto t) {
        using T = decltype(t);
        if (p->vocab < (uint32_t)Vec<T>::N) {
            logprobs_short_kernel<T><<<(p->rows + 255) / 256, 256, 0, ctx->stream>>>(a, p->rows);
            return;
        }
        auto run = [&](auto threads, auto room, auto held) {
            constexpr int THREADS = decltype(threads)::value, ROOM = decltype(room)::value;
            constexpr bool HELD = decltype(held)::value;
            if (THREADS > 64 && cut.parts > 1) {
                logprobs_kernel<T, THREADS, ROOM, HELD, THREADS != 64><<<dim3(cut.parts, p->rows), THREADS, 0, ctx->stream>>>(a);
                logprobs_join_kernel<T><<<p->rows, 256, 0, ctx->stream>>>(a);
            } else logprobs_kernel<T, THREADS, ROOM, HELD, false><<<p->rows, THREADS, 0, ctx->stream>>>(a);
        };
        using std::integral_constant;
        // Room for what is set aside: of rows in no particular order some k (1 + ln(turns)) pieces are, twice that where the lanes' maxima fall badly
        // (2048 x 131072 with 512 threads: k = 64 122 us in 1024 places, with 512 it overflowed and took 2355).
        auto go = [&](auto threads) {
            if (p->k == 0) run(threads, integral_constant<int, 0>{}, std::false_type{});
            else if (p->k <= 64) run(threads, integral_constant<int, 1024>{}, std::false_type{});
            else run(threads, integral_constant<int, 2048>{}, std::false_type{});
        };
        auto hold = [&](auto threads) {
            if (p->k == 0) run(threads, integral_constant<int, 0>{}, std::true_type{});
            else run(threads, integral_constant<int, 1>{}, std::true_type{});
        };
        // Several work groups to a compute unit, one of which reads while another puts in order: 2048 x 131072 bf16, k = 8, takes 107 us with 512 threads, 110 with
        // 256 and 123 with 1024, 4096 x 50021 100, 95 and 132, 8192 x 20000 97, 84 and 146.  From k = 65 on thresholds of few wavefronts take long: 512 then
        // (4096 x 50021, k = 128: 171 us, 241 with 256).  Short rows by a wavefront each once there are rows for all: 8192 x 1000, k = 8, 13.9 us, by four (then with pieces set
        // aside) 31.
        const uint64_t bytes = (uint64_t)cut.len * dtype_bytes(p->dtype);
        const bool few = p->k <= 32 || p->vocab <= 128;
        if (bytes > 131072 || (bytes > 32768 && p->k > 64)) go(integral_constant<int, 512>{});
        else if (bytes > 16384) go(integral_constant<int, 256>{});
        else if (bytes > 4096 || !few || (bytes > 1024 && p->rows < 1024)) hold(integral_constant<int, 256>{});
        else hold(integral_constant<int, 64>{});
    });
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
    bool past_cache;           // the gradient is far larger than the caches
};

// Of d = (z - M) c the gradient is 2^d (A + B d), with two numbers a row, and the token's own term.  A work group takes V pieces of 16 bytes a thread of a row,
// all on their way before the first is used: a row's elements need nothing of each other, so long rows are cut wherever it suits.  2055 x 50021 bf16, rows that start
// anywhere: 89 us (4.6 TB/s, memory).
template <class T, class R_, int THREADS, int V> __global__ __launch_bounds__(THREADS) void logprobs_grad_kernel(LogprobGradArgs a) {
    using raw = typename T::raw;
    constexpr int N = Vec<T>::N;
    const u64 row = blockIdx.x;
    raw* grad = (raw*)a.grad + row * a.ld_grad;
    const R_ in{(const raw*)a.z + row * a.ld_z, a.vocab};
    const uint32_t first = blockIdx.y * (THREADS * V) + threadIdx.x, pieces = in.pieces();
    Vec<T> x[V];
#pragma unroll
    for (int p = 0; p < V; p++) x[p] = in.load(first + p * THREADS);
    const float c = HE_LOG2E / a.tau;
    const float4 stats = a.stats[row];
    const uint32_t token = a.tokens ? (uint32_t)a.tokens[row] : ~0u;
    const float wl = a.logp_weights && token < a.vocab ? a.logp_weights[row] : 0.0f, wh = a.entropy_weights ? a.entropy_weights[row] : 0.0f;
    const bool zero = (wl == 0.0f && wh == 0.0f) || stats.y == 0.0f;
    const float by = 1.0f / (stats.y * a.tau), own = wl / a.tau;
    const float A = -(wl + wh * (stats.z - logf(stats.y))) * by, B = -wh * HE_LN2 * by;
#pragma unroll
    for (int p = 0; p < V; p++) {
        const uint32_t v = first + p * THREADS, at = token - in.base(v);
        if (v >= pieces) break;
        float y[N];
#pragma unroll
        for (int i = 0; i < N; i++) {
            const float d = (x[p][i] - stats.x) * c;
            y[i] = zero ? 0.0f : exp2_fast(d) * fmaf(B, fmaxf(d, LEAST_POWER), A);
        }
        if (at < (uint32_t)N && !zero)
#pragma unroll
            for (int i = 0; i < N; i++)
                if (at == (uint32_t)i) y[i] += own;
        Vec<T> g;
        g.set(y);
        in.store(grad, v, g, a.past_cache);
    }
}

template <class R> struct RowKind { using type = R; };

extern "C" int32_t he_token_logprobs_grad(he_ctx* ctx, const he_logprobs_grad_plan* p) {
    return he_guard(ctx, "he_token_logprobs_grad: host allocation failed", [&]() -> int32_t {
    if (!ctx) return HE_ERR_BADARG;
    HE_REFUSE(ctx, "he_token_logprobs_grad", refuse_logprobs_grad(p));
    if (p->rows == 0) return HE_OK;
    const OnDevice device(ctx);
    HE_HIP(ctx, device.status);
    const uint64_t bytes = (uint64_t)p->vocab * dtype_bytes(p->dtype);
    const LogprobGradArgs a = {p->d_z, p->d_tokens, (const float4*)p->d_stats, p->d_logp_weights, p->d_entropy_weights, p->d_grad, p->ld_z, p->ld_grad, p->vocab, p->tau,
                               bytes * p->rows > 64ull << 20};
    with_dtype(p->dtype, [&](auto t) {
        using T = decltype(t);
        auto go = [&](auto row, auto threads, auto pieces) {
            constexpr int THREADS = decltype(threads)::value, V = decltype(pieces)::value;
            const uint32_t of = THREADS * V * 16;         // bytes a work group
            logprobs_grad_kernel<T, typename decltype(row)::type, THREADS, V><<<dim3(p->rows, (uint32_t)((bytes + of - 1) / of)), THREADS, 0, ctx->stream>>>(a);
        };
        using std::integral_constant;
        if (p->vocab < (uint32_t)Vec<T>::N) go(RowKind<ShortRow<T>>{}, integral_constant<int, 64>{}, integral_constant<int, 1>{});
        else if (bytes <= 1024) go(RowKind<Row<T>>{}, integral_constant<int, 64>{}, integral_constant<int, 1>{});
        else if (bytes <= 4096) go(RowKind<Row<T>>{}, integral_constant<int, 64>{}, integral_constant<int, 4>{});
        else go(RowKind<Row<T>>{}, integral_constant<int, 256>{}, integral_constant<int, 4>{});
    });
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}
