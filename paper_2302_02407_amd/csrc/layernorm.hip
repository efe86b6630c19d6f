// Layer norm with a residual addition before it, and its gradients.
#include "plain.h"

struct LnArgs {
    const void *x, *res, *weight, *bias;
    void *sum, *y;
    float4* stats;
    u64 ld_x, ld_res, ld_sum, ld_y;
    uint32_t rows, dim;
    float eps;
};

// 1 / sqrt(v), or 0 where that is nothing to divide by
__device__ __forceinline__ float inverse_root(float v) { return v < 0x1p-120f ? 0.0f : 1.0f / sqrtf(v); }

// ROW threads a row, each with V pieces of 8 elements, piece p of a row with thread p % ROW, which stay in registers: everything is read and
// written once.  Rows of up to 256 columns take 16 lanes each, sixteen to a work group, rows of up to 1024 a wavefront, four to a work group; longer ones a work group.  The mean is a number of 32
// bits and what that lacks, the sum of the differences from it: so a row far from 0 keeps its variance, whose own sum is of those
// differences, and its gradient.
//
// 16384 x 4096 bf16 with a residual, parameters of 32 bits: 112 us (4.8 TB/s, memory); 60000 x 100 f32 14.7 us, 29.7 by a wavefront a row; 1 x 4096 8.3 us a call, its host
// side, the kernel 4.5.
template <class T, class P, bool RES, int ROW, int V> __global__ __launch_bounds__(ROW < 256 ? 256 : ROW) void layernorm_kernel(LnArgs a) {
    using raw = typename T::raw;
    constexpr int GROUP = ROW < 256 ? 256 : ROW, WAVES = ROW / 64;
    __shared__ float room[2 * (GROUP / 64)];
    const u64 row = (u64)blockIdx.x * (GROUP / ROW) + threadIdx.x / ROW;
    if (row >= a.rows) return;                            // ROW <= 64: no barrier follows, and sums are among the row's own lanes
    const uint32_t t = threadIdx.x % ROW, dim = a.dim;
    const raw* x = (const raw*)a.x + row * a.ld_x;
    const raw* res = (const raw*)a.res + row * a.ld_res;
    float h[V][8], s = 0;
#pragma unroll
    for (int p = 0; p < V; p++) {
        const uint32_t at = (p * ROW + t) * 8;
        load8<T>(x, at, dim, h[p]);
        if (RES) {
            float more[8];
            load8<T>(res, at, dim, more);
            Eight<T> sum;
#pragma unroll
            for (int i = 0; i < 8; i++) more[i] += h[p][i];
            sum.set(more);
#pragma unroll
            for (int i = 0; i < 8; i++) h[p][i] = sum[i];
            store8<T>((raw*)a.sum + row * a.ld_sum, at, dim, h[p]);       // over x or the residual at most what this thread has read
        }
#pragma unroll
        for (int i = 0; i < 8; i++) s += h[p][i];
        if (V >= 8) __builtin_amdgcn_sched_barrier(0);    // one piece's loads at a time: the numbers fill the registers
    }
    auto total = [&](float v) { return ROW == 16 ? row_sum(v) : group_sum<WAVES ? WAVES : 1>(v, room); };
    float mean = total(s) / (float)dim, low, var;
    // The variance, and what the mean lacks.  Where that is not far below the row's spread, the mean is rounded again with it and both are taken again: a constant then is its own
    // mean, and of numbers that differ by their last bits the variance is at least the square of what the nearest number lacks.
    auto spread = [&]() {
#pragma unroll 1
        for (int turn = 0;; turn++) {
            float d1 = 0, d2 = 0;
#pragma unroll
            for (int p = 0; p < V; p++) {
                const int left = (int)dim - (int)((p * ROW + t) * 8);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float d = i < left ? h[p][i] - mean : 0.0f;
                    d1 += d;
                    d2 = fmaf(d, d, d2);
                }
            }
            group_sum2<WAVES>(d1, d2, room);
            low = d1 / (float)dim;
            var = d2 / (float)dim - low * low;
            var = var < 0.0f ? 0.0f : var;                // a NaN stays one
            const float nearer = mean + low;
            if (turn == 2 || !(low * low > 0.015625f * var) || nearer == mean) break;
            mean = nearer;
        }
    };
    spread();
    float r = inverse_root(var + a.eps);
    float4 stats = {mean, low, r, 0};
    if (!(var < 0x1p126f)) {                              // squares, or the sum, that 32 bits do not hold: by a power of two
        float most = 0;
#pragma unroll
        for (int p = 0; p < V; p++)
#pragma unroll
            for (int i = 0; i < 8; i++) most = fmaxf(most, fabsf(h[p][i]));
        most = ROW == 16 ? __builtin_bit_cast(float, row_max(__builtin_bit_cast(int32_t, most))) : group_max<WAVES ? WAVES : 1>(most, room);
        if (most < INFINITY) {
            const int e = __builtin_amdgcn_frexp_expf(most);
            s = 0;
#pragma unroll
            for (int p = 0; p < V; p++)
#pragma unroll
                for (int i = 0; i < 8; i++) s += h[p][i] = ldexpf(h[p][i], -e);
            mean = total(s) / (float)dim;
            spread();
            // of a constant eps is all that is left, which has no power; another row's variance is at least 2^-70 beside it
            r = inverse_root(var == 0.0f ? a.eps : var + ldexpf(a.eps, -2 * e));
            stats = {ldexpf(mean, e), ldexpf(low, e), var == 0.0f ? r : ldexpf(r, -e), 0};
        }
    }
    if (a.stats && t == 0) a.stats[row] = stats;
#pragma unroll
    for (int p = 0; p < V; p++) {
        const uint32_t at = (p * ROW + t) * 8;
        if (at >= dim) break;
        if (V >= 8) __builtin_amdgcn_sched_barrier(0);
        float w[8], b[8];
        if (a.weight) load8<P>((const typename P::raw*)a.weight, at, dim, w);
        if (a.bias) load8<P>((const typename P::raw*)a.bias, at, dim, b);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float n = (h[p][i] - mean - low) * r;
            h[p][i] = fmaf(n, a.weight ? w[i] : 1.0f, a.bias ? b[i] : 0.0f);
        }
        store8<T>((raw*)a.y + row * a.ld_y, at, dim, h[p]);
    }
}

template <class T, class P, bool RES> static void launch_layernorm(const LnArgs& a, hipStream_t stream) {
    auto go = [&](auto row, auto v) {
        constexpr int ROW = decltype(row)::value, GROUP = ROW < 256 ? 256 : ROW;
        layernorm_kernel<T, P, RES, ROW, decltype(v)::value><<<(a.rows + GROUP / ROW - 1) / (GROUP / ROW), GROUP, 0, stream>>>(a);
    };
    using std::integral_constant;
    if (a.dim <= 128) go(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else if (a.dim <= 256) go(integral_constant<int, 16>{}, integral_constant<int, 2>{});
    else if (a.dim <= 512) go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (a.dim <= 1024) go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (a.dim <= 2048) go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    else if (a.dim <= 4096) go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    else if (a.dim <= 8192) go(integral_constant<int, 512>{}, integral_constant<int, 2>{});
    else if (a.dim <= 16384) go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
    else if (a.dim <= 32768) go(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
    else go(integral_constant<int, 1024>{}, integral_constant<int, 8>{});
}

// Calls f with the types of rows and parameters
template <class F> static void with_types(int32_t dtype, int32_t param_dtype, F&& f) {
    with_dtype(dtype, [&](auto t) {
        if (param_dtype == HE_F32) f(t, f32_t{});
        else f(t, t);
    });
}

extern "C" int32_t he_layernorm(he_ctx* ctx, const he_layernorm_plan* p) {
    return he_guard(ctx, "he_layernorm: host allocation failed", [&]() -> int32_t {
    if (!ctx) return HE_ERR_BADARG;
    HE_REFUSE(ctx, "he_layernorm", refuse_layernorm(p));
    if (p->rows == 0) return HE_OK;
    const OnDevice device(ctx);
    HE_HIP(ctx, device.status);
    const LnArgs a = {p->d_x, p->d_residual, p->d_weight, p->d_bias, p->d_sum, p->d_y, (float4*)p->d_stats, p->ld_x, p->ld_residual, p->ld_sum, p->ld_y, p->rows, p->dim, p->eps};
    with_types(p->dtype, p->param_dtype, [&](auto t, auto w) {
        if (p->d_residual) launch_layernorm<decltype(t), decltype(w), true>(a, ctx->stream);
        else launch_layernorm<decltype(t), decltype(w), false>(a, ctx->stream);
    });
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}

// ---- gradients

// n from a row's statistics.  By halves: the difference of two numbers of 32 bits may be none, half of it is, with the same rounding.
struct Normed {
    float mean, low, by;
    __device__ __forceinline__ Normed(const float4& stats) : mean(-0.5f * stats.x), low(0.5f * stats.y), by(2.0f * stats.z) {}
    __device__ __forceinline__ float operator()(float h) const { return (fmaf(h, 0.5f, mean) - low) * by; }
};

struct LnGradArgs {
    const void *h, *dy, *dsum, *weight;
    const float4* stats;
    void* dx;
    float* sums;                   // [parts][2][pitch]: of dy n and of dy, or null
    u64 ld_h, ld_dy, ld_dsum, ld_dx;
    uint32_t rows, dim, parts, pitch;
};

// Everything in one pass: a work group takes every parts-th row (of 64 threads a row: every parts-th four; of 16: every parts-th sixteen), whose two means it needs at once, and keeps the sums
// over its rows for its columns in registers; they go to memory once, for the join.  The next row is asked for before this one's means are there (but for four
// pieces a thread, whose registers it does not fit).  Pieces are of 8
// elements; the last one lies where it still fits the row, and what of it belongs to the one before has a gradient of 0 here and is not written.
//
// 16384 x 4096 bf16 with dsum, parameters of 32 bits: 103 us, 5 of them the join's (5.2 TB/s of what it cannot do without, memory; vector instructions 39% of
// cycles, counted); as a pass for the rows and one for the columns 245.  517 x 1001 f16 13 us in two launches.
template <class T, class P, bool DSUM, int ROW, int V> __global__ __launch_bounds__(ROW < 256 ? 256 : ROW) void layernorm_grad_kernel(LnGradArgs a) {
    using raw = typename T::raw;
    constexpr int GROUP = ROW < 256 ? 256 : ROW, SLOTS = GROUP / ROW, WAVES = ROW / 64;
    constexpr bool AHEAD = V <= 2;
    __shared__ float room[2][2 * WAVES + 1];
    const uint32_t t = threadIdx.x % ROW, slot = threadIdx.x / ROW, step = a.parts * SLOTS;
    const typename P::raw* w = (const typename P::raw*)a.weight;
    uint32_t base[V], past[V];
    Eight<P> weight[V];
    float dw[V][8], db[V][8];
#pragma unroll
    for (int p = 0; p < V; p++) {
        const uint32_t at = (p * ROW + t) * 8;
        base[p] = min(at, a.dim - 8);
        past[p] = at - base[p];
        if (w) weight[p].load(w + base[p]);
        else {
            const float ones[8] = {1, 1, 1, 1, 1, 1, 1, 1};
            weight[p].set(ones);
        }
#pragma unroll
        for (int i = 0; i < 8; i++) dw[p][i] = db[p][i] = 0;
    }
    struct Line {
        Eight<T> h[V], dy[V], dsum[DSUM ? V : 1];
        float4 stats;
    };
    auto load = [&](uint32_t row, Line& l) {
        const raw *h = (const raw*)a.h + (u64)row * a.ld_h, *dy = (const raw*)a.dy + (u64)row * a.ld_dy, *dsum = (const raw*)a.dsum + (u64)row * a.ld_dsum;
        l.stats = a.stats[row];
#pragma unroll
        for (int p = 0; p < V; p++) {
            l.h[p].load(h + base[p]);
            l.dy[p].load(dy + base[p]);
            if (DSUM && AHEAD) l.dsum[p].load(dsum + base[p]);
        }
    };
    uint32_t row = blockIdx.x * SLOTS + slot, turn = 0;
    Line now, next;
    if (AHEAD && row < a.rows) load(row, now);
    // ROW <= 64: a wavefront has rows of its own and no barrier; otherwise there is one slot, and all of the work group are here as often
    for (; row < a.rows; row += step, turn ^= 1) {
        if (!AHEAD) load(row, now);
        else if (row + step < a.rows) load(row + step, next);
        const Normed normed(now.stats);
        const float r = now.stats.z;
        float s1 = 0, s2 = 0;
#pragma unroll
        for (int p = 0; p < V; p++) {
            if (past[p])
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if ((uint32_t)i < past[p]) now.dy[p].v[i / Vec<T>::N].set(i % Vec<T>::N, 0.0f);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float d = now.dy[p][i], n = normed(now.h[p][i]), g = d * weight[p][i];
                dw[p][i] = fmaf(d, n, dw[p][i]);
                db[p][i] += d;
                s1 += g;
                s2 = fmaf(g, n, s2);
            }
        }
        s1 = ROW == 16 ? row_sum(s1) : wave_sum(s1);
        s2 = ROW == 16 ? row_sum(s2) : wave_sum(s2);
        if (WAVES > 1) {                                  // two rooms in turn: one barrier
            if ((threadIdx.x & 63) == 0) {
                room[turn][threadIdx.x >> 6] = s1;
                room[turn][WAVES + (threadIdx.x >> 6)] = s2;
            }
            __syncthreads();
            s1 = room[turn][0];
            s2 = room[turn][WAVES];
#pragma unroll
            for (int i = 1; i < WAVES; i++) {
                s1 += room[turn][i];
                s2 += room[turn][WAVES + i];
            }
        }
        s1 /= (float)a.dim;
        s2 /= (float)a.dim;
        raw* dx = (raw*)a.dx + (u64)row * a.ld_dx;
#pragma unroll
        for (int p = 0; p < V; p++) {
            float y[8];
            if (DSUM && !AHEAD) now.dsum[p].load((const raw*)a.dsum + (u64)row * a.ld_dsum + base[p]);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float n = normed(now.h[p][i]), g = now.dy[p][i] * weight[p][i];
                y[i] = fmaf(r, g - s1 - n * s2, DSUM ? now.dsum[p][i] : 0.0f);
            }
            if (past[p] == 0) {
                Eight<T> out;
                out.set(y);
#pragma unroll
                for (int v = 0; v < Eight<T>::VECS; v++) out.v[v].store_past(dx + base[p] + v * Vec<T>::N);
            } else
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if ((uint32_t)i >= past[p]) dx[base[p] + i] = from_float<T>(y[i]);
        }
        if (AHEAD) now = next;
    }
    if (!a.sums) return;
    float* to = a.sums + (u64)blockIdx.x * 2 * a.pitch;
    if constexpr (SLOTS > 1) {                            // of a wavefront's rows, then of the wavefronts, in order
        __shared__ float sums[4][2][V * ROW * 8];
        const uint32_t wave = threadIdx.x >> 6;
#pragma unroll
        for (int p = 0; p < V; p++)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                if constexpr (ROW == 16) {
                    dw[p][i] += __shfl_xor(dw[p][i], 16);
                    db[p][i] += __shfl_xor(db[p][i], 16);
                    dw[p][i] += __shfl_xor(dw[p][i], 32);
                    db[p][i] += __shfl_xor(db[p][i], 32);
                }
                if ((threadIdx.x & 63) < ROW && (uint32_t)i >= past[p]) {
                    sums[wave][0][base[p] + i] = dw[p][i];
                    sums[wave][1][base[p] + i] = db[p][i];
                }
            }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < 2 * a.dim; i += GROUP) {
            const uint32_t which = i >= a.dim, column = i - which * a.dim;
            to[which * a.pitch + column] = sums[0][which][column] + sums[1][which][column] + sums[2][which][column] + sums[3][which][column];
        }
    } else
#pragma unroll
        for (int p = 0; p < V; p++) {
            if (past[p] == 0) {
                __builtin_memcpy(to + base[p], dw[p], 32);
                __builtin_memcpy(to + a.pitch + base[p], db[p], 32);
            } else
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if ((uint32_t)i >= past[p]) {
                        to[base[p] + i] = dw[p][i];
                        to[a.pitch + base[p] + i] = db[p][i];
                    }
        }
}

// Rows too long for a work group's registers, or shorter than a piece: a row a work group, in two passes, its two means, then its gradient (2048 x 20000 bf16 118 us, 2.1
// TB/s of what it cannot do without: everything is read three times, once for the columns)
template <class T, class P, int THREADS> __global__ __launch_bounds__(THREADS) void layernorm_dx_kernel(LnGradArgs a) {
    using raw = typename T::raw;
    __shared__ float room[2 * (THREADS / 64)];
    const u64 row = blockIdx.x;
    const raw *h = (const raw*)a.h + row * a.ld_h, *dy = (const raw*)a.dy + row * a.ld_dy, *dsum = (const raw*)a.dsum + row * a.ld_dsum;
    const typename P::raw* w = (const typename P::raw*)a.weight;
    const float4 stats = a.stats[row];
    const Normed normed(stats);
    auto piece = [&](uint32_t at, float* n, float* g) {
        load8<T>(h, at, a.dim, n);
        load8<T>(dy, at, a.dim, g);
        float f[8];
        if (w) load8<P>(w, at, a.dim, f);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            n[i] = normed(n[i]);
            if (w) g[i] *= f[i];
        }
        if (at + 8 > a.dim)                               // past the row's end: 0 of g times what -mean / sqrt(v + eps) is, which may be no number
#pragma unroll
            for (int i = 0; i < 8; i++) n[i] = at + i < a.dim ? n[i] : 0.0f;
    };
    float s1 = 0, s2 = 0;
    for (uint32_t at = threadIdx.x * 8; at < a.dim; at += THREADS * 8) {
        float n[8], g[8];
        piece(at, n, g);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            s1 += g[i];                                   // 0 past the row's end
            s2 = fmaf(g[i], n[i], s2);
        }
    }
    group_sum2<THREADS / 64>(s1, s2, room);
    s1 /= (float)a.dim;
    s2 /= (float)a.dim;
    for (uint32_t at = threadIdx.x * 8; at < a.dim; at += THREADS * 8) {
        float n[8], g[8], more[8];
        piece(at, n, g);
        if (a.dsum) load8<T>(dsum, at, a.dim, more);
#pragma unroll
        for (int i = 0; i < 8; i++) g[i] = fmaf(stats.z, g[i] - s1 - n[i] * s2, a.dsum ? more[i] : 0.0f);
        store8<T>((raw*)a.dx + row * a.ld_dx, at, a.dim, g);
    }
}

// Their sums over a part of the rows, 512 columns a work group: each wavefront every fourth row, their sums joined in order
template <class T> __global__ __launch_bounds__(256) void layernorm_columns_kernel(LnGradArgs a) {
    using raw = typename T::raw;
    __shared__ float sums[4][2][512];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = blockIdx.x * 512 + lane * 8;
    const uint32_t from = (u64)a.rows * blockIdx.y / a.parts, to = (u64)a.rows * (blockIdx.y + 1) / a.parts;
    float dw[8] = {}, db[8] = {};
    if (at < a.dim)
        for (uint32_t row = from + wave; row < to; row += 4) {
            float n[8], g[8];
            load8<T>((const raw*)a.h + row * a.ld_h, at, a.dim, n);
            load8<T>((const raw*)a.dy + row * a.ld_dy, at, a.dim, g);
            const Normed normed(a.stats[row]);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                dw[i] = fmaf(g[i], normed(n[i]), dw[i]);
                db[i] += g[i];
            }
        }
#pragma unroll
    for (int i = 0; i < 8; i++) {
        sums[wave][0][lane * 8 + i] = dw[i];
        sums[wave][1][lane * 8 + i] = db[i];
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 1024; i += 256) {
        const uint32_t which = i >> 9, c = i & 511, column = blockIdx.x * 512 + c;
        if (column < a.dim) a.sums[((u64)blockIdx.y * 2 + which) * a.pitch + column] = sums[0][which][c] + sums[1][which][c] + sums[2][which][c] + sums[3][which][c];
    }
}

// The parts' sums, in a fixed order: 32 threads four columns, each every 32nd part
template <class P> __global__ __launch_bounds__(256) void layernorm_join_kernel(const float* parts, uint32_t n_parts, uint32_t dim, uint32_t pitch, void* dweight, void* dbias) {
    typedef float v4f __attribute__((ext_vector_type(4)));
    __shared__ v4f sums[32][8];
    const uint32_t lane = threadIdx.x / 8, at = (blockIdx.x * 8 + threadIdx.x % 8) * 4;      // of 2 * pitch
    v4f x = {0, 0, 0, 0};
    if (at < 2 * pitch)
#pragma unroll 4
        for (uint32_t p = lane; p < n_parts; p += 32) x += *(const v4f*)(parts + (u64)p * 2 * pitch + at);
    sums[lane][threadIdx.x % 8] = x;
    __syncthreads();
    if (lane || at >= 2 * pitch) return;
#pragma unroll
    for (int j = 1; j < 32; j++) x += sums[j][threadIdx.x];
    const uint32_t column = at % pitch;                   // a multiple of 4, as the pitch is
    typename P::raw* to = (typename P::raw*)(at < pitch ? dweight : dbias);
    if (!to) return;
#pragma unroll
    for (int i = 0; i < 4; i++)
        if (column + i < dim) to[column + i] = from_float<P>(x[i]);
}

template <class T, class P, bool DSUM> static void launch_layernorm_grad(const LnGradArgs& a, hipStream_t stream) {
    auto go = [&](auto row, auto v) {
        constexpr int ROW = decltype(row)::value;
        layernorm_grad_kernel<T, P, DSUM, ROW, decltype(v)::value><<<a.parts, ROW < 256 ? 256 : ROW, 0, stream>>>(a);
    };
    using std::integral_constant;
    if (a.dim <= 128) go(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else if (a.dim <= 256) go(integral_constant<int, 16>{}, integral_constant<int, 2>{});
    else if (a.dim <= 512) go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (a.dim <= 1024) go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (a.dim <= 2048) go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    else if (a.dim <= 4096) go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    else if (a.dim <= 8192) go(integral_constant<int, 512>{}, integral_constant<int, 2>{});
    else go(integral_constant<int, 512>{}, integral_constant<int, 4>{});
}

extern "C" int32_t he_work_layernorm_grad(const he_ctx* ctx, const he_layernorm_grad_plan* p, uint64_t* h_bytes) {
    return he_guard(ctx, "he_work_layernorm_grad: host allocation failed", [&]() -> int32_t {
    if (!ctx || !h_bytes) return HE_ERR_BADARG;
    HE_REFUSE(const_cast<he_ctx*>(ctx), "he_work_layernorm_grad", refuse_layernorm_grad(p, true));
    *h_bytes = layernorm_grad_work(p);
    return HE_OK;
    });
}

extern "C" int32_t he_layernorm_grad(he_ctx* ctx, const he_layernorm_grad_plan* p) {
    return he_guard(ctx, "he_layernorm_grad: host allocation failed", [&]() -> int32_t {
    if (!ctx) return HE_ERR_BADARG;
    HE_REFUSE(ctx, "he_layernorm_grad", refuse_layernorm_grad(p));
    const bool sums = p->d_dweight || p->d_dbias;
    const OnDevice device(ctx);
    HE_HIP(ctx, device.status);
    const LnGradArgs a = {p->d_h, p->d_dy, p->d_dsum, p->d_weight, (const float4*)p->d_stats, p->d_dx, sums ? (float*)p->d_work : nullptr, p->ld_h, p->ld_dy, p->ld_dsum, p->ld_dx,
                          p->rows, p->dim, p->rows ? layernorm_parts(p->rows, p->dim) : 0, layernorm_pitch(p->dim)};
    with_types(p->dtype, p->param_dtype, [&](auto t, auto w) {
        using T = decltype(t);
        using P = decltype(w);
        if (a.rows && layernorm_one_pass(a.dim)) {
            if (a.dsum) launch_layernorm_grad<T, P, true>(a, ctx->stream);
            else launch_layernorm_grad<T, P, false>(a, ctx->stream);
        } else if (a.rows) {                              // sums before dx, which may lie on dy
            if (sums) layernorm_columns_kernel<T><<<dim3((a.dim + 511) / 512, a.parts), 256, 0, ctx->stream>>>(a);
            if (a.dim < 8) layernorm_dx_kernel<T, P, 64><<<a.rows, 64, 0, ctx->stream>>>(a);
            else layernorm_dx_kernel<T, P, 1024><<<a.rows, 1024, 0, ctx->stream>>>(a);
        }
        if (sums) layernorm_join_kernel<P><<<(2 * a.pitch + 31) / 32, 256, 0, ctx->stream>>>((const float*)p->d_work, a.parts, a.dim, a.pitch, p->d_dweight, p->d_dbias);
    });
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}
