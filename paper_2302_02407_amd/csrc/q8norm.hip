// Residual addition, root-mean-square norm and output in 8 bits with a scale for each 128 columns.
#include "plain.h"

#define Q8_MAX 448.0f      // largest e4m3 value
#define Q8_BLOCK 128

struct NormArgs {
    const void *x, *res, *weight;
    void* sum;
    uint8_t* codes;
    float* scales;
    u64 ld_x, ld_res, ld_sum, ld_codes, ld_scales;
    uint32_t rows, dim;
    float eps;
};

// |y| as an integer: ordered like the numbers, infinity above them and NaN above that, so that a maximum keeps both
__device__ __forceinline__ int32_t magnitude(float y) { return __builtin_bit_cast(int32_t, y) & 0x7fffffff; }

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

// ROW threads a row, each with V pieces of 8 elements, piece p of a row with thread p % ROW: what it adds stays in registers between the sum of
// squares and the output, so that everything is read and written once.  16 lanes side by side hold a block of 128 columns and find its
// largest element among themselves.  Rows of up to 1024 columns take a wavefront each, four to a work group; longer ones a work group.
// All loads are on their way before the first is used; a piece that the row's end cuts is read from inside the row and then again element by
// element.
//
// 16384 x 4096 bf16 with residual: 81 us (5.8 TB/s, memory); 1 x 4096: 7 us a call, its host side.
template <class T, bool RES, int ROW, int V> __global__ __launch_bounds__(ROW < 256 ? 256 : ROW) void rmsnorm_q8_kernel(NormArgs a) {
    using raw = typename T::raw;
    constexpr int GROUP = ROW < 256 ? 256 : ROW;
    __shared__ float room[GROUP / 64];
    const u64 row = (u64)blockIdx.x * (GROUP / ROW) + threadIdx.x / ROW;
    if (row >= a.rows) return;                            // ROW = 64: a whole wavefront, and no barrier follows
    const uint32_t t = threadIdx.x % ROW;
    const raw* x = (const raw*)a.x + row * a.ld_x;
    const raw* res = (const raw*)a.res + row * a.ld_res;
    const raw* w = (const raw*)a.weight;
    constexpr bool ALL = V < 8;                           // a row's pieces and weights fit the registers beside the numbers
    Eight<T> in[V], more[RES ? V : 1], scale[V];
    const bool weighted = w != nullptr;
    if (ALL && a.dim >= 8) {
#pragma unroll
        for (int p = 0; p < V; p++) {
            const uint32_t at = min((p * ROW + t) * 8, a.dim - 8);
            in[p].load(x + at);
            if (RES) more[p].load(res + at);
        }
        if (weighted)
#pragma unroll
            for (int p = 0; p < V; p++) scale[p].load(w + min((p * ROW + t) * 8, a.dim - 8));
    }
    float h[V][8], sq = 0;
#pragma unroll
    for (int p = 0; p < V; p++) {
        const uint32_t at = (p * ROW + t) * 8;
        if (!ALL) {
            in[p].load(x + min(at, a.dim - 8));
            if (RES) more[p].load(res + min(at, a.dim - 8));
            if (p & 1) __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < 8; i++) h[p][i] = RES ? in[p][i] + more[p][i] : in[p][i];
        if (at + 8 > a.dim)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                h[p][i] = 0;
                if (at + i < a.dim) h[p][i] = RES ? to_float<T>(x[at + i]) + to_float<T>(res[at + i]) : to_float<T>(x[at + i]);
            }
#pragma unroll
        for (int i = 0; i < 8; i++) sq += h[p][i] * h[p][i];
    }
    sq = group_sum<ROW / 64>(sq, room);
    float mean = sq / (float)a.dim, r = 1.0f / sqrtf(mean + a.eps);
    int e = 0;                                            // of a power of two that the row is taken by
    if (mean < 0x1p-100f || mean == INFINITY) {           // squares that are no numbers, or rounded to the smallest ones: anew, by the largest element
        float most = 0;
#pragma unroll
        for (int p = 0; p < V; p++)
#pragma unroll
            for (int i = 0; i < 8; i++) most = fmaxf(most, fabsf(h[p][i]));
        most = group_max<ROW / 64>(most, room);
        if (most == 0.0f) r = 0;                          // zeros stay zeros, without eps too
        else if (most < INFINITY) {
            e = __builtin_amdgcn_readfirstlane(__builtin_amdgcn_frexp_expf(most));
            sq = 0;
#pragma unroll
            for (int p = 0; p < V; p++)
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float x = ldexpf(h[p][i], -e);
                    sq += x * x;
                }
            mean = group_sum<ROW / 64>(sq, room) / (float)a.dim;
            const float root = ldexpf(sqrtf(a.eps), -e);  // where it is far above the row's size, what the row adds is below its rounding
            r = root > 0x1p30f ? ldexpf(1.0f / sqrtf(a.eps), e) : 1.0f / sqrtf(mean + root * root);
        }
    }
#pragma unroll
    for (int p = 0; p < V; p++) {
        const uint32_t at = (p * ROW + t) * 8;
        const bool cut = at + 8 > a.dim;
        if (RES) {
            raw* sum = (raw*)a.sum + row * a.ld_sum;
            Eight<T> out;
            out.set(h[p]);
            if (!cut) out.store(sum + at);
            else
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if (at + i < a.dim) sum[at + i] = from_float<T>(h[p][i]);
        }
        if (e)
#pragma unroll
            for (int i = 0; i < 8; i++) h[p][i] = ldexpf(h[p][i], -e);
        if (!ALL) {
            __builtin_amdgcn_sched_barrier(0);
            if (weighted) scale[p].load(w + min(at, a.dim - 8));
        }
        // y = h w r and scale = max|y| / 448, so y / scale = h w (448 / max|h w|): without r, and with what the product and the quotient
        // were rounded by, off by one rounding before the one to 8 bits
        int32_t most = 0;
        float y[8], low[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float f = !weighted ? 1.0f : !cut ? scale[p][i] : at + i < a.dim ? to_float<T>(w[at + i]) : 0.0f;
            y[i] = h[p][i] * f;
            low[i] = fmaf(h[p][i], f, -y[i]);
            most = max(most, magnitude(y[i]));
        }
        const float top = __builtin_bit_cast(float, row_max(most)), s = top * r / Q8_MAX;
        const float up = top < 0x1p-100f ? 0x1p100f : 1.0f, by = top * up, inv = s != s ? NAN : Q8_MAX / by, inv_low = fmaf(-inv, by, Q8_MAX) / by;
        if (at < a.dim && (t & 15) == 0) a.scales[row * a.ld_scales + at / Q8_BLOCK] = s;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float v = y[i] * up;
            y[i] = s == 0.0f ? 0.0f : fmaf(v, inv, fmaf(v, inv_low, low[i] * up * inv));
        }
        uint32_t lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
        uint8_t* codes = a.codes + row * a.ld_codes + at;
        if (!cut) *(uint2*)codes = make_uint2(lo, hi);
        else
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (at + i < a.dim) codes[i] = (uint8_t)((i < 4 ? lo : hi) >> 8 * (i & 3));
    }
}

template <class T, bool RES> static void launch_norm(const NormArgs& a, hipStream_t stream) {
    auto go = [&](auto row, auto v) {
        constexpr int ROW = decltype(row)::value, GROUP = ROW < 256 ? 256 : ROW;
        rmsnorm_q8_kernel<T, RES, ROW, decltype(v)::value><<<(a.rows + GROUP / ROW - 1) / (GROUP / ROW), GROUP, 0, stream>>>(a);
    };
    using std::integral_constant;
    if (a.dim <= 512) go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (a.dim <= 1024) go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (a.dim <= 2048) go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    else if (a.dim <= 4096) go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    else if (a.dim <= 8192) go(integral_constant<int, 512>{}, integral_constant<int, 2>{});
    else if (a.dim <= 16384) go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
    else if (a.dim <= 32768) go(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
    else go(integral_constant<int, 1024>{}, integral_constant<int, 8>{});
}

extern "C" int32_t he_rmsnorm_q8(he_ctx* ctx, const he_rmsnorm_plan* p) {
    return he_guard(ctx, "he_rmsnorm_q8: host allocation failed", [&]() -> int32_t {
    if (!ctx) return HE_ERR_BADARG;
    if (!p) return he_fail(ctx, HE_ERR_BADARG, "he_rmsnorm_q8: null plan");
    if (!dtype_known(p->dtype)) return he_fail(ctx, HE_ERR_BADARG, "he_rmsnorm_q8: unknown type %d", p->dtype);
    if (p->dim == 0 || p->dim > 65536) return he_fail(ctx, HE_ERR_BADARG, "he_rmsnorm_q8: %u columns outside 1..65536", p->dim);
    if (!(p->eps >= 0.0f)) return he_fail(ctx, HE_ERR_BADARG, "he_rmsnorm_q8: eps is negative or not a number");
    if (p->rows > HE_ROWS_MAX) return he_fail(ctx, HE_ERR_BADARG, "he_rmsnorm_q8: more than 2^21 rows");
    if (p->rows == 0) return HE_OK;
    if (!p->d_x || !p->d_codes || !p->d_scales) return he_fail(ctx, HE_ERR_BADARG, "he_rmsnorm_q8: null argument");
    if (!p->d_residual != !p->d_sum) return he_fail(ctx, HE_ERR_BADARG, "he_rmsnorm_q8: a residual and its sum come together");
    const uint32_t es = dtype_bytes(p->dtype), nb = (p->dim + Q8_BLOCK - 1) / Q8_BLOCK;
    const bool res = p->d_residual != nullptr;
    if (!ld_fits(p->ld_x, p->dim) || !ld_fits(p->ld_codes, p->dim) || !ld_fits(p->ld_scales, nb) || (res && !(ld_fits(p->ld_residual, p->dim) && ld_fits(p->ld_sum, p->dim))))
        return he_fail(ctx, HE_ERR_BADARG, "he_rmsnorm_q8: an ld is below the row's length or above 2^28");
    if (((uintptr_t)p->d_codes | p->ld_codes) & 15) return he_fail(ctx, HE_ERR_BADARG, "he_rmsnorm_q8: rows of codes start at multiples of 16 bytes");
    if (((uintptr_t)p->d_x | (uintptr_t)p->d_residual | (uintptr_t)p->d_weight | (uintptr_t)p->d_sum) & (es - 1) || (uintptr_t)p->d_scales & 3)
        return he_fail(ctx, HE_ERR_BADARG, "he_rmsnorm_q8: a pointer is not aligned to its elements");
    const struct { const void* d; uint64_t n; } in[3] = {{p->d_x, span(p->rows, p->dim, p->ld_x, es)}, {p->d_residual, span(p->rows, p->dim, p->ld_residual, es)},
                                                         {p->d_weight, (uint64_t)p->dim * es}},
        out[3] = {{p->d_sum, span(p->rows, p->dim, p->ld_sum, es)}, {p->d_codes, span(p->rows, p->dim, p->ld_codes, 1)}, {p->d_scales, span(p->rows, nb, p->ld_scales, 4)}};
    for (int o = 0; o < 3; o++) {
        for (int i = 0; i < 3; i++) {
            const bool same = o == 0 && i < 2 && in[i].d == out[0].d && (i ? p->ld_residual : p->ld_x) == p->ld_sum;
            if (!same && overlap(out[o].d, out[o].n, in[i].d, in[i].n)) return he_fail(ctx, HE_ERR_BADARG, "he_rmsnorm_q8: an output overlaps an input");
        }
        for (int i = 0; i < o; i++)
            if (overlap(out[o].d, out[o].n, out[i].d, out[i].n)) return he_fail(ctx, HE_ERR_BADARG, "he_rmsnorm_q8: two outputs overlap");
    }
    const NormArgs a = {p->d_x, p->d_residual, p->d_weight, p->d_sum, p->d_codes, p->d_scales, p->ld_x, p->ld_residual, p->ld_sum, p->ld_codes, p->ld_scales, p->rows, p->dim, p->eps};
    with_dtype(p->dtype, [&](auto t) {
        using T = decltype(t);
        if (res) launch_norm<T, true>(a, ctx->stream);
        else launch_norm<T, false>(a, ctx->stream);
    });
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}
