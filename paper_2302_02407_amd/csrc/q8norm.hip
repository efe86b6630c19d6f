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
    uint32_t dim;
    float eps;
};

// |y| as an integer: ordered like the numbers, infinity above them and NaN above that, so that a maximum keeps both
__device__ __forceinline__ uint32_t magnitude(float y) { return __builtin_bit_cast(uint32_t, y) & 0x7fffffffu; }

// One row a work group: the sum of squares, then a block of 128 columns at a time by each wavefront, two columns a lane.
template <class T, bool RES, bool WEIGHT> __global__ __launch_bounds__(256) void rmsnorm_q8_kernel(NormArgs a) {
    using raw = typename T::raw;
    __shared__ float room[4];
    const u64 row = blockIdx.x;
    const raw* x = (const raw*)a.x + row * a.ld_x;
    const raw* res = (const raw*)a.res + row * a.ld_res;
    const raw* w = (const raw*)a.weight;
    raw* sum = (raw*)a.sum + row * a.ld_sum;
    uint8_t* codes = a.codes + row * a.ld_codes;
    float* scales = a.scales + row * a.ld_scales;
    float sq = 0;
    for (uint32_t i = threadIdx.x; i < a.dim; i += 256) {
        float h = to_float<T>(x[i]);
        if (RES) h += to_float<T>(res[i]);
        sq += h * h;
    }
    sq = group_sum<4>(sq, room);
    const float r = 1.0f / sqrtf(sq / (float)a.dim + a.eps);
    const uint32_t lane = threadIdx.x & 63;
    for (uint32_t b = threadIdx.x >> 6; b * Q8_BLOCK < a.dim; b += 4) {
        float y[2];
        uint32_t most = 0;
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const uint32_t i = b * Q8_BLOCK + lane + 64 * u;
            y[u] = 0;
            if (i < a.dim) {
                float h = to_float<T>(x[i]);
                if (RES) h += to_float<T>(res[i]);
                if (RES) sum[i] = from_float<T>(h);
                y[u] = h * r;
                if (WEIGHT) y[u] *= to_float<T>(w[i]);
            }
            most = max(most, magnitude(y[u]));
        }
#pragma unroll
        for (int o = 32; o; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o));
        const float scale = __builtin_bit_cast(float, most) / Q8_MAX;
        if (lane == 0) scales[b] = scale;
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const uint32_t i = b * Q8_BLOCK + lane + 64 * u;
            const float v = scale == 0.0f ? 0.0f : y[u] / scale;
            if (i < a.dim) codes[i] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false);
        }
    }
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
    const NormArgs a = {p->d_x, p->d_residual, p->d_weight, p->d_sum, p->d_codes, p->d_scales, p->ld_x, p->ld_residual, p->ld_sum, p->ld_codes, p->ld_scales, p->dim, p->eps};
    with_dtype(p->dtype, [&](auto t) {
        using T = decltype(t);
        if (res && p->d_weight) rmsnorm_q8_kernel<T, true, true><<<p->rows, 256, 0, ctx->stream>>>(a);
        else if (res) rmsnorm_q8_kernel<T, true, false><<<p->rows, 256, 0, ctx->stream>>>(a);
        else if (p->d_weight) rmsnorm_q8_kernel<T, false, true><<<p->rows, 256, 0, ctx->stream>>>(a);
        else rmsnorm_q8_kernel<T, false, false><<<p->rows, 256, 0, ctx->stream>>>(a);
    });
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}
