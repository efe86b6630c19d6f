// A polynomial activation that keeps its input in 8 bits, and its gradients from what is kept.
#include "plain.h"

struct PolyArgs {
    const void* u;
    const float* coefs;
    void* y;
    uint8_t *codes, *exponents;
    u64 ld_u, ld_y, ld_codes, ld_exponents;
    uint32_t rows, dim, n_coefs, blocks, inverse;      // blocks of 128 columns a row; 2^32 / blocks, rounded up
};

// Byte of the smallest power of two from 2^-110 on at which 448 times it is at least the number of magnitude `most` (its bits without the sign):
// 448 is 1.75 * 2^8, so a fraction above 1.75 takes the next power.  255: not a finite number.  118 (2^-9)
// for zeros is a convention, as any power would do.
__device__ __forceinline__ uint32_t power_byte(uint32_t most) {
    if (most >= 0x7f800000u) return 255;
    if (most == 0) return 118;
    return (uint32_t)max((int32_t)((most + 0x1fffffu) >> 23) - 8, 17);
}
__device__ __forceinline__ float power_of(uint32_t byte) { return __builtin_bit_cast(float, byte == 255 ? 0x7fc00000u : byte << 23); }
// One over it; 0 for what is not finite, whose codes are set apart
__device__ __forceinline__ float inverse_power(uint32_t byte) { return byte == 255 ? 0.0f : __builtin_bit_cast(float, (254 - byte) << 23); }

// Where a block of 128 columns lies: blocks of all rows are counted through, and a row is found by a product with 2^32 / blocks, rounded up, which is
// at most one too many.
struct Place {
    uint32_t row, block;
    __device__ __forceinline__ Place(uint32_t unit, uint32_t blocks, uint32_t inverse) {
        row = __umulhi(unit, inverse);
        block = unit - row * blocks;
        if ((int32_t)block < 0) {
            row--;
            block += blocks;
        }
        if (inverse == 0) row = unit, block = 0;             // one block a row
    }
};
static uint32_t inverse_of(uint32_t blocks) { return (uint32_t)(((1ull << 32) + blocks - 1) / blocks); }

// Coefficients of a polynomial times f(i), the same in all lanes, read once; what is past them is 0
struct Coefs {
    float c[HE_POLY_MAX];
    template <class F> __device__ __forceinline__ Coefs(const float* coefs, uint32_t n, F f) {
#pragma unroll
        for (uint32_t i = 0; i < HE_POLY_MAX; i++)
            c[i] = i < n ? __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int32_t, coefs[i] * f(i)))) : 0.0f;
    }
};
// Coefficients from .. n - 1 as those of 1, u, ...
template <int FROM> __device__ __forceinline__ void horner(const Coefs& k, uint32_t n, const float* u, float* y) {
#pragma unroll
    for (int i = 0; i < 8; i++) y[i] = 0;
#pragma unroll
    for (int j = HE_POLY_MAX - 1; j >= FROM; j--)
        if (j < (int)n) {                                    // the same in all lanes
            if (j == (int)n - 1)
#pragma unroll
                for (int i = 0; i < 8; i++) y[i] = k.c[j];   // not 0 u + c: u may be infinite
            else
#pragma unroll
                for (int i = 0; i < 8; i++) y[i] = fmaf(y[i], u[i], k.c[j]);
        }
}

// Sixteen lanes a block of 128 columns, eight elements each: they find the largest among themselves.  A block at a time and many wavefronts: two or four at a
// time, their loads together, are no faster (16384 x 8192 bf16, degree 3, when work groups went on from block to block: 142 us, 143 and 146; gradients 145, 198 and 196, for
// want of registers).  Memory is what bounds it: 112 us, 6.0 TB/s; gradients 127 us, 5.3 TB/s (148 with
// the next block asked for ahead: its registers leave fewer wavefronts).
template <class T, bool Y> __global__ __launch_bounds__(256) void poly_q8_kernel(PolyArgs a) {
    using raw = typename T::raw;
    const uint32_t lane = threadIdx.x & 15, all = a.rows * a.blocks;
    const Coefs k(a.coefs, Y ? a.n_coefs : 0, [](uint32_t) { return 1.0f; });
    for (uint32_t unit = blockIdx.x * 16 + (threadIdx.x >> 4); unit < all; unit += gridDim.x * 16) {
        const Place p(unit, a.blocks, a.inverse);
        const uint32_t at = p.block * 128 + lane * 8;
        float u[8];
        load8<T>((const raw*)a.u + (u64)p.row * a.ld_u, at, a.dim, u);
        int32_t most = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) most = max(most, __builtin_bit_cast(int32_t, u[i]) & 0x7fffffff);
        most = row_max(most);
        const uint32_t byte = power_byte((uint32_t)most);
        const float inv = inverse_power(byte);
        uint32_t lo = __builtin_amdgcn_cvt_pk_fp8_f32(u[0] * inv, u[1] * inv, 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(u[4] * inv, u[5] * inv, 0, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(u[2] * inv, u[3] * inv, lo, true);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(u[6] * inv, u[7] * inv, hi, true);
        if (byte == 255) lo = hi = 0x7f7f7f7fu;
        if (lane == 0) a.exponents[(u64)p.row * a.ld_exponents + p.block] = (uint8_t)byte;
        uint8_t* codes = a.codes + (u64)p.row * a.ld_codes + at;
        if (at + 8 <= a.dim) *(uint2*)codes = make_uint2(lo, hi);
        else
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (at + i < a.dim) codes[i] = (uint8_t)((i < 4 ? lo : hi) >> 8 * (i & 3));
        if (Y) {
            float y[8];
            horner<0>(k, a.n_coefs, u, y);
            store8<T>((raw*)a.y + (u64)p.row * a.ld_y, at, a.dim, y);
        }
    }
}

extern "C" int32_t he_poly_q8(he_ctx* ctx, const he_poly_plan* p) {
    return he_guard(ctx, "he_poly_q8: host allocation failed", [&]() -> int32_t {
    if (!ctx) return HE_ERR_BADARG;
    HE_REFUSE(ctx, "he_poly_q8", refuse_poly(p));
    if (p->rows == 0) return HE_OK;
    const OnDevice device(ctx);
    HE_HIP(ctx, device.status);
    const PolyArgs a = {p->d_u, p->d_coefs, p->d_y, p->d_codes, p->d_exponents, p->ld_u, p->ld_y, p->ld_codes, p->ld_exponents, p->rows, p->dim, p->n_coefs, blocks_of(p->dim),
                        inverse_of(blocks_of(p->dim))};
    const uint32_t groups = poly_groups(p->rows, p->dim, HE_GROUPS_MAX);
    with_dtype(p->dtype, [&](auto t) {
        if (p->d_y) poly_q8_kernel<decltype(t), true><<<groups, 256, 0, ctx->stream>>>(a);
        else poly_q8_kernel<decltype(t), false><<<groups, 256, 0, ctx->stream>>>(a);
    });
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}

// ---- gradients

struct PolyGradArgs {
    const uint8_t *codes, *exponents;
    const float* coefs;
    const void* dy;
    void* du;
    double* parts;                            // [work groups][n_coefs], or null
    u64 ld_codes, ld_exponents, ld_dy, ld_du;
    uint32_t rows, dim, n_coefs, blocks, inverse;
};

// Sums of dy v^i: of a piece of eight elements in 32 bits, over pieces in 64; of two powers at a time, t = dy v^i as it is and times v.  SUMS: how many
// coefficients there may be sums for.
template <class T, int SUMS> __global__ __launch_bounds__(256) void poly_grad_kernel(PolyGradArgs a) {
    using raw = typename T::raw;
    __shared__ double sums[SUMS ? SUMS : 1][4];
    const uint32_t lane = threadIdx.x & 15, all = a.rows * a.blocks;
    const Coefs k(a.coefs, a.n_coefs, [](uint32_t i) { return (float)i; });
    double total[SUMS ? SUMS : 1] = {};
    for (uint32_t unit = blockIdx.x * 16 + (threadIdx.x >> 4); unit < all; unit += gridDim.x * 16) {
        const Place p(unit, a.blocks, a.inverse);
        const uint32_t at = p.block * 128 + lane * 8;
        if (at >= a.dim) continue;
        const uint32_t byte = a.exponents[(u64)p.row * a.ld_exponents + p.block];
        const float power = power_of(byte);
        const uint2 codes = *(const uint2*)(a.codes + (u64)p.row * a.ld_codes + at);       // there up to a multiple of 16
        float g[8], v[8], slope[8];
        load8<T>((const raw*)a.dy + (u64)p.row * a.ld_dy, at, a.dim, g);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const uint32_t w = i < 4 ? codes.x : codes.y;
            const auto pair = i & 2 ? __builtin_amdgcn_cvt_pk_f32_fp8(w, true) : __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
            v[i] = pair[0] * power;
            v[i + 1] = pair[1] * power;
        }
        if (at + 8 > a.dim)
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = at + i < a.dim ? v[i] : 0.0f;
        horner<1>(k, a.n_coefs, v, slope);
#pragma unroll
        for (int i = 0; i < 8; i++) slope[i] *= g[i];
        store8<T>((raw*)a.du + (u64)p.row * a.ld_du, at, a.dim, slope);
        auto add = [&](auto times) {                           // times(i): g[i] v[i]^2
#pragma unroll
            for (int j = 0; j < SUMS; j += 2) {
                float s = g[0], t = g[0] * v[0];
#pragma unroll
                for (int i = 1; i < 8; i++) {
                    s += g[i];
                    t = fmaf(g[i], v[i], t);
                }
                total[j] += s;
                if (j + 1 < SUMS) total[j + 1] += t;
                if (j + 2 < SUMS)
#pragma unroll
                    for (int i = 0; i < 8; i++) g[i] = times(i);
            }
        };
        // A square of its own 32 bits need not hold beside a g, so v is multiplied twice.  Of powers from 2^-54 to 2^54 it is a normal number, taken once for all g, which tells where
        // there are more than two of them (16384 x 8192 bf16, degree 8, 155 us, 161 without; degree 3 128, 126 without).
        if (SUMS > 4 && __all(byte - 73u <= 108u)) add([&](int i) { return g[i] * (v[i] * v[i]); });
        else add([&](int i) { return g[i] * v[i] * v[i]; });
    }
    if constexpr (SUMS > 0) {
#pragma unroll
        for (int j = 0; j < SUMS; j++) {
            double s = total[j];
            for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
            if ((threadIdx.x & 63) == 0) sums[j][threadIdx.x >> 6] = s;
        }
        __syncthreads();
        if (threadIdx.x < a.n_coefs) a.parts[(u64)blockIdx.x * a.n_coefs + threadIdx.x] = sums[threadIdx.x][0] + sums[threadIdx.x][1] + sums[threadIdx.x][2] + sums[threadIdx.x][3];
    }
}

// A coefficient a work group: the parts' sums
__global__ __launch_bounds__(256) void poly_join_kernel(const double* parts, uint32_t n, uint32_t n_coefs, float* dcoefs) {
    __shared__ double sums[256];
    double s = 0;
    for (uint32_t i = threadIdx.x; i < n; i += 256) s += parts[(u64)i * n_coefs + blockIdx.x];
    sums[threadIdx.x] = s;
    for (uint32_t d = 128; d; d >>= 1) {
        __syncthreads();
        if (threadIdx.x < d) sums[threadIdx.x] += sums[threadIdx.x + d];
    }
    if (threadIdx.x == 0) dcoefs[blockIdx.x] = (float)sums[0];
}

extern "C" int32_t he_work_poly_grad_q8(const he_ctx* ctx, const he_poly_grad_plan* p, uint64_t* h_bytes) {
    return he_guard(ctx, "he_work_poly_grad_q8: host allocation failed", [&]() -> int32_t {
    if (!ctx || !h_bytes) return HE_ERR_BADARG;
    HE_REFUSE(const_cast<he_ctx*>(ctx), "he_work_poly_grad_q8", refuse_poly_grad(p, true));
    *h_bytes = poly_grad_work(p);
    return HE_OK;
    });
}

extern "C" int32_t he_poly_grad_q8(he_ctx* ctx, const he_poly_grad_plan* p) {
    return he_guard(ctx, "he_poly_grad_q8: host allocation failed", [&]() -> int32_t {
    if (!ctx) return HE_ERR_BADARG;
    HE_REFUSE(ctx, "he_poly_grad_q8", refuse_poly_grad(p));
    const OnDevice device(ctx);
    HE_HIP(ctx, device.status);
    const uint32_t groups = p->rows ? poly_groups(p->rows, p->dim, p->d_dcoefs ? HE_POLY_GROUPS : HE_GROUPS_MAX) : 0;
    const PolyGradArgs a = {p->d_codes, p->d_exponents, p->d_coefs, p->d_dy, p->d_du, p->d_dcoefs ? (double*)p->d_work : nullptr, p->ld_codes, p->ld_exponents, p->ld_dy, p->ld_du,
                            p->rows, p->dim, p->n_coefs, blocks_of(p->dim), inverse_of(blocks_of(p->dim))};
    if (groups) with_dtype(p->dtype, [&](auto t) {
        using T = decltype(t);
        // sums for three, four, six or nine coefficients: more than there are cost their arithmetic
        if (!p->d_dcoefs) poly_grad_kernel<T, 0><<<groups, 256, 0, ctx->stream>>>(a);
        else if (p->n_coefs <= 3) poly_grad_kernel<T, 3><<<groups, 256, 0, ctx->stream>>>(a);
        else if (p->n_coefs <= 4) poly_grad_kernel<T, 4><<<groups, 256, 0, ctx->stream>>>(a);
        else if (p->n_coefs <= 6) poly_grad_kernel<T, 6><<<groups, 256, 0, ctx->stream>>>(a);
        else poly_grad_kernel<T, HE_POLY_MAX><<<groups, 256, 0, ctx->stream>>>(a);
    });
    if (p->d_dcoefs) poly_join_kernel<<<p->n_coefs, 256, 0, ctx->stream>>>((const double*)p->d_work, groups, p->n_coefs, p->d_dcoefs);
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}
