// The gradient of a linear layer's weight from its input as kept in 8 bits: dw[n][k] = sum over m of dy[m][n] v[m][k].
//
// What is kept is a code of 4 significant bits times a power of two, a bfloat16 number exactly.  dy is cut into bfloat16 numbers exactly too, 8 of its
// significant bits at a time: one of them for bf16, two for f16, three for f32.  So the matrix instruction of bfloat16 takes products that are
// exact, and adds in 32 bits.
#include "plain.h"

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

struct WeightArgs {
    const void* dy;
    const uint8_t *codes, *exponents;
    void* dw;
    u64 ld_dy, ld_codes, ld_exponents, ld_dw;
    uint32_t m, n, k;
    uint32_t per;              // steps of 32 rows a part takes
    u64 part;                  // elements from one part's sums to the next's
    uint32_t accumulate;
};

template <class T> struct Parts;
template <> struct Parts<bf16_t> { static constexpr int N = 1; };
template <> struct Parts<f16_t> { static constexpr int N = 2; };
template <> struct Parts<f32_t> { static constexpr int N = 3; };

// The upper half of a number of 32 bits, and what it leaves: nothing of an infinity
__device__ __forceinline__ uint32_t upper(float& x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x) & 0xffff0000u;
    x = (b & 0x7fffffffu) == 0x7f800000u && x == x ? 0.0f : x - __builtin_bit_cast(float, b);
    return b >> 16;
}

template <class T, class O> __global__ __launch_bounds__(256) void weight_grad_kernel(WeightArgs a) {
    using raw = typename T::raw;
    constexpr int PARTS = Parts<T>::N, PITCH = 80;               // 32 rows of m, 2 bytes each, and 16 more against bank conflicts
    __shared__ __align__(16) uint8_t lds[(PARTS + 1) * 128 * PITCH];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l = lane & 31, g = lane >> 5;
    const uint32_t tiles_k = (a.k + 127) / 128, n0 = blockIdx.x / tiles_k * 128, k0 = blockIdx.x % tiles_k * 128;
    const uint32_t steps = min((a.m + 31) / 32 - blockIdx.y * a.per, a.per), first = blockIdx.y * a.per * 32;
    const raw* dy = (const raw*)a.dy;
    v16f acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
        for (int j = 0; j < 2; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0;
    for (uint32_t s = 0; s < steps; s++) {
        // eight rows of two columns a thread, each column's eight together
        const uint32_t m0 = first + s * 32 + wave * 8;
        __syncthreads();
#pragma unroll
        for (int c = 0; c < 2; c++) {
            const uint32_t col = 2 * lane + c, n = n0 + col, k = k0 + col;
            uint16_t y[PARTS][8], x[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                float v = n < a.n && m0 + i < a.m ? to_float<T>(dy[(u64)(m0 + i) * a.ld_dy + n]) : 0.0f;
#pragma unroll
                for (int q = 0; q < PARTS; q++) y[q][i] = (uint16_t)upper(v);
                float u = 0;
                if (k < a.k && m0 + i < a.m) {
                    const uint32_t byte = a.exponents[(u64)(m0 + i) * a.ld_exponents + k / 128], code = a.codes[(u64)(m0 + i) * a.ld_codes + k];
                    u = __builtin_amdgcn_cvt_f32_fp8(code, 0) * __builtin_bit_cast(float, byte == 255 ? 0x7fc00000u : byte << 23);
                }
                x[i] = (uint16_t)(__builtin_bit_cast(uint32_t, u) >> 16);
            }
#pragma unroll
            for (int q = 0; q < PARTS; q++) __builtin_memcpy(__builtin_assume_aligned(lds + (q * 128 + col) * PITCH + wave * 16, 16), y[q], 16);
            __builtin_memcpy(__builtin_assume_aligned(lds + (PARTS * 128 + col) * PITCH + wave * 16, 16), x, 16);
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; h++) {
            v8b xf[2];
#pragma unroll
            for (int j = 0; j < 2; j++) xf[j] = *(const v8b*)(lds + (PARTS * 128 + (wave & 1) * 64 + j * 32 + l) * PITCH + (2 * h + g) * 16);
#pragma unroll
            for (int q = PARTS - 1; q >= 0; q--)
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const v8b yf = *(const v8b*)(lds + (q * 128 + (wave >> 1) * 64 + i * 32 + l) * PITCH + (2 * h + g) * 16);
#pragma unroll
                    for (int j = 0; j < 2; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(yf, xf[j], acc[i][j], 0, 0, 0);
                }
        }
    }
    // element e of a square: row 8 (e / 4) + 4 g + e % 4, column l
    typename O::raw* dw = (typename O::raw*)a.dw + blockIdx.y * a.part;
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
        for (int j = 0; j < 2; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) {
                const uint32_t n = n0 + (wave >> 1) * 64 + i * 32 + 8 * (e / 4) + 4 * g + e % 4, k = k0 + (wave & 1) * 64 + j * 32 + l;
                if (n >= a.n || k >= a.k) continue;
                typename O::raw* to = dw + n * a.ld_dw + k;
                *to = from_float<O>(a.accumulate ? to_float<O>(*to) + acc[i][j][e] : acc[i][j][e]);
            }
}

// Sums the parts, in order
template <class O> __global__ __launch_bounds__(256) void weight_join_kernel(const float* parts, uint32_t n_parts, u64 part, u64 ld_part, typename O::raw* dw, u64 ld_dw, uint32_t k, uint32_t accumulate) {
    const uint32_t i = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= k) return;
    const float* p = parts + blockIdx.y * ld_part + i;
    v4f x = {0, 0, 0, 0};
    for (uint32_t q = 0; q < n_parts; q++) x += *(const v4f*)(p + q * part);
#pragma unroll
    for (uint32_t e = 0; e < 4; e++)
        if (i + e < k) {
            typename O::raw* to = dw + blockIdx.y * ld_dw + i + e;
            *to = from_float<O>(accumulate ? to_float<O>(*to) + x[e] : x[e]);
        }
}

extern "C" int32_t he_work_weight_grad_q8(const he_ctx* ctx, const he_weight_grad_plan* p, uint64_t* h_bytes) {
    return he_guard(ctx, "he_work_weight_grad_q8: host allocation failed", [&]() -> int32_t {
    if (!ctx || !h_bytes) return HE_ERR_BADARG;
    HE_REFUSE(const_cast<he_ctx*>(ctx), "he_work_weight_grad_q8", refuse_weight_grad(p, true));
    *h_bytes = weight_grad_work(p);
    return HE_OK;
    });
}

extern "C" int32_t he_weight_grad_q8(he_ctx* ctx, const he_weight_grad_plan* p) {
    return he_guard(ctx, "he_weight_grad_q8: host allocation failed", [&]() -> int32_t {
    if (!ctx) return HE_ERR_BADARG;
    HE_REFUSE(ctx, "he_weight_grad_q8", refuse_weight_grad(p));
    if (p->n == 0 || p->k == 0 || (p->m == 0 && p->accumulate)) return HE_OK;
    const OnDevice device(ctx);
    HE_HIP(ctx, device.status);
    const WeightCut c = weight_cut(p->m, p->n, p->k);
    const bool joined = p->m == 0 || c.parts > 1;
    WeightArgs a = {p->d_dy, p->d_codes, p->d_exponents, p->d_dw, p->ld_dy, p->ld_codes, p->ld_exponents, p->ld_dw, p->m, p->n, p->k, c.per, 0, p->accumulate};
    if (joined) {
        a.dw = p->d_work;
        a.ld_dw = weight_pitch(p->k);
        a.part = p->n * a.ld_dw;
        a.accumulate = 0;
    }
    const dim3 grid(((p->n + 127) / 128) * ((p->k + 127) / 128), c.parts);
    with_dtype(p->out_dtype, [&](auto o) {
        using O = decltype(o);
        if (p->m) with_dtype(p->dtype, [&](auto t) {
            using T = decltype(t);
            if (joined) weight_grad_kernel<T, f32_t><<<grid, 256, 0, ctx->stream>>>(a);
            else weight_grad_kernel<T, O><<<grid, 256, 0, ctx->stream>>>(a);
        });
        if (joined)
            for (uint32_t r = 0; r < p->n; r += 65535)    // a grid's second side
                weight_join_kernel<O><<<dim3((p->k + 1023) / 1024, min(p->n - r, 65535u)), 256, 0, ctx->stream>>>(
                    (const float*)p->d_work + r * a.ld_dw, p->m ? c.parts : 0, a.part, a.ld_dw, (typename O::raw*)p->d_dw + r * p->ld_dw, p->ld_dw, p->k, p->accumulate);
    });
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}
