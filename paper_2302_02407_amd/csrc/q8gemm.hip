// Matrix product of 8-bit codes (e4m3) with a scale for each block of 128: out = A W^T, A [M][K], W [N][K].
#include "plain.h"

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

struct GemmArgs {
    const uint8_t *a, *w;
    const float *sa, *sw;
    void* out;
    u64 ld_a, ld_w, ld_sa, ld_sw, ld_out;
    uint32_t m, n, k;
};

// Eight codes as f16: exact, an e4m3 number has 4 bits of mantissa and 18 binary orders.
__device__ __forceinline__ v8h halves(uint32_t lo, uint32_t hi) {
    const v2h a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    const v2h c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
    return v8h{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The 16 x 16 products over 128 columns: rows of the first operand by lane % 16, of the second likewise, 32 columns by lane / 16 in
// both (any assignment of columns to lanes gives the same sum as long as both have it).  Lane l holds column l % 16 (a row of the
// second operand) of rows 4 * (l / 16) .. + 3 (of the first).  The codes go through the matrix instruction of f16, which adds in 32
// bits; the one of 8 bits aligns the products of a group to the largest and drops what lies 2^-13 below it.
__device__ __forceinline__ v4f mfma128(v8i a, v8i b) {
    v4f c = {0, 0, 0, 0};
#pragma unroll
    for (int h = 0; h < 4; h++) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves(a[2 * h], a[2 * h + 1]), halves(b[2 * h], b[2 * h + 1]), c, 0, 0, 0);
    return c;
}

// Columns at and after `left` of 16 become zeros (code 0)
__device__ __forceinline__ v4i keep(v4i v, int left) {
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const int n = left - 4 * j;
        v[j] = n >= 4 ? v[j] : n <= 0 ? 0 : v[j] & (int)((1u << (8 * n)) - 1);
    }
    return v;
}

// A lane's 32 codes of a row from column `at`, zeros from column k on
__device__ __forceinline__ v8i codes32(const uint8_t* row, uint32_t at, uint32_t k) {
    v4i lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
    if (at < k) lo = keep(*(const v4i*)(row + at), (int)min(k - at, 16u));
    if (at + 16 < k) hi = keep(*(const v4i*)(row + at + 16), (int)min(k - at - 16, 16u));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// One wavefront a tile of 16 x 16, operands straight from memory
template <class T> __global__ __launch_bounds__(64) void matmul_q8_kernel(GemmArgs a) {
    using raw = typename T::raw;
    const uint32_t l = threadIdx.x & 15, g = threadIdx.x >> 4, tiles_n = (a.n + 15) / 16;
    const uint32_t m = blockIdx.x / tiles_n * 16 + l, n0 = blockIdx.x % tiles_n * 16;
    const uint32_t mr = min(m, a.m - 1), nr = min(n0 + l, a.n - 1);
    const uint8_t *ar = a.a + mr * a.ld_a, *wr = a.w + nr * a.ld_w;
    const float *sa = a.sa + mr * a.ld_sa, *sw = a.sw + (n0 >> 7) * a.ld_sw;
    v4f acc = {0, 0, 0, 0};
    for (uint32_t k = 0; k < a.k; k += 128) {
        const v4f p = mfma128(codes32(wr, k + 32 * g, a.k), codes32(ar, k + 32 * g, a.k));
        const float s = sa[k >> 7] * sw[k >> 7];
        acc += p * s;
    }
    raw* out = (raw*)a.out + (u64)m * a.ld_out;
    if (m < a.m)
#pragma unroll
        for (uint32_t j = 0; j < 4; j++)
            if (n0 + 4 * g + j < a.n) out[n0 + 4 * g + j] = from_float<T>(acc[j]);
}

extern "C" int32_t he_matmul_q8(he_ctx* ctx, const he_matmul_plan* p) {
    return he_guard(ctx, "he_matmul_q8: host allocation failed", [&]() -> int32_t {
    if (!ctx) return HE_ERR_BADARG;
    if (!p) return he_fail(ctx, HE_ERR_BADARG, "he_matmul_q8: null plan");
    if (!dtype_known(p->out_dtype)) return he_fail(ctx, HE_ERR_BADARG, "he_matmul_q8: unknown type %d", p->out_dtype);
    if (p->k == 0 || p->k > (1u << 20)) return he_fail(ctx, HE_ERR_BADARG, "he_matmul_q8: %u columns to sum over, outside 1..2^20", p->k);
    if (p->m > (1u << 20) || p->n > (1u << 20)) return he_fail(ctx, HE_ERR_BADARG, "he_matmul_q8: more than 2^20 rows");
    if ((uint64_t)p->m * p->n > 1ull << 33) return he_fail(ctx, HE_ERR_BADARG, "he_matmul_q8: more than 2^33 results");
    if (p->m == 0 || p->n == 0) return HE_OK;
    if (!p->d_a || !p->d_w || !p->d_a_scales || !p->d_w_scales || !p->d_out) return he_fail(ctx, HE_ERR_BADARG, "he_matmul_q8: null argument");
    const uint32_t kb = (p->k + 127) / 128, nb = (p->n + 127) / 128, es = dtype_bytes(p->out_dtype);
    const uint64_t k16 = (p->k + 15ull) & ~15ull;
    if (!ld_fits(p->ld_a, p->k) || !ld_fits(p->ld_w, p->k) || !ld_fits(p->ld_a_scales, kb) || !ld_fits(p->ld_w_scales, kb) || !ld_fits(p->ld_out, p->n))
        return he_fail(ctx, HE_ERR_BADARG, "he_matmul_q8: an ld is below the row's length or above 2^28");
    if (((uintptr_t)p->d_a | p->ld_a | (uintptr_t)p->d_w | p->ld_w) & 15) return he_fail(ctx, HE_ERR_BADARG, "he_matmul_q8: rows of codes start at multiples of 16 bytes");
    if (((uintptr_t)p->d_a_scales | (uintptr_t)p->d_w_scales) & 3 || (uintptr_t)p->d_out & (es - 1))
        return he_fail(ctx, HE_ERR_BADARG, "he_matmul_q8: a pointer is not aligned to its elements");
    const uint64_t no = span(p->m, p->n, p->ld_out, es);
    if (overlap(p->d_out, no, p->d_a, span(p->m, k16, p->ld_a, 1)) || overlap(p->d_out, no, p->d_w, span(p->n, k16, p->ld_w, 1)) ||
        overlap(p->d_out, no, p->d_a_scales, span(p->m, kb, p->ld_a_scales, 4)) || overlap(p->d_out, no, p->d_w_scales, span(nb, kb, p->ld_w_scales, 4)))
        return he_fail(ctx, HE_ERR_BADARG, "he_matmul_q8: the output overlaps an operand");
    const GemmArgs a = {p->d_a, p->d_w, p->d_a_scales, p->d_w_scales, p->d_out, p->ld_a, p->ld_w, p->ld_a_scales, p->ld_w_scales, p->ld_out, p->m, p->n, p->k};
    with_dtype(p->out_dtype, [&](auto t) { matmul_q8_kernel<decltype(t)><<<((p->n + 15) / 16) * ((p->m + 15) / 16), 64, 0, ctx->stream>>>(a); });
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}
