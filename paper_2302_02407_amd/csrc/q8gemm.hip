// Matrix product of 8-bit codes (e4m3) with a scale for each block of 128: out = A W^T, A [M][K], W [N][K].
#include "plain.h"

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
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

// ---- tiles staged in LDS
//
// A work group owns BN rows of W by BM rows of A and goes through the sum 128 columns (one block of scales) at a time.  Both operands'
// rows of 128 bytes come into LDS straight from memory, two buffers in turn: while one is multiplied the other is filled.  A wavefront
// owns TN x TM squares of 32 x 32; its rows of W lie in one block of scales, and every lane holds results of one row of A a square
// (the second operand's), so a block's sums need one factor a lane and square: 16 multiply-adds beside the 2 matrix instructions (64 passes
// each) that made them.
//
// The 16-byte piece c of row r lies at piece c ^ (r / 2 & 7): the lanes of a fragment read take the same piece of consecutive rows, and any
// sixteen of them, two rows of 128 bytes to a line of all 64 banks, cover every bank once.  The fills are spread over the first half of a
// block's squares: all at once they wait for the cache's 64 bytes a cycle and hold the wavefront's matrix instructions back.
//
// 8192 x 32768 x 4096 to bf16 1.08 ms (2030 TFLOP/s), exact sums to f32 2.15 ms (1020).  With no fills at all (on what lies there)
// the first takes 0.91 ms; the matrix instructions alone are 45% of its cycles, the multiply-adds 30%, and of the two kinds about half can
// run at a time (a pair of the first and 16 of the second take 172 cycles, not 130, with two wavefronts to a unit).
typedef const __attribute__((address_space(1))) void* gptr;
typedef __attribute__((address_space(3))) void* lptr;

template <int WN, int WM, int TN, int TM> struct Tile {
    static constexpr int BN = WN * TN * 32, BM = WM * TM * 32, THREADS = WN * WM * 64;
    static constexpr int BYTES = (BN + BM) * 128;      // a buffer
    static constexpr int SCALES = 8 * BM * 4;          // scales of A's rows, eight blocks at a time
    static constexpr int LDS = 2 * BYTES + 2 * SCALES;
};

__device__ __forceinline__ v16f zero16() { return v16f{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0}; }
// Pieces c and c + 1 of row r (r0 = the row's first byte)
__device__ __forceinline__ v8i fragment(const uint8_t* r0, uint32_t c, uint32_t r) {
    const v4i lo = *(const v4i*)(r0 + ((c ^ (r >> 1 & 7)) << 4)), hi = *(const v4i*)(r0 + (((c + 1) ^ (r >> 1 & 7)) << 4));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Which tile a work group owns.  Work groups go to the 8 dies in turn and each die has a cache of its own, so die x takes the x-th
// eighth of the tiles, in stripes of 8 tiles of A's rows: its 32 compute units then work on about 8 x 4 tiles at a time, which read
// 12 strips of rows instead of 33.
__device__ __forceinline__ bool tile_of(uint32_t tiles_n, uint32_t tiles_m, uint32_t& n, uint32_t& m) {
    const uint32_t all = tiles_n * tiles_m, each = (all + 7) / 8, t = blockIdx.x % 8 * each + blockIdx.x / 8;
    if (blockIdx.x / 8 >= each || t >= all) return false;
    const uint32_t stripe = t / (8 * tiles_n), high = min(8u, tiles_m - 8 * stripe), r = t - stripe * 8 * tiles_n;
    m = 8 * stripe + r % high;
    n = r / high;
    return true;
}

template <class T, bool FAST, int WN, int WM, int TN, int TM> __global__ __launch_bounds__(WN* WM * 64, 2) void matmul_q8_tiles_kernel(GemmArgs a) {
    using raw = typename T::raw;
    using G = Tile<WN, WM, TN, TM>;
    extern __shared__ __align__(1024) uint8_t lds[];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l = lane & 31, g = lane >> 5;
    const uint32_t wn = wave % WN, wm = wave / WN;
    uint32_t n0, m0;
    if (!tile_of((a.n + G::BN - 1) / G::BN, (a.m + G::BM - 1) / G::BM, n0, m0)) return;
    n0 *= G::BN;
    m0 *= G::BM;
    const uint32_t blocks = (a.k + 127) / 128;

    // a wavefront fills eight rows at a time: lane i the piece i % 8 of row i / 8
    constexpr int WAVES = WN * WM, FW = G::BN / 8 / WAVES, FA = G::BM / 8 / WAVES, FILLS = FW + FA;
    const uint8_t *w0 = a.w + n0 * a.ld_w, *a0 = a.a + m0 * a.ld_a;
    const uint32_t piece = (lane & 7) ^ ((wave & 1) * 4 + (lane >> 4));
    uint32_t off[FILLS];                               // ld <= 2^23: 256 rows stay below 2^31
#pragma unroll
    for (int f = 0; f < FILLS; f++) {
        const uint32_t r = ((f < FW ? f : f - FW) * WAVES + wave) * 8 + (lane >> 3);
        off[f] = f < FW ? min(r, a.n - 1 - n0) * (uint32_t)a.ld_w : min(r, a.m - 1 - m0) * (uint32_t)a.ld_a;
    }
    auto fill = [&](uint32_t b, int from, int end) {
        const uint32_t at = b * 128 + piece * 16, in = at < a.k ? at : 0;          // past the end: anything that is there, cleared below
        uint8_t* to = lds + (b & 1) * G::BYTES + wave * 1024;
#pragma unroll
        for (int f = from; f < end; f++)
            __builtin_amdgcn_global_load_lds((gptr)((f < FW ? w0 : a0) + (off[f] + in)), (lptr)(to + f * WAVES * 1024), 16, 0, 0);
    };
    float* scales = (float*)(lds + 2 * G::BYTES);
    const float* sw = a.sw + min(n0 + wn * TN * 32, a.n - 1) / 128 * a.ld_sw;
    v16f acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; i++)
#pragma unroll
        for (int j = 0; j < TM; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0;

    fill(0, 0, FILLS);
    for (uint32_t b = 0; b < blocks; b++) {
        if ((b & 7) == 0) {                              // scales of the next eight blocks
            float* to = scales + (b >> 3 & 1) * 8 * G::BM;
            for (uint32_t i = tid; i < 8 * G::BM; i += G::THREADS) {
                const uint32_t r = i / 8, c = b + i % 8;
                to[i % 8 * G::BM + r] = c < blocks ? a.sa[min(m0 + r, a.m - 1) * a.ld_sa + c] : 0.0f;
            }
        }
        const float swb = sw[b];
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (!FAST && b + 1 < blocks) fill(b + 1, 0, FILLS);
        uint8_t* buf = lds + (b & 1) * G::BYTES;
        if (b + 1 == blocks && (a.k & 127)) {            // columns past the end become zeros, in both operands
            const uint32_t left = a.k & 127;
            for (uint32_t i = tid; i < (G::BN + G::BM) * 8; i += G::THREADS) {
                const uint32_t r = i >> 3, c = (i & 7) ^ (r >> 1 & 7);
                v4i* p = (v4i*)(buf + i * 16);
                if (16 * c + 16 > left) *p = 16 * c < left ? keep(*p, (int)(left - 16 * c)) : v4i{0, 0, 0, 0};
            }
            __syncthreads();
        }
        float s[TM];
#pragma unroll
        for (int j = 0; j < TM; j++) s[j] = scales[((b >> 3 & 1) * 8 + (b & 7)) * G::BM + (wm * TM + j) * 32 + l] * swb;
        const uint8_t *wb = buf + (wn * TN * 32 + l) * 128, *ab = buf + (G::BN + wm * TM * 32 + l) * 128;
        if (FAST) {
            v8i af[TM][2];
#pragma unroll
            for (int j = 0; j < TM; j++)
#pragma unroll
                for (int h = 0; h < 2; h++) af[j][h] = fragment(ab + j * 4096, 4 * h + 2 * g, l);
#pragma unroll
            for (int i = 0; i < TN; i++) {
                v8i wf[2];
#pragma unroll
                for (int h = 0; h < 2; h++) wf[h] = fragment(wb + i * 4096, 4 * h + 2 * g, l);
#pragma unroll
                for (int j = 0; j < TM; j++) {
                    if (i < 2 && b + 1 < blocks) fill(b + 1, (i * TM + j) * FILLS / 4, (i * TM + j + 1) * FILLS / 4);
                    v16f p = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wf[0], af[j][0], zero16(), 0, 0, 0, 0, 0, 0);
                    p = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wf[1], af[j][1], p, 0, 0, 0, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 16; e++) acc[i][j][e] += p[e] * s[j];
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        } else {
            v8h af[TM][8];                               // piece 2c + g of a row: 32 columns at a time
#pragma unroll
            for (int j = 0; j < TM; j++)
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    const v4i v = *(const v4i*)(ab + j * 4096 + (((2 * c + g) ^ (l >> 1 & 7)) << 4));
                    af[j][2 * c] = halves(v[0], v[1]);
                    af[j][2 * c + 1] = halves(v[2], v[3]);
                }
#pragma unroll
            for (int i = 0; i < TN; i++) {
                v16f p[TM];
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    const v4i v = *(const v4i*)(wb + i * 4096 + (((2 * c + g) ^ (l >> 1 & 7)) << 4));
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        const v8h wf = halves(v[2 * h], v[2 * h + 1]);
#pragma unroll
                        for (int j = 0; j < TM; j++) p[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(wf, af[j][2 * c + h], c == 0 && h == 0 ? zero16() : p[j], 0, 0, 0);
                    }
                }
#pragma unroll
                for (int j = 0; j < TM; j++)
#pragma unroll
                    for (int e = 0; e < 16; e++) acc[i][j][e] += p[j][e] * s[j];
            }
        }
    }
    // Element e of a square: row 8 (e / 4) + 4 g + e % 4 of W, row l of A.  Results go out through LDS, 32 rows of a wavefront at a time,
    // so that a row's are written in a piece: TN * 32 in a row, 16 bytes a lane.
    constexpr int ES = sizeof(raw), PITCH = TN * 32 * ES + 16, LANES = TN * 32 * ES / 16;    // lanes a row
    static_assert(WAVES * 32 * PITCH <= G::LDS, "the staged results fit");
    uint8_t* mine = lds + wave * 32 * PITCH;
    const uint32_t nw = n0 + wn * TN * 32;
    const bool whole = !(((uintptr_t)a.out | a.ld_out * ES) & 15) && nw + TN * 32 <= a.n;
#pragma unroll
    for (int j = 0; j < TM; j++) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TN; i++)
#pragma unroll
            for (int q = 0; q < 4; q++) {
                raw v[4];
#pragma unroll
                for (int e = 0; e < 4; e++) v[e] = from_float<T>(acc[i][j][4 * q + e]);
                __builtin_memcpy(__builtin_assume_aligned(mine + l * PITCH + (i * 32 + 8 * q + 4 * g) * ES, 4 * ES), v, 4 * ES);
            }
        __syncthreads();
        const uint32_t mw = m0 + (wm * TM + j) * 32;
        if (whole) {
#pragma unroll
            for (int r = 0; r < 32; r += 64 / LANES) {
                const uint32_t row = r + lane / LANES, at = lane % LANES * 16;
                if (mw + row < a.m) *(v4i*)((uint8_t*)a.out + ((mw + row) * a.ld_out + nw) * ES + at) = *(const v4i*)(mine + row * PITCH + at);
            }
        } else {
            for (uint32_t r = 0; r < 32 && mw + r < a.m; r++)
                for (uint32_t n = lane; n < TN * 32 && nw + n < a.n; n += 64)
                    ((raw*)a.out)[(mw + r) * a.ld_out + nw + n] = ((const raw*)(mine + r * PITCH))[n];
        }
    }
}

template <class T, bool FAST, int WN, int WM, int TN, int TM> static hipError_t launch_tiles(const GemmArgs& a, hipStream_t stream) {
    using G = Tile<WN, WM, TN, TM>;
    const auto kernel = matmul_q8_tiles_kernel<T, FAST, WN, WM, TN, TM>;
    static const hipError_t ready = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS);
    if (ready != hipSuccess) return ready;
    const uint32_t tiles = ((a.n + G::BN - 1) / G::BN) * ((a.m + G::BM - 1) / G::BM);
    kernel<<<(tiles + 7) / 8 * 8, G::THREADS, G::LDS, stream>>>(a);
    return hipGetLastError();
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
    if (!ld_fits(p->ld_a, p->k) || !ld_fits(p->ld_w, p->k) || !ld_fits(p->ld_a_scales, kb) || !ld_fits(p->ld_w_scales, kb) || !ld_fits(p->ld_out, p->n) ||
        p->ld_a > (1u << 23) || p->ld_w > (1u << 23))
        return he_fail(ctx, HE_ERR_BADARG, "he_matmul_q8: an ld is below the row's length or above 2^28 (codes: 2^23)");
    if (((uintptr_t)p->d_a | p->ld_a | (uintptr_t)p->d_w | p->ld_w) & 15) return he_fail(ctx, HE_ERR_BADARG, "he_matmul_q8: rows of codes start at multiples of 16 bytes");
    if (((uintptr_t)p->d_a_scales | (uintptr_t)p->d_w_scales) & 3 || (uintptr_t)p->d_out & (es - 1))
        return he_fail(ctx, HE_ERR_BADARG, "he_matmul_q8: a pointer is not aligned to its elements");
    const uint64_t no = span(p->m, p->n, p->ld_out, es);
    if (overlap(p->d_out, no, p->d_a, span(p->m, k16, p->ld_a, 1)) || overlap(p->d_out, no, p->d_w, span(p->n, k16, p->ld_w, 1)) ||
        overlap(p->d_out, no, p->d_a_scales, span(p->m, kb, p->ld_a_scales, 4)) || overlap(p->d_out, no, p->d_w_scales, span(nb, kb, p->ld_w_scales, 4)))
        return he_fail(ctx, HE_ERR_BADARG, "he_matmul_q8: the output overlaps an operand");
    const GemmArgs a = {p->d_a, p->d_w, p->d_a_scales, p->d_w_scales, p->d_out, p->ld_a, p->ld_w, p->ld_a_scales, p->ld_w_scales, p->ld_out, p->m, p->n, p->k};
    hipError_t rc = hipSuccess;
    if (p->m > 64) {
        with_dtype(p->out_dtype, [&](auto t) {
            rc = p->fast_sums ? launch_tiles<decltype(t), true, 2, 4, 4, 2>(a, ctx->stream) : launch_tiles<decltype(t), false, 2, 4, 2, 2>(a, ctx->stream);
        });
        if (rc != hipSuccess) return he_fail(ctx, HE_ERR_HIP, "he_matmul_q8: %s", hipGetErrorString(rc));
        return HE_OK;
    }
    with_dtype(p->out_dtype, [&](auto t) { matmul_q8_kernel<decltype(t)><<<((p->n + 15) / 16) * ((p->m + 15) / 16), 64, 0, ctx->stream>>>(a); });
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}
