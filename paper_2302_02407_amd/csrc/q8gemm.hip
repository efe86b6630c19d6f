// Matrix product of 8-bit codes (e4m3) with a scale for each block of 128: out = A W^T, A [M][K], W [N][K].
#include "plain.h"

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v4i_any __attribute__((ext_vector_type(4), aligned(2)));
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
    uint32_t per;      // tiles: blocks of 128 columns a part of the sum's axis takes
    u64 part;          // ... and elements from one part's results to the next's
};

// Eight codes as f16: exact, an e4m3 number has 4 bits of mantissa and 18 binary orders.
__device__ __forceinline__ v8h halves(uint32_t lo, uint32_t hi) {
    const v2h a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    const v2h c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
    return v8h{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
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

// ---- few rows of A and W straight from memory
//
// A wavefront owns NT times 16 rows of W by MT times 16 rows of A and every KS-th block of 128 columns; the KS wavefronts of a work group
// join their sums in LDS, in order.  KS is chosen so that about 8192 wavefronts are there: what bounds it is W's bytes (or, where
// there are few of them, one launch's latency), and the pieces on the way of 32 wavefronts to a compute unit keep memory busy.  A and
// the scales come from the caches, A's pieces once for the NT tiles.  Pieces of 16 bytes go to lanes so that four lanes side by side read
// 64 bytes of a row; any assignment of columns to lanes gives the same products as long as both operands have it.  Codes go through
// the matrix instruction of f16, which adds in 32 bits: exact, and not what bounds it.  Every wavefront asks for one block more than it
// multiplies, whichever is the last.
template <class T, int NT, int MT> __global__ __launch_bounds__(1024) void matmul_q8_few_kernel(GemmArgs a) {
    using raw = typename T::raw;
    constexpr int PITCH = 20;
    extern __shared__ float sums[];                                                   // [KS][NT][MT][16 rows of A][PITCH]
    const uint32_t lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4, ks = blockDim.x / 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t n0 = blockIdx.x * (16 * NT), blocks = (a.k + 127) / 128;
    const uint8_t *wr[NT], *ar[MT];
    const float *sw = a.sw + (n0 >> 7) * a.ld_sw, *sa[MT];
    v4f acc[NT][MT];
#pragma unroll
    for (int j = 0; j < MT; j++) {
        const uint64_t m = min(16 * j + l, a.m - 1);
        ar[j] = a.a + m * a.ld_a;
        sa[j] = a.sa + m * a.ld_sa;
    }
#pragma unroll
    for (int i = 0; i < NT; i++) {
        wr[i] = a.w + min(n0 + 16 * i + l, a.n - 1) * a.ld_w;
#pragma unroll
        for (int j = 0; j < MT; j++) acc[i][j] = v4f{0, 0, 0, 0};
    }
    struct Pieces {
        v4i w[NT][2], a[MT][2];
        float s[MT];
    };
    auto load = [&](uint32_t b, Pieces& p) {
#pragma unroll
        for (int c = 0; c < 2; c++) {
            const uint32_t at = b * 128 + (c * 4 + g) * 16, in = at < a.k ? at : 0;       // past the end: cleared when it is used
#pragma unroll
            for (int i = 0; i < NT; i++) p.w[i][c] = *(const v4i*)(wr[i] + in);
#pragma unroll
            for (int j = 0; j < MT; j++) p.a[j][c] = *(const v4i*)(ar[j] + in);
        }
        const float swb = sw[b];
#pragma unroll
        for (int j = 0; j < MT; j++) p.s[j] = sa[j][b] * swb;
    };
    auto multiply = [&](uint32_t b, Pieces& p) {
        v4f x[NT][MT];
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
            for (int j = 0; j < MT; j++) x[i][j] = v4f{0, 0, 0, 0};
        const bool cut = (b + 1) * 128 > a.k;
#pragma unroll
        for (int c = 0; c < 2; c++) {
            if (cut) {
                const int left = max(0, (int)a.k - (int)(b * 128 + (c * 4 + g) * 16));
#pragma unroll
                for (int j = 0; j < MT; j++) p.a[j][c] = keep(p.a[j][c], left);
#pragma unroll
                for (int i = 0; i < NT; i++) p.w[i][c] = keep(p.w[i][c], left);
            }
#pragma unroll
            for (int h = 0; h < 2; h++) {
                v8h y[MT];
#pragma unroll
                for (int j = 0; j < MT; j++) y[j] = halves(p.a[j][c][2 * h], p.a[j][c][2 * h + 1]);
#pragma unroll
                for (int i = 0; i < NT; i++) {
                    const v8h w = halves(p.w[i][c][2 * h], p.w[i][c][2 * h + 1]);
#pragma unroll
                    for (int j = 0; j < MT; j++) x[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w, y[j], x[i][j], 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
            for (int j = 0; j < MT; j++) acc[i][j] += x[i][j] * p.s[j];
    };
    if (wave < blocks) {
        Pieces one, two;
        load(wave, one);
        for (uint32_t b = wave; b < blocks; b += 2 * ks) {
            load(min(b + ks, blocks - 1), two);
            multiply(b, one);
            if (b + ks < blocks) {
                load(min(b + 2 * ks, blocks - 1), one);
                multiply(b + ks, two);
            }
        }
    }
    // element e: row 4 g + e of W, row l of A
#pragma unroll
    for (int i = 0; i < NT; i++)
#pragma unroll
        for (int j = 0; j < MT; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) sums[(((wave * NT + i) * MT + j) * 16 + l) * PITCH + 4 * g + e] = acc[i][j][e];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 256 * NT * MT; i += blockDim.x) {
        const uint32_t r = i / (16 * NT), n = i % (16 * NT);
        if (r >= a.m || n0 + n >= a.n) continue;
        float x = 0;
        for (uint32_t k = 0; k < ks; k++) x += sums[(((k * NT + n / 16) * MT + r / 16) * 16 + r % 16) * PITCH + n % 16];
        ((raw*)a.out)[r * a.ld_out + n0 + n] = from_float<T>(x);
    }
}

// With up to 32 rows of A: products whose W has less than 32 MiB, where the tiles below would need a second launch for the parts of the
// sum's axis (16 x 1000 x 2048: 6.8 us, there 9.7; 16 x 10007 x 4096: 22.6, there 13.4), and those of up to 4 rows with so many of W that
// the tiles come in one round and a third (1 x 131072 x 4096: 107 us, there 131; with 16 rows 148, there 134).  4 rows and 98304 were drawn
// between these and 1 x 32768 x 4096, not measured; other W whose tiles end in a part of a round go by the same line.
static bool few_rows(uint32_t m, uint32_t n, uint32_t k) { return m <= 32 && ((uint64_t)n * k < 1u << 25 || (m <= 4 && n > 98304)); }

template <class T, int NT, int MT> static hipError_t launch_few(const GemmArgs& a, hipStream_t stream) {
    const auto kernel = matmul_q8_few_kernel<T, NT, MT>;
    constexpr int LDS = NT * MT * 16 * 20 * 4;           // a wavefront
    static const hipError_t ready = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 16 * LDS);
    if (ready != hipSuccess) return ready;
    const uint32_t blocks = (a.k + 127) / 128, tiles = (a.n + 16 * NT - 1) / (16 * NT);
    uint32_t ks = 1;
    while (ks < 16 && ks < blocks && tiles * ks < 8192) ks *= 2;
    kernel<<<tiles, 64 * ks, ks * LDS, stream>>>(a);
    return hipGetLastError();
}
template <class T> static hipError_t run_few(const GemmArgs& a, hipStream_t stream) {
    if (a.m <= 16) return a.n >= 16384 ? launch_few<T, 2, 1>(a, stream) : launch_few<T, 1, 1>(a, stream);     // two tiles a wavefront where that fills the card
    return launch_few<T, 1, 2>(a, stream);
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
// 8192 x 32768 x 4096 to bf16 1.03 to 1.07 ms by card (2130 to 2060 TFLOP/s), exact sums to f32 2.07 to 2.12 ms (1060).  With no fills at all (on what lies there)
// the first takes 0.91 ms; matrix instructions fill 51% of its cycles and the multiply-adds 26% (counted), and of the two kinds about half can
// run at a time (a pair of the first and 16 of the second take 172 cycles, not 130, with two wavefronts to a unit).  So a square's
// multiply-adds stand between the next one's two instructions: with them behind its own, 1.09 ms, and 777 x 10007 x 2040 38.5 us, not
// 35.9.  A third buffer does not fit beside the largest tile, and beside the smaller ones it takes the room of a second work group, which
// covers more (777 x 10007 x 2040 44 us); asking for lines two or three blocks early, so that fills find them in the
// die's cache, takes 1.11 ms.
typedef const __attribute__((address_space(1))) void* gptr;
typedef __attribute__((address_space(3))) void* lptr;
typedef const __attribute__((address_space(4))) float* cptr;    // read by scalar loads

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

// A tile's rows from one column on, for loads that check their bounds: what lies past the last row, or past the last row's k columns (to a
// multiple of 16), comes as zeros.  So no lane holds an offset for every row it loads, and there is room for the results of two squares.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_from(const uint8_t* p, uint32_t rows, uint32_t ld, uint32_t k) {
    constexpr int RAW_DWORDS = 0x00027000;               // word 3 of a descriptor without a stride: offsets are compared with the size in bytes
    return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, (min(rows, 256u) - 1) * ld + (k + 15) / 16 * 16, RAW_DWORDS);    // ld <= 2^23: below 2^32
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
    const uint32_t first = blockIdx.y * a.per, blocks = min((a.k + 127) / 128 - first, a.per), k = a.k - first * 128;     // this part's

    // a wavefront fills eight rows at a time: lane i the piece i % 8 of row i / 8
    constexpr int WAVES = WN * WM, FW = G::BN / 8 / WAVES, FA = G::BM / 8 / WAVES, FILLS = FW + FA;
    const auto w_rows = rows_from(a.w + n0 * a.ld_w + first * 128, a.n - n0, (uint32_t)a.ld_w, k);
    const auto a_rows = rows_from(a.a + m0 * a.ld_a + first * 128, a.m - m0, (uint32_t)a.ld_a, k);
    const uint32_t r0 = wave * 8 + (lane >> 3), piece = (lane & 7) ^ ((wave & 1) * 4 + (lane >> 4));
    const uint32_t w_at = r0 * (uint32_t)a.ld_w + piece * 16, w_step = WAVES * 8 * (uint32_t)a.ld_w;
    const uint32_t a_at = r0 * (uint32_t)a.ld_a + piece * 16, a_step = WAVES * 8 * (uint32_t)a.ld_a;
    auto fill = [&](uint32_t b, int from, int end) {     // pieces past the k columns: anything that is there, cleared below
        uint8_t* to = lds + (b & 1) * G::BYTES + wave * 1024;
#pragma unroll
        for (int f = from; f < end; f++)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(f < FW ? w_rows : a_rows, (lptr)(to + f * WAVES * 1024), 16,
                                                     f < FW ? w_at + (f * w_step + b * 128) : a_at + ((f - FW) * a_step + b * 128), 0, 0, 0);
    };
    float* scales = (float*)(lds + 2 * G::BYTES);        // [2][BM rows][8 blocks]
    // Of blocks b .. b + 7, b a multiple of 8; asked for 4 blocks early, as loads to registers they would be waited for (1024 x 4096 x 4096
    // to bf16 31.4 us, 32.5 then; exact sums of large tiles 2.07 ms, 2.04 then).
    auto fill_scales = [&](uint32_t b) {
#pragma unroll
        for (int i = 0; i < G::BM / 8 / WAVES; i++) {
            const uint32_t at = i * WAVES + wave, r = at * 8 + (lane >> 3), c = min(b + (lane & 7), blocks - 1);
            __builtin_amdgcn_global_load_lds((gptr)(a.sa + min(m0 + r, a.m - 1) * a.ld_sa + first + c), (lptr)(scales + (b >> 3 & 1) * 8 * G::BM + at * 64), 4, 0, 0);
        }
    };
    const cptr sw = (cptr)(uintptr_t)(a.sw + min(n0 + wn * TN * 32, a.n - 1) / 128 * a.ld_sw + first);
    float swb = sw[0];
    v16f acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; i++)
#pragma unroll
        for (int j = 0; j < TM; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0;

    fill_scales(0);
    fill(0, 0, FILLS);
    for (uint32_t b = 0; b < blocks; b++) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __syncthreads();
        if ((b & 7) == 4 && b + 4 < blocks) fill_scales(b + 4);
        if (!FAST && b + 1 < blocks) fill(b + 1, 0, FILLS);
        uint8_t* buf = lds + (b & 1) * G::BYTES;
        if (b + 1 == blocks && b * 128 + 128 > k) {            // columns past the end become zeros, in both operands
            const uint32_t left = k & 127;
            for (uint32_t i = tid; i < (G::BN + G::BM) * 8; i += G::THREADS) {
                const uint32_t r = i >> 3, c = (i & 7) ^ (r >> 1 & 7);
                v4i* p = (v4i*)(buf + i * 16);
                if (16 * c + 16 > left) *p = 16 * c < left ? keep(*p, (int)(left - 16 * c)) : v4i{0, 0, 0, 0};
            }
            __syncthreads();
        }
        float s[TM];
#pragma unroll
        for (int j = 0; j < TM; j++) s[j] = scales[(b >> 3 & 1) * 8 * G::BM + ((wm * TM + j) * 32 + l) * 8 + (b & 7)] * swb;
        if (b + 1 < blocks) swb = sw[b + 1];
        const uint8_t *wb = buf + (wn * TN * 32 + l) * 128, *ab = buf + (G::BN + wm * TM * 32 + l) * 128;
        if (FAST) {
            v8i af[TM][2];
#pragma unroll
            for (int j = 0; j < TM; j++)
#pragma unroll
                for (int h = 0; h < 2; h++) af[j][h] = fragment(ab + j * 4096, 4 * h + 2 * g, l);
            v16f p[2];                                   // of square q, and of the one before, which joins the sums meanwhile
            v8i wf[2];
#pragma unroll
            for (int q = 0; q <= TN * TM; q++) {
                const int i = q / TM, j = q % TM;
                if (q < TN * TM && j == 0)
#pragma unroll
                    for (int h = 0; h < 2; h++) wf[h] = fragment(wb + i * 4096, 4 * h + 2 * g, l);
                constexpr int HALF = (TN * TM + 1) / 2;
                if (q < HALF && b + 1 < blocks) fill(b + 1, q * FILLS / HALF, (q + 1) * FILLS / HALF);
                if (q < TN * TM) p[q & 1] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wf[0], af[j][0], zero16(), 0, 0, 0, 0, 0, 0);
                if (q)
#pragma unroll
                    for (int e = 0; e < 8; e++) acc[(q - 1) / TM][(q - 1) % TM][e] += p[~q & 1][e] * s[(q - 1) % TM];
                if (q < TN * TM) p[q & 1] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wf[1], af[j][1], p[q & 1], 0, 0, 0, 0, 0, 0);
                if (q)
#pragma unroll
                    for (int e = 8; e < 16; e++) acc[(q - 1) / TM][(q - 1) % TM][e] += p[~q & 1][e] * s[(q - 1) % TM];
                __builtin_amdgcn_sched_barrier(0);
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
    raw* const results = (raw*)a.out + blockIdx.y * a.part;
    uint8_t* mine = lds + wave * 32 * PITCH;
    const uint32_t nw = n0 + wn * TN * 32;
    const bool whole = nw + TN * 32 <= a.n;              // rows start anywhere: 16 bytes at a time all the same
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
                if (mw + row < a.m) *(v4i_any*)((uint8_t*)results + ((mw + row) * a.ld_out + nw) * ES + at) = *(const v4i*)(mine + row * PITCH + at);
            }
        } else {
            for (uint32_t r = 0; r < 32 && mw + r < a.m; r++)
                for (uint32_t n = lane; n < TN * 32 && nw + n < a.n; n += 64)
                    results[(mw + r) * a.ld_out + nw + n] = ((const raw*)(mine + r * PITCH))[n];
        }
    }
}

// Sums the parts' results, in order
template <class T> __global__ __launch_bounds__(256) void matmul_q8_join_kernel(const float* parts, uint32_t n_parts, u64 part, u64 ld_part, typename T::raw* out, u64 ld_out, uint32_t n) {
    const uint32_t i = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= n) return;
    const float* p = parts + blockIdx.y * ld_part + i;
    v4f x = *(const v4f*)p;
    for (uint32_t k = 1; k < n_parts; k++) x += *(const v4f*)(p + k * part);
#pragma unroll
    for (uint32_t e = 0; e < 4; e++)
        if (i + e < n) out[blockIdx.y * ld_out + i + e] = from_float<T>(x[e]);
}

template <class T, bool FAST, int WN, int WM, int TN, int TM> static hipError_t launch_tiles(const GemmArgs& a, uint32_t parts, hipStream_t stream) {
    using G = Tile<WN, WM, TN, TM>;
    const auto kernel = matmul_q8_tiles_kernel<T, FAST, WN, WM, TN, TM>;
    static const hipError_t ready = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS);
    if (ready != hipSuccess) return ready;
    const uint32_t tiles = ((a.n + G::BN - 1) / G::BN) * ((a.m + G::BM - 1) / G::BM);
    kernel<<<dim3((tiles + 7) / 8 * 8, parts), G::THREADS, G::LDS, stream>>>(a);
    return hipGetLastError();
}

// How the other products are cut: rows of W and of A to a tile, parts of the sum's axis.  Tiles of 256 x 256 read least
// and run fastest once there are enough of them for the 256 compute units; below, smaller ones, of which two or three share a unit, and
// where these do not fill the card either, the sum's axis in parts of at least 4 blocks, joined by a second kernel.  Exact sums go by the same
// counts, though their largest tile has 128 rows of W: twice as many as the rule counts.
struct Cut {
    uint32_t bn, bm, parts, per;
};
static Cut cut_of(uint32_t m, uint32_t n, uint32_t k) {
    const uint32_t blocks = (k + 127) / 128;
    auto tiles = [&](uint32_t bn, uint32_t bm) { return ((n + bn - 1) / bn) * ((m + bm - 1) / bm); };
    Cut c = {128, m <= 32 ? 32u : m <= 64 ? 64u : 128u, 1, blocks};
    if (m > 128 && tiles(256, 256) >= 224) c.bn = c.bm = 256;
    const uint32_t want = c.bm == 256 ? 0 : 512, have = tiles(c.bn, c.bm);
    if (have < want) {
        const uint32_t parts = min(min((want + have - 1) / have, blocks / 4), 16u);
        if (parts > 1) {
            c.per = (blocks + parts - 1) / parts;
            c.parts = (blocks + c.per - 1) / c.per;
        }
    }
    return c;
}
static uint64_t cut_bytes(const Cut& c, uint32_t m, uint32_t n) { return c.parts > 1 ? (uint64_t)c.parts * m * ((n + 3) & ~3u) * 4 : 0; }

template <class T> static hipError_t run_tiles(const GemmArgs& a, const Cut& c, bool fast, hipStream_t stream) {
    if (c.bm == 256) return fast ? launch_tiles<T, true, 2, 4, 4, 2>(a, c.parts, stream) : launch_tiles<T, false, 2, 4, 2, 2>(a, c.parts, stream);
    if (c.bm == 128) return fast ? launch_tiles<T, true, 2, 2, 2, 2>(a, c.parts, stream) : launch_tiles<T, false, 2, 2, 2, 2>(a, c.parts, stream);
    if (c.bm == 64) return launch_tiles<T, false, 2, 2, 2, 1>(a, c.parts, stream);
    return launch_tiles<T, false, 4, 1, 1, 1>(a, c.parts, stream);
}

static int32_t check_matmul(he_ctx* ctx, const he_matmul_plan* p, const char* who) {
    if (!p) return he_fail(ctx, HE_ERR_BADARG, "%s: null plan", who);
    if (!dtype_known(p->out_dtype)) return he_fail(ctx, HE_ERR_BADARG, "%s: unknown type %d", who, p->out_dtype);
    if (p->k == 0 || p->k > (1u << 20)) return he_fail(ctx, HE_ERR_BADARG, "%s: %u columns to sum over, outside 1..2^20", who, p->k);
    if (p->m > (1u << 20) || p->n > (1u << 20)) return he_fail(ctx, HE_ERR_BADARG, "%s: more than 2^20 rows", who);
    if ((uint64_t)p->m * p->n > 1ull << 33) return he_fail(ctx, HE_ERR_BADARG, "%s: more than 2^33 results", who);
    return HE_OK;
}

extern "C" int32_t he_ws_query_matmul_q8(const he_ctx* ctx, const he_matmul_plan* p, uint64_t* h_bytes) {
    return he_guard(ctx, "he_ws_query_matmul_q8: host allocation failed", [&]() -> int32_t {
    if (!ctx || !h_bytes) return HE_ERR_BADARG;
    const int32_t rc = check_matmul(const_cast<he_ctx*>(ctx), p, "he_ws_query_matmul_q8");
    if (rc != HE_OK) return rc;
    *h_bytes = p->m && p->n && !few_rows(p->m, p->n, p->k) ? cut_bytes(cut_of(p->m, p->n, p->k), p->m, p->n) : 0;
    return HE_OK;
    });
}

extern "C" int32_t he_matmul_q8(he_ctx* ctx, const he_matmul_plan* p) {
    return he_guard(ctx, "he_matmul_q8: host allocation failed", [&]() -> int32_t {
    if (!ctx) return HE_ERR_BADARG;
    int32_t rc = check_matmul(ctx, p, "he_matmul_q8");
    if (rc != HE_OK) return rc;
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
    GemmArgs a = {p->d_a, p->d_w, p->d_a_scales, p->d_w_scales, p->d_out, p->ld_a, p->ld_w, p->ld_a_scales, p->ld_w_scales, p->ld_out, p->m, p->n, p->k, kb, 0};
    const Cut c = cut_of(p->m, p->n, p->k);
    const bool few = few_rows(p->m, p->n, p->k), parts = !few && c.parts > 1;
    if (parts) {
        if ((rc = he_ensure_ws(ctx, cut_bytes(c, p->m, p->n))) != HE_OK) return rc;
        a.ld_out = (p->n + 3) & ~3u;
        a.part = p->m * a.ld_out;
        a.out = ctx->d_ws;
        a.per = c.per;
    }
    hipError_t err = hipSuccess;
    with_dtype(p->out_dtype, [&](auto t) {
        using T = decltype(t);
        if (few) err = run_few<T>(a, ctx->stream);
        else if (!parts) err = run_tiles<T>(a, c, p->fast_sums != 0, ctx->stream);
        else if ((err = run_tiles<f32_t>(a, c, p->fast_sums != 0, ctx->stream)) == hipSuccess) {
            for (uint32_t r = 0; r < p->m; r += 65535)   // a grid's second side
                matmul_q8_join_kernel<T><<<dim3((p->n + 1023) / 1024, min(p->m - r, 65535u)), 256, 0, ctx->stream>>>(
                    (const float*)ctx->d_ws + r * a.ld_out, c.parts, a.part, a.ld_out, (typename T::raw*)p->d_out + r * p->ld_out, p->ld_out, p->n);
            err = hipGetLastError();
        }
    });
    if (err != hipSuccess) return he_fail(ctx, HE_ERR_HIP, "he_matmul_q8: %s", hipGetErrorString(err));
    return HE_OK;
    });
}
