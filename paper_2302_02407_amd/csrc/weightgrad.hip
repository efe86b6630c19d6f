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
    uint32_t parts, per;       // steps of 32 rows a part takes
    u64 part;                  // elements from one part's sums to the next's
    int32_t out_dtype;
    uint32_t accumulate;
};

template <class T> struct Parts;
template <> struct Parts<bf16_t> { static constexpr int N = 1; };
template <> struct Parts<f16_t> { static constexpr int N = 2; };
template <> struct Parts<f32_t> { static constexpr int N = 3; };

// The upper halves of two numbers of 32 bits side by side
__device__ __forceinline__ uint32_t uppers(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }
__device__ __forceinline__ uint32_t uppers(float lo, float hi) { return uppers(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)); }
// Two neighbours' bfloat16 parts, pair j of a piece: 8 significant bits each, cut off
__device__ __forceinline__ void parts_of(const Eight<f32_t>& y, int j, uint32_t (&w)[3]) {
    const uint32_t word[2] = {y.v[j / 2].w[2 * (j % 2)], y.v[j / 2].w[2 * (j % 2) + 1]};
    float mid[2], low[2];
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const float x = __builtin_bit_cast(float, word[i]);
        mid[i] = x - __builtin_bit_cast(float, word[i] & 0xffff0000u);
        if (__builtin_isinf(x)) mid[i] = 0.0f;               // nothing but itself of an infinity
        low[i] = mid[i] - __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, mid[i]) & 0xffff0000u);
    }
    w[0] = uppers(word[0], word[1]);
    w[1] = uppers(mid[0], mid[1]);
    w[2] = uppers(low[0], low[1]);
}
// Of 11 significant bits the last three are the second part, of numbers of 32 bits, in which every NaN has the highest of its bits.  Of an infinity it is that of the largest number of its
// sign, which beside an infinity is nothing.
__device__ __forceinline__ void parts_of(const Eight<f16_t>& y, int j, uint32_t (&w)[2]) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const h2 pair = __builtin_bit_cast(h2, y.v[0].w[j]);
    float x[2], low[2];
#pragma unroll
    for (int i = 0; i < 2; i++) {
        x[i] = (float)pair[i];
        const float finite = __builtin_amdgcn_fmed3f(x[i], -65504.0f, 65504.0f);
        low[i] = finite - __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, finite) & 0xffff0000u);
    }
    w[0] = uppers(x[0], x[1]);
    w[1] = uppers(low[0], low[1]);
}

// A work group owns BN columns of dy by BK columns of what is kept and goes through the rows 32 at a time.
template <class T, int WN, int WK, int TN, int TK> struct WeightTile {
    static constexpr int PARTS = Parts<T>::N, BN = WN * TN * 32, BK = WK * TK * 32, BLOCKS = BK / 128, THREADS = 64 * WN * WK;
    static constexpr int PLANE = 32 * BN * 2, X = PARTS * PLANE, S = X + 32 * BK, BYTES = S + 32 * BLOCKS * 4, LDS = 2 * BYTES;
    static constexpr int FY = 4 * BN / THREADS, FX = 2 * BK / THREADS;       // pieces of 8 elements of dy, of 16 codes, a thread
};

typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s* lds_v4s;
typedef __attribute__((address_space(3))) uint8_t* lds_ptr;

// Both operands lie in LDS as they lie in memory, a row of m after another.  dy's fragments, eight rows of a column a lane, come by reads
// that transpose: sixteen lanes name four rows of sixteen columns and each gets a column of four.  Those rows would lie in the same banks, so the
// 16-byte piece p of row r lies at p ^ 4 (r & 3).  What is kept stays codes until it is used: a lane reads four columns of each of its eight rows,
// turns each row's into bfloat16 by that row's power, and puts pairs of rows together: the fragments of four squares, in which lane l
// holds columns 4 l .. 4 l + 3, so that results are written 16 bytes a lane.  Rows r and r + 8 go to the two halves of a wavefront
// and are 128 bytes, half of the banks, apart: no conflicts (counted).
//
// Tiles of 256 x 256 by eight wavefronts of 64 x 128: 16384 x 8192 x 4096 bf16 to f32 979 us (1123 TFLOP/s; a library product of two bfloat16 matrices that lie so
// takes 1019), matrix instructions 55% of its cycles, vector instructions 42% (counted).  Steps on the way:
// read and multiplied in turn 1256, in the pipeline below 1124, loads by pointers 1095, asked for two steps ahead 1040.  Wavefronts of 128 x 64, which convert half as much,
// read codes two bytes a lane: 1190 where this took 1095, for LDS instructions.  Four wavefronts of 128 x 128 do not fit the registers.  Smaller tiles,
// 128 x 128 by four wavefronts of 64 x 64, two or three to a unit, where few large ones are there: 4096 x 2048 x 2048
// 63 us; 64 x 256 by four of 64 x 64 for up to 64 columns of dy: 22070 x 25 x 4773 f16 39 us, in tiles of 128 x 128 76 when this took 44.
template <class T, int WN, int WK, int TN, int TK, int AHEAD, bool NARROW> __global__ __launch_bounds__(64 * WN * WK, 2) void weight_grad_kernel(WeightArgs a) {
    using raw = typename T::raw;
    using G = WeightTile<T, WN, WK, TN, TK>;
    using codes_t = std::conditional_t<TK == 4, uint32_t, uint16_t>;         // a lane's columns of a row
    constexpr int PARTS = G::PARTS;
    extern __shared__ __align__(1024) uint8_t lds[];
    // a piece's place in row r, so that four rows' lie in different banks: a row is all 64 banks, or half of them
    auto turned = [](uint32_t p, uint32_t r) { return G::BN >= 128 ? p ^ 4 * (r & 3) : p ^ 4 * (r >> 1 & 1); };
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l = lane & 31, g = lane >> 5;
    const uint32_t wn = wave / WK, wk = wave % WK;
    // All tiles of a part, then those of the next: a die takes an eighth of that, and its cache holds the rows that the tiles of a part share.  (With the parts on
    // another axis of the grid and fewer tiles than dies, some dies had nothing: 65536 x 256 x 256 bf16 43 us, 28 now.)
    uint32_t n_own, k0;
    const uint32_t tiles_n = (a.n + G::BN - 1) / G::BN, tiles_k = (a.k + G::BK - 1) / G::BK, tiles = tiles_n * tiles_k, all = tiles * a.parts, each = (all + 7) / 8;
    const uint32_t item = blockIdx.x % 8 * each + blockIdx.x / 8, part = item / tiles;
    if (blockIdx.x / 8 >= each || item >= all) return;
    tile_in_order(item - part * tiles, tiles_n, tiles_k, n_own, k0);
    n_own *= G::BN;
    k0 *= G::BK;
    // the last tile begins earlier, so that all its columns are there; the rows of dw that another one has are left to that
    const uint32_t n0 = NARROW ? 0 : min(n_own, a.n - G::BN);
    const uint32_t first = part * a.per * 32, steps = min((a.m - first + 31) / 32, a.per);
    const uint32_t codes_end = (a.k + 15) / 16 * 16, blocks = (a.k + 127) / 128;

    struct Stage {
        Eight<T> y[G::FY];
        uint4 x[G::FX];
        uint32_t e;
    };
    // The last 32 rows, of which some may not be there, come first, so that it is before the loop that they are made zeros; then the others.  Past the
    // last step: one that is there again, for nothing.
    const raw* y_from[G::FY];
    const uint8_t *x_from[G::FX], *e_from;
    auto place = [&](uint32_t m0) {
#pragma unroll
        for (int f = 0; f < G::FY; f++) {
            const uint32_t i = f * G::THREADS + tid, row = min(m0 + i / (G::BN / 8), a.m - 1);
            const uint32_t at = n0 + i % (G::BN / 8) * 8;
            y_from[f] = (const raw*)a.dy + (u64)row * a.ld_dy + (!NARROW ? at : a.n >= 8 ? min(at, a.n - 8) : 0);
        }
#pragma unroll
        for (int f = 0; f < G::FX; f++) {
            const uint32_t i = f * G::THREADS + tid, row = min(m0 + i / (G::BK / 16), a.m - 1);
            x_from[f] = a.codes + (u64)row * a.ld_codes + min(k0 + i % (G::BK / 16) * 16, codes_end - 16);
        }
        const uint32_t row = min(m0 + tid % 32, a.m - 1), block = min(k0 / 128 + tid / 32 % G::BLOCKS, blocks - 1);
        e_from = a.exponents + (u64)row * a.ld_exponents + block;
    };
    auto load = [&](uint32_t step, Stage& st) {
        const u64 on = step != 0 && step + 1 < steps ? 32 : 0;       // rows to the next step's
#pragma unroll
        for (int f = 0; f < G::FY; f++) {
            if (!NARROW || a.n >= 8) st.y[f].load(y_from[f]);
            else {
                float x[8];
                load8<T>(y_from[f], 0, a.n, x);
                st.y[f].set(x);
            }
            y_from[f] += on * a.ld_dy;
        }
#pragma unroll
        for (int f = 0; f < G::FX; f++) {
            st.x[f] = *(const uint4*)x_from[f];
            x_from[f] += on * a.ld_codes;
        }
        st.e = *e_from;
        e_from += on * a.ld_exponents;
    };
    auto cut = [&](Stage& st) {                           // zeros past the last row, in both operands
        const uint32_t left = a.m - first - (steps - 1) * 32;
#pragma unroll
        for (int f = 0; f < G::FY; f++)
            if ((f * G::THREADS + tid) / (G::BN / 8) >= left)
#pragma unroll
                for (int v = 0; v < Eight<T>::VECS; v++)
#pragma unroll
                    for (int i = 0; i < 4; i++) st.y[f].v[v].w[i] = 0;
#pragma unroll
        for (int f = 0; f < G::FX; f++)
            if ((f * G::THREADS + tid) / (G::BK / 16) >= left) st.x[f] = make_uint4(0, 0, 0, 0);
        if (tid % 32 >= left) st.e = 127;
    };
    auto store = [&](uint32_t step, Stage& st) {
        uint8_t* buf = lds + (step & 1) * G::BYTES;
#pragma unroll
        for (int f = 0; f < G::FY; f++) {
            const uint32_t i = f * G::THREADS + tid, r = i / (G::BN / 8), p = i % (G::BN / 8);
            if (NARROW && a.n > 8 && a.n % 8) {           // the last piece was read from inside the row: its own elements to the front
                const uint32_t on = p * 8 + 8 > a.n ? p * 8 + 8 - a.n : 0;
                constexpr int WORDS = 4 * Eight<T>::VECS;
                uint32_t w[WORDS + 8];
#pragma unroll
                for (int j = 0; j < WORDS + 8; j++) w[j] = j < WORDS ? st.y[f].v[j / 4].w[j % 4] : 0;
#pragma unroll
                for (int by = 4; by; by /= 2) {
                    const uint32_t bits = by * sizeof(raw) * 8;
#pragma unroll
                    for (int j = 0; j < WORDS; j++) w[j] = !(on & by) ? w[j] : bits >= 32 ? w[j + bits / 32] : w[j] >> 16 | w[j + 1] << 16;
                }
#pragma unroll
                for (int j = 0; j < WORDS; j++) st.y[f].v[j / 4].w[j % 4] = w[j];
            }
            uint8_t* to = buf + r * (G::BN * 2) + turned(p, r) * 16;
            if constexpr (PARTS == 1) *(uint4*)to = make_uint4(st.y[f].v[0].w[0], st.y[f].v[0].w[1], st.y[f].v[0].w[2], st.y[f].v[0].w[3]);
            else {
                uint32_t w[PARTS][4];
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    uint32_t pair[PARTS];
                    parts_of(st.y[f], j, pair);
#pragma unroll
                    for (int q = 0; q < PARTS; q++) w[q][j] = pair[q];
                }
#pragma unroll
                for (int q = 0; q < PARTS; q++) *(uint4*)(to + q * G::PLANE) = make_uint4(w[q][0], w[q][1], w[q][2], w[q][3]);
            }
        }
#pragma unroll
        for (int f = 0; f < G::FX; f++) {
            const uint32_t i = f * G::THREADS + tid, r = i / (G::BK / 16), c = i % (G::BK / 16) * 16;
            *(uint4*)(buf + G::X + ((r * G::BK + c) ^ ((r >> 3 & 1) * 128))) = st.x[f];
        }
        ((uint32_t*)(buf + G::S))[tid % (32 * G::BLOCKS)] = st.e == 255 ? 0x7fc00000u : st.e << 23;      // several threads the same
    };

    // half h of a step: sixteen rows, eight a lane
    struct Half {
        v4s y[PARTS][TN][2];
        uint32_t x[8];
        v4f s[2];
    };
    uint32_t y_at[TN], x_at[2];
#pragma unroll
    for (int q = 0; q < TN; q++)
        y_at[q] = (8 * g + (lane & 15) / 4) * (G::BN * 2) + turned(wn * TN * 4 + 4 * q + (lane >> 4 & 1) * 2 + (lane & 3) / 2, (lane & 15) / 4) * 16 + (lane & 1) * 8;
#pragma unroll
    for (int i = 0; i < 2; i++) x_at[i] = G::X + (((8 * g + i) * G::BK + (wk * 32 + l) * TK) ^ (g * 128));
    auto read_x = [&](uint32_t step, int h, Half& f) {
        const uint32_t buf = (step & 1) * G::BYTES;
#pragma unroll
        for (int u = 0; u < 4; u++)
#pragma unroll
            for (int i = 0; i < 2; i++) f.x[2 * u + i] = *(const codes_t*)(lds + buf + x_at[i] + (16 * h + 2 * u) * G::BK);
#pragma unroll
        for (int i = 0; i < 2; i++) f.s[i] = *(const v4f*)(lds + buf + G::S + (wk * TK / 4 * 32 + 16 * h + 8 * g + 4 * i) * 4);
    };
    auto read_y = [&](uint32_t step, int h, Half& f) {
        const uint32_t buf = (step & 1) * G::BYTES;
#pragma unroll
        for (int q = PARTS - 1; q >= 0; q--)
#pragma unroll
            for (int i = 0; i < TN; i++)
#pragma unroll
                for (int t = 0; t < 2; t++)
                    f.y[q][i][t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)((lds_ptr)lds + buf + y_at[i] + (q * 32 + 16 * h + 4 * t) * (G::BN * 2)));
    };
    auto read = [&](uint32_t step, int h, Half& f) {
        read_x(step, h, f);
        read_y(step, h, f);
    };
    v16f acc[TN][TK];
#pragma unroll
    for (int i = 0; i < TN; i++)
#pragma unroll
        for (int j = 0; j < TK; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0;
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    struct Kept {
        u4 x[TK];                                         // of each square
    };
    auto convert = [&](const Half& f, Kept& to) {
        uint32_t c[8][TK / 2];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float s = f.s[i / 4][i % 4];
            c[i][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f.x[i], s, false));
            if constexpr (TK == 4) c[i][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f.x[i], s, true));
        }
#pragma unroll
        for (int j = 0; j < TK; j++)
#pragma unroll
            for (int u = 0; u < 4; u++) to.x[j][u] = __builtin_amdgcn_perm(c[2 * u + 1][j / 2], c[2 * u][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
    };
    auto multiply = [&](const Half& f, const Kept& kept) {
#pragma unroll
        for (int q = PARTS - 1; q >= 0; q--)
#pragma unroll
            for (int i = 0; i < TN; i++) {
                const v8b y = __builtin_bit_cast(v8b, __builtin_shufflevector(f.y[q][i][0], f.y[q][i][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int j = 0; j < TK; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y, __builtin_bit_cast(v8b, kept.x[j]), acc[i][j], 0, 0, 0);
            }
    };
    // What a wavefront has written to LDS is there for the others, and what it has asked for has come
    auto meet = [&]() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

    // between two matrix instructions a few of what turns the next half's codes
    auto interleave = [&]() {
#pragma unroll
        for (int i = 0; i < TN * TK; i++) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 8 / TN, 0);
        }
    };
    // rows are asked for AHEAD steps before they go to LDS: step j's (from 1 on) are in stage (j - 1) % AHEAD until then
    Stage st[AHEAD];
    {
        Stage zero;
        place(first + (steps - 1) * 32);
        load(0, zero);
        if (steps > 1) place(first);
#pragma unroll
        for (int j = 0; j < AHEAD; j++) load(j + 1, st[j]);
        cut(zero);
        store(0, zero);
    }
    meet();
    if constexpr (PARTS == 1) {
        // Three halves are on their way: one is multiplied while the next is turned into bfloat16 and the one behind that is read; so a step's
        // rows are read while the step before is multiplied, and the buffer of that takes the step after.
        Half one, two;
        Kept k_one, k_two;
        read(0, 0, one);
        read(0, 1, two);
        store(1, st[0]);
        load(AHEAD + 1, st[0]);
        convert(one, k_one);
        meet();
        for (uint32_t b0 = 0; b0 < steps; b0 += AHEAD)
#pragma unroll
            for (int d = 0; d < AHEAD; d++) {
                const uint32_t b = b0 + d;
                if (d && b >= steps) break;
                Stage& now = st[(d + 1) % AHEAD];
                Half half, next;
                read(b + 1, 0, half);
                multiply(one, k_one);
                convert(two, k_two);
                interleave();
                store(b + 2, now);
                load(b + 2 + AHEAD, now);
                read(b + 1, 1, next);
                multiply(two, k_two);
                convert(half, k_one);
                interleave();
                one = half;
                two = next;
                meet();
            }
    } else {
        // Several matrix products to a half: the next one is read and turned while they run, and the registers hold no third (60294 x 663 x 6360 f16 1030 -> 980 us, 16384
        // x 4096 x 4096 f32 1248 -> 1200, 1374 TFLOP/s of its three products; small tiles lose their third work group to a compute unit for it and still gain, 1000 x 500 x
        // 4000 f32 37 -> 33; 8192 x 200 x 8000 f16 88 -> 89)
        Half half;
        Kept kept, other;
        read(0, 0, half);
        convert(half, kept);
        for (uint32_t b0 = 0; b0 < steps; b0 += AHEAD)
#pragma unroll
            for (int d = 0; d < AHEAD; d++) {
                const uint32_t b = b0 + d;
                if (d && b >= steps) break;
                Half next;
                read(b, 1, next);
                multiply(half, kept);
                convert(next, other);
                interleave();
                store(b + 1, st[d]);                      // the other buffer: its last reads lie before the last barrier
                load(b + 1 + AHEAD, st[d]);
                meet();
                read(b + 1, 0, half);
                multiply(next, other);
                convert(half, kept);
                interleave();
            }
    }
    // element e of a square: row 8 (e / 4) + 4 g + e % 4, square j column TK l + j
    const uint32_t k = k0 + (wk * 32 + l) * TK;
    auto put = [&](auto o, u64 at, const float* x) {
        using O = decltype(o);
        typename O::raw *to = (typename O::raw*)a.dw + at, v[TK];
        if (k + TK <= a.k) {
            if (a.accumulate) __builtin_memcpy(v, to, sizeof v);
#pragma unroll
            for (int j = 0; j < TK; j++) v[j] = from_float<O>(a.accumulate ? to_float<O>(v[j]) + x[j] : x[j]);
            __builtin_memcpy(to, v, sizeof v);
        } else
#pragma unroll
            for (int j = 0; j < TK; j++)
                if (k + j < a.k) to[j] = from_float<O>(a.accumulate ? to_float<O>(to[j]) + x[j] : x[j]);
    };
#pragma unroll
    for (int i = 0; i < TN; i++)
#pragma unroll
        for (int e = 0; e < 16; e++) {
            const uint32_t n = n0 + (wn * TN + i) * 32 + 8 * (e / 4) + 4 * g + e % 4;
            float x[TK];
#pragma unroll
            for (int j = 0; j < TK; j++) x[j] = acc[i][j][e];
            const u64 at = part * a.part + n * a.ld_dw + k;
            if (n >= n_own && n < a.n && k < a.k) {
                if (a.out_dtype == HE_F32) put(f32_t{}, at, x);
                else if (a.out_dtype == HE_BF16) put(bf16_t{}, at, x);
                else put(f16_t{}, at, x);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
}

// Sums the parts, in a fixed order: four elements a thread, LANES of which take every LANES-th part of the same four.  Parts lie as dw does, their rows
// ld_part apart, a multiple of 4.
template <class O, int LANES> __global__ __launch_bounds__(256)
void weight_join_kernel(const float* parts, uint32_t n_parts, u64 part, uint32_t ld_part, typename O::raw* dw, u64 ld_dw, uint32_t k, uint32_t accumulate) {
    constexpr int GROUP = 256 / LANES;
    __shared__ v4f sums[LANES][GROUP];
    const u64 i = (((u64)blockIdx.y * gridDim.x + blockIdx.x) * GROUP + threadIdx.x % GROUP) * 4;
    const uint32_t lane = threadIdx.x / GROUP;
    v4f x = {0, 0, 0, 0};
    if (i < part)
#pragma unroll 4
        for (uint32_t q = lane; q < n_parts; q += LANES) x += *(const v4f*)(parts + q * part + i);
    if (LANES > 1) {
        sums[lane][threadIdx.x % GROUP] = x;
        __syncthreads();
        if (lane) return;
#pragma unroll
        for (int j = 1; j < LANES; j++) x += sums[j][threadIdx.x];
    }
    if (i >= part) return;
    const uint32_t row = (uint32_t)(i / ld_part), at = (uint32_t)(i - (u64)row * ld_part);
    typename O::raw *to = dw + row * ld_dw + at, v[4];
    if (at + 4 <= k) {
        if (accumulate) __builtin_memcpy(v, to, sizeof v);
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = from_float<O>(accumulate ? to_float<O>(v[e]) + x[e] : x[e]);
        __builtin_memcpy(to, v, sizeof v);
    } else
#pragma unroll
        for (uint32_t e = 0; e < 4; e++)
            if (at + e < k) to[e] = from_float<O>(accumulate ? to_float<O>(to[e]) + x[e] : x[e]);
}

template <class T, int WN, int WK, int TN, int TK, int AHEAD, bool NARROW> static hipError_t launch_weight_grad(const WeightArgs& a, const WeightCut& c, hipStream_t stream) {
    using G = WeightTile<T, WN, WK, TN, TK>;
    const auto kernel = weight_grad_kernel<T, WN, WK, TN, TK, AHEAD, NARROW>;
    const hipError_t ready = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS);
    if (ready != hipSuccess) return ready;
    const uint64_t all = (uint64_t)((a.n + G::BN - 1) / G::BN) * ((a.k + G::BK - 1) / G::BK) * a.parts;      // at most 2^20 tiles, and parts only of far fewer
    kernel<<<(uint32_t)((all + 7) / 8 * 8), G::THREADS, G::LDS, stream>>>(a);
    return hipGetLastError();
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
    const WeightCut c = weight_cut(p->m, p->n, p->k, p->dtype);
    const bool joined = p->m == 0 || c.parts > 1;
    WeightArgs a = {p->d_dy, p->d_codes, p->d_exponents, p->d_dw, p->ld_dy, p->ld_codes, p->ld_exponents, p->ld_dw, p->m, p->n, p->k, c.parts, c.per, 0, p->out_dtype, p->accumulate};
    if (joined) {
        a.dw = p->d_work;
        a.ld_dw = weight_pitch(p->k);
        a.part = p->n * a.ld_dw;
        a.out_dtype = HE_F32;
        a.accumulate = 0;
    }
    hipError_t err = hipSuccess;
    if (p->m) with_dtype(p->dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int MANY = Parts<T>::N < 3 ? 4 : 2;     // stages that the registers have room for at two work groups to a compute unit
        auto small = [&](auto wn, auto narrow) {
            constexpr int WN = decltype(wn)::value;
            constexpr bool N = decltype(narrow)::value;
            if constexpr (Parts<T>::N == 1)
                if (!c.ahead) return launch_weight_grad<T, WN, 4 / WN, 2, 2, 1, N>(a, c, ctx->stream);
            return launch_weight_grad<T, WN, 4 / WN, 2, 2, MANY, N>(a, c, ctx->stream);
        };
        const std::integral_constant<int, 1> one;
        const std::integral_constant<int, 2> two;
        if (c.side == 256) err = launch_weight_grad<T, 4, 2, 2, 4, Parts<T>::N == 1 ? 2 : 1, false>(a, c, ctx->stream);
        else if (c.side == 64) err = small(one, std::true_type{});
        else err = p->n >= 128 ? small(two, std::false_type{}) : small(two, std::true_type{});
    });
    HE_HIP(ctx, err);
    if (joined) with_dtype(p->out_dtype, [&](auto o) {
        using O = decltype(o);
        const u64 all = (u64)p->n * a.ld_dw;              // at most 2^34
        const uint32_t parts = p->m ? c.parts : 0;
        auto go = [&](auto lanes) {
            constexpr int LANES = decltype(lanes)::value;
            const u64 groups = (all + 1024 / LANES - 1) / (1024 / LANES), side = groups < HE_GROUPS_MAX ? groups : HE_GROUPS_MAX;
            weight_join_kernel<O, LANES><<<dim3((uint32_t)side, (uint32_t)((groups + side - 1) / side)), 256, 0, ctx->stream>>>(
                (const float*)p->d_work, parts, all, (uint32_t)a.ld_dw, (typename O::raw*)p->d_dw, p->ld_dw, p->k, p->accumulate);
        };
        if (parts > 8) go(std::integral_constant<int, 8>{});
        else go(std::integral_constant<int, 1>{});
    });
    HE_LAUNCHED(ctx);
    return HE_OK;
    });
}
