// Plans of the plaintext operators: what is refused, and how the work is cut where scratch memory depends on it.  Host code that needs no GPU and
// no HIP header.  A check returns why a plan is refused, or a null pointer.
#ifndef HE_CHECKS_H
#define HE_CHECKS_H

#include <stdint.h>

#include "../../include/he_mi355x.h"

#define HE_ROWS_MAX (1u << 21)     // a work group of at most 1024 threads a row: a launch's threads stay below 2^32
#define HE_VOCAB_MAX (1u << 20)
#define HE_DIM_MAX 65536u
#define HE_BLOCK 128u              // columns that share a power or a scale

static inline uint32_t dtype_bytes(int32_t dtype) { return dtype == HE_F32 ? 4 : 2; }
static inline bool dtype_known(int32_t dtype) { return dtype == HE_F32 || dtype == HE_BF16 || dtype == HE_F16; }
// Whether [a, a + na) and [b, b + nb) share a byte
static inline bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
    return a && b && na && nb && (const char*)a < (const char*)b + nb && (const char*)b < (const char*)a + na;
}
// Bytes from the first to past the last element of `rows` rows of `cols` elements, `ld` elements apart
static inline uint64_t span(uint64_t rows, uint64_t cols, uint64_t ld, uint64_t size) { return rows && cols ? ((rows - 1) * ld + cols) * size : 0; }
// Rows of `cols` elements, ld apart: they do not overlap, and no offset of HE_ROWS_MAX of them leaves 64 bits
static inline bool ld_fits(uint64_t ld, uint64_t cols) { return ld >= cols && ld <= (1u << 28); }
// Temperatures of which log2(e) / tau and tau^2 are numbers, and at which a masked logit, from 2^126 on, is far from any other
static inline bool tau_fits(float tau) { return tau >= 0x1p-60f && tau <= 0x1p60f; }

// Memory that a call reads or writes.  same: an input that the output may lie on exactly, with the same ld
struct Span {
    const void* d;
    uint64_t bytes, ld;
};
static inline Span rows_of(const void* d, uint64_t rows, uint64_t cols, uint64_t ld, uint64_t size) { return Span{d, d ? span(rows, cols, ld, size) : 0, ld}; }
static inline Span vector_of(const void* d, uint64_t n, uint64_t size) { return Span{d, d ? n * size : 0, 0}; }
// Outputs against inputs and each other; bit i of same[o]: output o may be input i
template <int I, int O> static inline const char* apart(const Span (&in)[I], const Span (&out)[O], const uint32_t (&same)[O]) {
    for (int o = 0; o < O; o++) {
        for (int i = 0; i < I; i++)
            if (!(same[o] >> i & 1 && in[i].d == out[o].d && in[i].ld == out[o].ld) && overlap(out[o].d, out[o].bytes, in[i].d, in[i].bytes)) return "an output overlaps an input";
        for (int i = 0; i < o; i++)
            if (overlap(out[o].d, out[o].bytes, out[i].d, out[i].bytes)) return "two outputs overlap";
    }
    return nullptr;
}
static inline bool off(const void* d, uint64_t size) { return ((uintptr_t)d & (size - 1)) != 0; }

// ---- layer norm

static inline const char* layernorm_sizes(uint32_t rows, uint32_t dim, int32_t dtype, int32_t param_dtype) {
    if (!dtype_known(dtype)) return "unknown type";
    if (param_dtype != dtype && param_dtype != HE_F32) return "parameters are of the rows' type or of 32 bits";
    if (dim == 0 || dim > HE_DIM_MAX) return "columns outside 1..65536";
    if (rows > HE_ROWS_MAX) return "more than 2^21 rows";
    return nullptr;
}
static inline const char* refuse_layernorm(const he_layernorm_plan* p) {
    if (!p) return "null plan";
    if (const char* w = layernorm_sizes(p->rows, p->dim, p->dtype, p->param_dtype)) return w;
    if (!(p->eps >= 0.0f && p->eps <= 0x1p120f)) return "eps is not a number from 0 to 2^120";
    if (p->rows == 0) return nullptr;
    if (!p->d_x || !p->d_y) return "null argument";
    if (!p->d_residual != !p->d_sum) return "a residual and its sum come together";
    const bool res = p->d_residual != nullptr;
    if (!ld_fits(p->ld_x, p->dim) || !ld_fits(p->ld_y, p->dim) || (res && !(ld_fits(p->ld_residual, p->dim) && ld_fits(p->ld_sum, p->dim))))
        return "an ld is below the row's length or above 2^28";
    const uint32_t es = dtype_bytes(p->dtype), ps = dtype_bytes(p->param_dtype);
    if (off(p->d_x, es) || off(p->d_residual, es) || off(p->d_sum, es) || off(p->d_y, es) || off(p->d_weight, ps) || off(p->d_bias, ps) || off(p->d_stats, 4))
        return "a pointer is not aligned to its elements";
    const Span in[] = {rows_of(p->d_x, p->rows, p->dim, p->ld_x, es), rows_of(p->d_residual, p->rows, p->dim, p->ld_residual, es), vector_of(p->d_weight, p->dim, ps),
                       vector_of(p->d_bias, p->dim, ps)};
    const Span out[] = {rows_of(p->d_sum, p->rows, p->dim, p->ld_sum, es), rows_of(p->d_y, p->rows, p->dim, p->ld_y, es), vector_of(p->d_stats, 4ull * p->rows, 4)};
    return apart(in, out, {3, 3, 0});
}

// Rows whose gradient, and the sums over them, one kernel takes: at least a piece of 8 elements, at most what 512 threads keep in registers
static inline bool layernorm_one_pass(uint32_t dim) { return dim >= 8 && dim <= 16384; }
// Parts of the rows, each a work group's with a sum of its own for every column.  More of them keep more rows on the way, and have more to join: 16384 x 4096 bf16 takes
// 124 us with 256, 103 with 512 and 114 with 1024; 4096 x 16384 81, 96 and 130; 60000 x 100 f32 56, 34 and 28.
static inline uint32_t layernorm_parts(uint32_t rows, uint32_t dim) {
    if (!layernorm_one_pass(dim)) return rows < 256 ? rows : 256;
    const uint32_t slots = dim <= 256 ? 16 : dim <= 1024 ? 4 : 1, groups = (rows + slots - 1) / slots, most = dim <= 512 ? 1024 : dim <= 4096 ? 512 : 256;
    return groups < most ? groups : most;
}
static inline uint32_t layernorm_pitch(uint32_t dim) { return (dim + 7) & ~7u; }
static inline uint64_t layernorm_grad_work(const he_layernorm_grad_plan* p) {
    return p->rows && (p->d_dweight || p->d_dbias) ? 8ull * layernorm_pitch(p->dim) * layernorm_parts(p->rows, p->dim) : 0;
}
static inline const char* refuse_layernorm_grad(const he_layernorm_grad_plan* p, bool query = false) {
    if (!p) return "null plan";
    if (const char* w = layernorm_sizes(p->rows, p->dim, p->dtype, p->param_dtype)) return w;
    if (query) return nullptr;
    const uint32_t es = dtype_bytes(p->dtype), ps = dtype_bytes(p->param_dtype);
    if (off(p->d_dweight, ps) || off(p->d_dbias, ps)) return "a pointer is not aligned to its elements";
    if (p->rows == 0) return overlap(p->d_dweight, (uint64_t)p->dim * ps, p->d_dbias, (uint64_t)p->dim * ps) ? "two outputs overlap" : nullptr;
    if (!p->d_h || !p->d_stats || !p->d_dy || !p->d_dx) return "null argument";
    if (!ld_fits(p->ld_h, p->dim) || !ld_fits(p->ld_dy, p->dim) || !ld_fits(p->ld_dx, p->dim) || (p->d_dsum && !ld_fits(p->ld_dsum, p->dim)))
        return "an ld is below the row's length or above 2^28";
    if (off(p->d_h, es) || off(p->d_dy, es) || off(p->d_dsum, es) || off(p->d_dx, es) || off(p->d_weight, ps) || off(p->d_stats, 4))
        return "a pointer is not aligned to its elements";
    const uint64_t work = layernorm_grad_work(p);
    if (work && (!p->d_work || p->work_bytes < work || off(p->d_work, 16))) return "the scratch memory is too small, or not aligned to 16 bytes";
    const Span in[] = {rows_of(p->d_h, p->rows, p->dim, p->ld_h, es), rows_of(p->d_dy, p->rows, p->dim, p->ld_dy, es), rows_of(p->d_dsum, p->rows, p->dim, p->ld_dsum, es),
                       vector_of(p->d_weight, p->dim, ps), vector_of(p->d_stats, 4ull * p->rows, 4)};
    const Span out[] = {rows_of(p->d_dx, p->rows, p->dim, p->ld_dx, es), vector_of(p->d_dweight, p->dim, ps), vector_of(p->d_dbias, p->dim, ps), vector_of(work ? p->d_work : nullptr, work, 1)};
    return apart(in, out, {6, 0, 0, 0});
}

// ---- the activation that keeps its input in 8 bits

static inline const char* poly_sizes(uint32_t rows, uint32_t dim, int32_t dtype) {
    if (!dtype_known(dtype)) return "unknown type";
    if (dim == 0 || dim > HE_DIM_MAX) return "columns outside 1..65536";
    if (rows > HE_ROWS_MAX) return "more than 2^21 rows";
    return nullptr;
}
static inline uint32_t blocks_of(uint32_t dim) { return (dim + HE_BLOCK - 1) / HE_BLOCK; }
static inline uint64_t to16(uint64_t n) { return (n + 15) & ~15ull; }
static inline const char* refuse_poly(const he_poly_plan* p) {
    if (!p) return "null plan";
    if (const char* w = poly_sizes(p->rows, p->dim, p->dtype)) return w;
    if (p->n_coefs > HE_POLY_MAX) return "more than 9 coefficients";
    if (p->rows == 0) return nullptr;
    if ((p->n_coefs == 0) != !p->d_y || (p->n_coefs == 0) != !p->d_coefs) return "coefficients and an output come together";
    if (!p->d_u || !p->d_codes || !p->d_exponents) return "null argument";
    if (!ld_fits(p->ld_u, p->dim) || !ld_fits(p->ld_codes, p->dim) || !ld_fits(p->ld_exponents, blocks_of(p->dim)) || (p->d_y && !ld_fits(p->ld_y, p->dim)))
        return "an ld is below the row's length or above 2^28";
    if (off(p->d_codes, 16) || p->ld_codes & 15) return "rows of codes start at multiples of 16 bytes";
    const uint32_t es = dtype_bytes(p->dtype);
    if (off(p->d_u, es) || off(p->d_y, es) || off(p->d_coefs, 4)) return "a pointer is not aligned to its elements";
    const Span in[] = {rows_of(p->d_u, p->rows, p->dim, p->ld_u, es), vector_of(p->d_coefs, p->n_coefs, 4)};
    const Span out[] = {rows_of(p->d_y, p->rows, p->dim, p->ld_y, es), rows_of(p->d_codes, p->rows, p->dim, p->ld_codes, 1),
                        rows_of(p->d_exponents, p->rows, blocks_of(p->dim), p->ld_exponents, 1)};
    return apart(in, out, {1, 0, 0});
}

// Work groups of 256 threads, 16 to a block of 128 columns.  What sums nothing has one for every sixteen blocks (16384 x 8192 bf16, degree 3: 112 us; 2048 that go on: 142).  Sums
// want few, as many as are there at a time: the gradients of that take 127 us with 1024, 129 with 2048 and 177 with 512; of 777 x 10007 f16, degree 7, 19, 24 and 20.
#define HE_POLY_GROUPS 1024u
#define HE_GROUPS_MAX (1u << 23)   // of 256 threads: 2^31, a launch's must stay below 2^32
static inline uint32_t poly_groups(uint32_t rows, uint32_t dim, uint32_t most) {
    const uint64_t groups = ((uint64_t)rows * blocks_of(dim) + 15) / 16;
    return groups < most ? (uint32_t)groups : most;
}
static inline uint64_t poly_grad_work(const he_poly_grad_plan* p) { return p->rows && p->d_dcoefs ? 8ull * p->n_coefs * poly_groups(p->rows, p->dim, HE_POLY_GROUPS) : 0; }
static inline const char* refuse_poly_grad(const he_poly_grad_plan* p, bool query = false) {
    if (!p) return "null plan";
    if (const char* w = poly_sizes(p->rows, p->dim, p->dtype)) return w;
    if (p->n_coefs == 0 || p->n_coefs > HE_POLY_MAX) return "1 to 9 coefficients";
    if (query) return nullptr;
    if (off(p->d_dcoefs, 4)) return "a pointer is not aligned to its elements";
    if (p->rows == 0) return nullptr;
    if (!p->d_codes || !p->d_exponents || !p->d_coefs || !p->d_dy || !p->d_du) return "null argument";
    if (!ld_fits(p->ld_codes, p->dim) || !ld_fits(p->ld_exponents, blocks_of(p->dim)) || !ld_fits(p->ld_dy, p->dim) || !ld_fits(p->ld_du, p->dim))
        return "an ld is below the row's length or above 2^28";
    if (off(p->d_codes, 16) || p->ld_codes & 15) return "rows of codes start at multiples of 16 bytes";
    const uint32_t es = dtype_bytes(p->dtype);
    if (off(p->d_dy, es) || off(p->d_du, es) || off(p->d_coefs, 4)) return "a pointer is not aligned to its elements";
    const uint64_t work = poly_grad_work(p);
    if (work && (!p->d_work || p->work_bytes < work || off(p->d_work, 16))) return "the scratch memory is too small, or not aligned to 16 bytes";
    const Span in[] = {rows_of(p->d_dy, p->rows, p->dim, p->ld_dy, es), rows_of(p->d_codes, p->rows, to16(p->dim), p->ld_codes, 1),
                       rows_of(p->d_exponents, p->rows, blocks_of(p->dim), p->ld_exponents, 1), vector_of(p->d_coefs, p->n_coefs, 4)};
    const Span out[] = {rows_of(p->d_du, p->rows, p->dim, p->ld_du, es), vector_of(p->d_dcoefs, p->n_coefs, 4), vector_of(work ? p->d_work : nullptr, work, 1)};
    return apart(in, out, {1, 0, 0});
}

// ---- a weight's gradient from an input kept in 8 bits

#define HE_SIDE_MAX (1u << 17)
#define HE_WORK_MAX (1ull << 30)   // bytes of a weight gradient's scratch memory

// Tiles of `side` rows by as many columns of dw, or of 64 by 256, the sum over the rows of dy in `parts` parts of `per` steps of 32 rows, joined by a second kernel
struct WeightCut {
    uint32_t side, parts, per;
    bool ahead;                // small tiles of bf16, at most two to a compute unit: rows are asked for four steps ahead, for which three have no registers (65536 x 256 x 256: 28 us, 30)
};
static inline uint64_t weight_pitch(uint32_t k) { return (k + 3) & ~3u; }
// The cut that costs least, by what was measured of steps and joins (bf16; in fifths of a step of a compute unit's three small tiles, 0.19 us): a step of a
// unit takes 5.5 with a tile of 256 x 256, and 3, 4, 5 with one, two, three of 128 x 128; a step of f16 1.4 times that and one of f32 2 times, their matrix
// products being two and three (between 1.2 and 1.6, and 1.6 and 2.3, cuts or times of few shapes change).  The second launch takes 16 and a part 8 bytes an
// element at 4.5 TB/s.  Measured against the best of five rules of thumb on eleven shapes from 500 x 100 x 100 to 65536 x 256 x 256; shapes between go by the same line.
// No more parts than HE_WORK_MAX has room for, which binds only from some 10^12 products on.
static inline WeightCut weight_cut(uint32_t m, uint32_t n, uint32_t k, int32_t dtype) {
    const uint64_t steps = (m + 31) / 32, kind = dtype == HE_BF16 ? 10 : dtype == HE_F16 ? 14 : 20;
    WeightCut best = {128, 1, (uint32_t)steps, false};
    if (steps == 0) return best;
    uint64_t least = ~0ull;
    for (uint32_t side = n > 64 ? 128 : 64; side <= 256; side *= 2) {
        if (side == 256 ? n < 256 : side == 128 && n <= 64) break;
        const uint64_t wide = side == 64 ? 256 : side, tiles = ((n + side - 1) / side) * ((k + wide - 1) / wide);
        static const uint32_t wants[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128};
        for (const uint32_t want : wants) {
            if (want > 1 && steps < 4 * want) break;
            const uint64_t per = (steps + want - 1) / want, parts = (steps + per - 1) / per, each = (tiles * parts + 255) / 256;
            if (parts > 1 && parts * n * weight_pitch(k) * 4 > HE_WORK_MAX) break;
            const uint64_t step = side == 256 ? 11 * each : 2 * (each / 3 * 5 + (each % 3 ? each % 3 + 2 : 0));
            const uint64_t cost = per * step * kind + (parts > 1 ? 320 + parts * n * k / 5350 : 0);          // in twentieths
            if (cost < least) least = cost, best = {side, (uint32_t)parts, (uint32_t)per, each <= 2};
        }
    }
    return best;
}
static inline uint64_t weight_grad_work(const he_weight_grad_plan* p) {
    if (!p->m || !p->n || !p->k) return 0;
    const WeightCut c = weight_cut(p->m, p->n, p->k, p->dtype);
    return c.parts > 1 ? c.parts * p->n * weight_pitch(p->k) * 4 : 0;
}
static inline const char* refuse_weight_grad(const he_weight_grad_plan* p, bool query = false) {
    if (!p) return "null plan";
    if (!dtype_known(p->dtype) || !dtype_known(p->out_dtype)) return "unknown type";
    if (p->m > HE_ROWS_MAX) return "more than 2^21 rows to sum over";
    if (p->n > HE_SIDE_MAX || p->k > HE_SIDE_MAX) return "more than 2^17 rows or columns of the gradient";
    if (query || p->n == 0 || p->k == 0) return nullptr;
    const uint32_t es = dtype_bytes(p->dtype), os = dtype_bytes(p->out_dtype);
    if (!p->d_dw || (p->m && (!p->d_dy || !p->d_codes || !p->d_exponents))) return "null argument";
    if (!ld_fits(p->ld_dw, p->k) || (p->m && (!ld_fits(p->ld_dy, p->n) || !ld_fits(p->ld_codes, p->k) || !ld_fits(p->ld_exponents, blocks_of(p->k)))))
        return "an ld is below the row's length or above 2^28";
    if (off(p->d_dw, os)) return "a pointer is not aligned to its elements";
    if (p->m == 0) return nullptr;
    if (off(p->d_codes, 16) || p->ld_codes & 15) return "rows of codes start at multiples of 16 bytes";
    if (off(p->d_dy, es)) return "a pointer is not aligned to its elements";
    const uint64_t work = weight_grad_work(p);
    if (work && (!p->d_work || p->work_bytes < work || off(p->d_work, 16))) return "the scratch memory is too small, or not aligned to 16 bytes";
    const Span in[] = {rows_of(p->d_dy, p->m, p->n, p->ld_dy, es), rows_of(p->d_codes, p->m, to16(p->k), p->ld_codes, 1), rows_of(p->d_exponents, p->m, blocks_of(p->k), p->ld_exponents, 1)};
    const Span out[] = {rows_of(p->d_dw, p->n, p->k, p->ld_dw, os), vector_of(work ? p->d_work : nullptr, work, 1)};
    return apart(in, out, {0, 0});
}

// ---- log probabilities of given tokens

static inline const char* logits_sizes(uint32_t rows, uint32_t vocab, int32_t dtype, float tau) {
    if (!dtype_known(dtype)) return "unknown type";
    if (vocab == 0 || vocab > HE_VOCAB_MAX) return "logits outside 1..2^20";
    if (!tau_fits(tau)) return "the temperature is not a number from 2^-60 to 2^60";
    if (rows > HE_ROWS_MAX) return "more than 2^21 rows";
    return nullptr;
}
// A row's parts, each a work group's, and the elements of one
struct LogprobCut {
    uint32_t parts, len;
};
#define HE_JOIN_PARTS 32               // at most so many parts: lanes and room of the kernel that joins them
// Few long rows are cut in up to 32 parts of at least 8 KiB, which are joined by a second launch (128 x 131072 bf16, k = 8, in four parts 17.8 us,
// whole 20.1; 1 x 131072, k = 20, in 32 parts 11.3)
// Every part, the last too, has to have at least HE_TOP_MAX elements, the first k of which are put in order, and more than 4 KiB, what a launch of single wavefronts, which knows no
// parts, takes.
static inline LogprobCut logprobs_cut(uint32_t rows, uint32_t vocab, int32_t dtype) {
    const uint32_t piece = 8192 / dtype_bytes(dtype);
    uint32_t parts = rows ? 512 / rows : 1;
    if (parts > vocab / piece) parts = vocab / piece;
    if (parts > HE_JOIN_PARTS) parts = HE_JOIN_PARTS;
    if (parts < 4) return {1, vocab};
    const uint32_t len = ((vocab + parts - 1) / parts + 15) & ~15u;
    return {(vocab + len - 1) / len, len};
}
static inline uint64_t logprobs_work(const he_logprobs_plan* p) {
    const uint32_t parts = logprobs_cut(p->rows, p->vocab, p->dtype).parts;
    return parts > 1 ? (uint64_t)p->rows * parts * (16 + 8ull * p->k) : 0;
}
static inline const char* refuse_logprobs(const he_logprobs_plan* p, bool query = false) {
    if (!p) return "null plan";
    if (const char* w = logits_sizes(p->rows, p->vocab, p->dtype, p->tau)) return w;
    if (p->k > HE_TOP_MAX || p->k > p->vocab) return "more alternatives than min(vocab, 128)";
    if (query || p->rows == 0) return nullptr;
    if (!p->d_z) return "null argument";
    if (!p->d_tokens != !p->d_logp) return "tokens and their log probabilities come together";
    if ((p->k == 0) != !p->d_values || (p->k == 0) != !p->d_index) return "alternatives have values and indices";
    if (!p->d_logp && !p->d_entropy && !p->d_values && !p->d_stats) return "nothing is asked for";
    if (!ld_fits(p->ld_z, p->vocab)) return "ld_z is below the row's length or above 2^28";
    const uint32_t es = dtype_bytes(p->dtype);
    if (off(p->d_z, es) || off(p->d_tokens, 4) || off(p->d_logp, 4) || off(p->d_entropy, 4) || off(p->d_values, 4) || off(p->d_index, 4) || off(p->d_stats, 4))
        return "a pointer is not aligned to its elements";
    const uint64_t work = logprobs_work(p);
    if (work && (!p->d_work || p->work_bytes < work || off(p->d_work, 16))) return "the scratch memory is too small, or not aligned to 16 bytes";
    const uint64_t rows = p->rows;
    const Span in[] = {rows_of(p->d_z, rows, p->vocab, p->ld_z, es), vector_of(p->d_tokens, rows, 4)};
    const Span out[] = {vector_of(p->d_logp, rows, 4), vector_of(p->d_entropy, rows, 4), vector_of(p->d_values, rows * p->k, 4), vector_of(p->d_index, rows * p->k, 4),
                        vector_of(p->d_stats, 4 * rows, 4), vector_of(work ? p->d_work : nullptr, work, 1)};
    return apart(in, out, {0, 0, 0, 0, 0, 0});
}
static inline const char* refuse_logprobs_grad(const he_logprobs_grad_plan* p) {
    if (!p) return "null plan";
    if (const char* w = logits_sizes(p->rows, p->vocab, p->dtype, p->tau)) return w;
    if (p->rows == 0) return nullptr;
    if (!p->d_z || !p->d_stats || !p->d_grad) return "null argument";
    if (p->d_logp_weights && !p->d_tokens) return "log probabilities need their tokens";
    if (!ld_fits(p->ld_z, p->vocab) || !ld_fits(p->ld_grad, p->vocab)) return "an ld is below the row's length or above 2^28";
    const uint32_t es = dtype_bytes(p->dtype);
    if (off(p->d_z, es) || off(p->d_grad, es) || off(p->d_tokens, 4) || off(p->d_stats, 4) || off(p->d_logp_weights, 4) || off(p->d_entropy_weights, 4))
        return "a pointer is not aligned to its elements";
    const uint64_t rows = p->rows;
    const Span in[] = {rows_of(p->d_z, rows, p->vocab, p->ld_z, es), vector_of(p->d_tokens, rows, 4), vector_of(p->d_stats, 4 * rows, 4), vector_of(p->d_logp_weights, rows, 4),
                       vector_of(p->d_entropy_weights, rows, 4)};
    const Span out[] = {rows_of(p->d_grad, rows, p->vocab, p->ld_grad, es)};
    return apart(in, out, {1});
}

#endif
