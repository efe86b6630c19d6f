"""CPU: what the operators of a training step refuse, and the scratch memory they ask for, from the header that their calls go by, compiled for the host."""
import os
import struct
import subprocess

import pytest

from paper_2302_02407_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
FIELDS = {
    "he_layernorm_plan": (B._LAYERNORM, "rows dim dtype param_dtype eps d_x ld_x d_residual ld_residual d_weight d_bias d_sum ld_sum d_y ld_y d_stats"),
    "he_layernorm_grad_plan": (B._LAYERNORM_GRAD, "rows dim dtype param_dtype d_h ld_h d_stats d_dy ld_dy d_weight d_dsum ld_dsum d_dx ld_dx d_dweight d_dbias d_work work_bytes"),
    "he_poly_plan": (B._POLY, "rows dim n_coefs dtype d_u ld_u d_coefs d_y ld_y d_codes ld_codes d_exponents ld_exponents"),
    "he_poly_grad_plan": (B._POLY_GRAD, "rows dim n_coefs dtype d_codes ld_codes d_exponents ld_exponents d_coefs d_dy ld_dy d_du ld_du d_dcoefs d_work work_bytes"),
    "he_weight_grad_plan": (B._WEIGHT_GRAD, "m n k dtype out_dtype accumulate d_dy ld_dy d_codes ld_codes d_exponents ld_exponents d_dw ld_dw d_work work_bytes"),
    "he_logprobs_plan": (B._LOGPROBS, "rows vocab k dtype tau d_z ld_z d_tokens d_logp d_entropy d_values d_index d_stats d_work work_bytes"),
    "he_logprobs_grad_plan": (B._LOGPROBS_GRAD, "rows vocab dtype tau d_z ld_z d_tokens d_stats d_logp_weights d_entropy_weights d_grad ld_grad"),
}


def offsets(fmt):
    at, out = "@", []
    for c in fmt.format.lstrip("@"):
        at += c
        out.append(struct.calcsize(at) - struct.calcsize("@" + c))
    return out


@pytest.mark.parametrize("name", sorted(FIELDS))
def test_plan_layout(name, tmp_path):
    fmt, fields = FIELDS[name]
    lines = "".join('    printf("%%zu\\n", offsetof(%s, %s));\n' % (name, f) for f in fields.split())
    src, exe = tmp_path / "plan.c", tmp_path / "plan"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "he_mi355x.h"\nint main(void) {\n%s    printf("%%zu\\n", sizeof(%s));\n    return 0;\n}\n' % (lines, name))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True, timeout=60)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True, timeout=60).stdout.split()]
    assert got[:-1] == offsets(fmt)
    assert struct.calcsize(fmt.format) <= got[-1] < struct.calcsize(fmt.format) + 8


PROGRAM = r'''
#include <math.h>
#include <stdio.h>
#include <string.h>
#include "checks.h"

static int bad = 0;
// Addresses only: nothing behind them is touched
static void* at(uint64_t a) { return (void*)(uintptr_t)a; }
template <class P> static void fine(const char* what, const P&, const char* why) { if (why) { bad++; printf("%s refused: %s\n", what, why); } }
template <class P> static void refused(const char* what, const P&, const char* why) { if (!why) { bad++; printf("%s taken\n", what); } }
#define MUST(check, plan, change) do { auto p = plan; change; refused(#check ": " #change, p, check(&p)); } while (0)
#define MAY(check, plan, change) do { auto p = plan; change; fine(#check ": " #change, p, check(&p)); } while (0)
static const char* grad_of(const he_layernorm_grad_plan* p) { return refuse_layernorm_grad(p); }
static const char* poly_grad_of(const he_poly_grad_plan* p) { return refuse_poly_grad(p); }
static const char* weight_of(const he_weight_grad_plan* p) { return refuse_weight_grad(p); }
static const char* logprobs_of(const he_logprobs_plan* p) { return refuse_logprobs(p); }

int main() {
    const uint64_t G = 1ull << 40;                   // far apart
    he_layernorm_plan ln = {10, 100, HE_BF16, HE_F32, 1e-5f, at(G), 100, at(2 * G), 100, at(3 * G), at(4 * G), at(5 * G), 100, at(6 * G), 100, (float*)at(7 * G)};
    MAY(refuse_layernorm, ln, (void)p);
    MAY(refuse_layernorm, ln, p.d_sum = (void*)p.d_x);
    MAY(refuse_layernorm, ln, p.d_y = (void*)p.d_residual);
    MAY(refuse_layernorm, ln, p.d_weight = p.d_bias = p.d_stats = nullptr);
    MAY(refuse_layernorm, ln, (p.d_residual = nullptr, p.d_sum = nullptr));
    MAY(refuse_layernorm, ln, p.dim = 65536; p.ld_x = p.ld_y = p.ld_sum = p.ld_residual = 1 << 28);
    MAY(refuse_layernorm, ln, p = he_layernorm_plan(); p.dim = 1);
    MUST(refuse_layernorm, ln, p.dim = 0);
    MUST(refuse_layernorm, ln, p.dim = 65537);
    MUST(refuse_layernorm, ln, p.rows = (1 << 21) + 1);
    MUST(refuse_layernorm, ln, p.dtype = 3);
    MUST(refuse_layernorm, ln, p.dtype = -1);
    MUST(refuse_layernorm, ln, p.param_dtype = HE_F16);
    MUST(refuse_layernorm, ln, p.eps = -1e-9f);
    MUST(refuse_layernorm, ln, p.eps = NAN);
    MUST(refuse_layernorm, ln, p.eps = INFINITY);
    MUST(refuse_layernorm, ln, p.d_x = nullptr);
    MUST(refuse_layernorm, ln, p.d_y = nullptr);
    MUST(refuse_layernorm, ln, p.d_sum = nullptr);
    MUST(refuse_layernorm, ln, p.d_residual = nullptr);
    MUST(refuse_layernorm, ln, p.ld_x = 99);
    MUST(refuse_layernorm, ln, p.ld_sum = 99);
    MUST(refuse_layernorm, ln, p.ld_y = (1 << 28) + 1);
    MUST(refuse_layernorm, ln, p.d_x = at(G + 1));
    MUST(refuse_layernorm, ln, p.d_weight = at(3 * G + 2));
    MUST(refuse_layernorm, ln, p.d_stats = (float*)at(7 * G + 2));
    MUST(refuse_layernorm, ln, p.d_y = p.d_sum);
    MUST(refuse_layernorm, ln, p.d_y = (void*)p.d_x; p.ld_y = 101);
    MUST(refuse_layernorm, ln, p.d_y = at(G + 200));
    MUST(refuse_layernorm, ln, p.d_stats = (float*)p.d_y);
    MUST(refuse_layernorm, ln, p.d_y = (void*)p.d_bias);
    refused("no plan", 0, refuse_layernorm(nullptr));

    he_layernorm_grad_plan lg = {10, 100, HE_F16, HE_F16, at(G), 100, (float*)at(2 * G), at(3 * G), 100, at(4 * G), at(5 * G), 100, at(6 * G), 100, at(7 * G), at(8 * G), at(9 * G), 1 << 20};
    MAY(grad_of, lg, (void)p);
    MAY(grad_of, lg, p.d_dx = (void*)p.d_dy);
    MAY(grad_of, lg, p.d_dx = (void*)p.d_dsum);
    MAY(grad_of, lg, p.work_bytes = layernorm_grad_work(&p));
    MAY(grad_of, lg, p.d_dweight = p.d_dbias = p.d_work = nullptr; p.work_bytes = 0);
    MAY(grad_of, lg, p.rows = 0; p.d_h = p.d_dy = nullptr; p.d_dx = nullptr);
    MUST(grad_of, lg, p.work_bytes = layernorm_grad_work(&p) - 1);
    MUST(grad_of, lg, p.d_work = nullptr);
    MUST(grad_of, lg, p.d_work = at(9 * G + 8));
    MUST(grad_of, lg, p.d_work = (void*)p.d_h);
    MUST(grad_of, lg, p.d_work = p.d_dbias);
    MUST(grad_of, lg, p.d_dx = (void*)p.d_h);
    MUST(grad_of, lg, p.d_dx = (void*)p.d_dy; p.ld_dx = 104);
    MUST(grad_of, lg, p.d_dbias = p.d_dweight);
    MUST(grad_of, lg, p.rows = 0; p.d_dbias = p.d_dweight);
    MUST(grad_of, lg, p.d_dweight = at(7 * G + 1));
    MUST(grad_of, lg, p.d_stats = nullptr);
    MUST(grad_of, lg, p.ld_dsum = 1);

    he_poly_plan po = {10, 100, 4, HE_BF16, at(G), 100, (float*)at(2 * G), at(3 * G), 100, (uint8_t*)at(4 * G), 112, (uint8_t*)at(5 * G), 1};
    MAY(refuse_poly, po, (void)p);
    MAY(refuse_poly, po, p.n_coefs = 0; p.d_coefs = nullptr; p.d_y = nullptr);
    MAY(refuse_poly, po, p.d_y = (void*)p.d_u);
    MAY(refuse_poly, po, p.rows = 0; p.d_y = nullptr);
    MUST(refuse_poly, po, p.n_coefs = 10);
    MUST(refuse_poly, po, p.n_coefs = 0);
    MUST(refuse_poly, po, p.d_y = nullptr);
    MUST(refuse_poly, po, p.d_coefs = nullptr);
    MUST(refuse_poly, po, p.d_codes = (uint8_t*)at(4 * G + 8));
    MUST(refuse_poly, po, p.ld_codes = 104);
    MUST(refuse_poly, po, p.ld_exponents = 0);
    MUST(refuse_poly, po, p.dim = 129; p.ld_u = p.ld_y = p.ld_codes = 144);
    MUST(refuse_poly, po, p.d_codes = (uint8_t*)p.d_u);
    MUST(refuse_poly, po, p.d_exponents = p.d_codes);
    MUST(refuse_poly, po, p.d_y = at(G + 2));

    he_poly_grad_plan pg = {10, 100, 4, HE_BF16, (uint8_t*)at(G), 112, (uint8_t*)at(2 * G), 1, (float*)at(3 * G), at(4 * G), 100, at(5 * G), 100, (float*)at(6 * G), at(7 * G), 1 << 20};
    MAY(poly_grad_of, pg, (void)p);
    MAY(poly_grad_of, pg, p.d_du = (void*)p.d_dy);
    MAY(poly_grad_of, pg, p.d_dcoefs = nullptr; p.d_work = nullptr);
    MUST(poly_grad_of, pg, p.n_coefs = 0);
    MUST(poly_grad_of, pg, p.n_coefs = 10);
    MUST(poly_grad_of, pg, p.work_bytes = poly_grad_work(&p) - 1);
    MUST(poly_grad_of, pg, p.d_coefs = nullptr);
    MUST(poly_grad_of, pg, p.d_dcoefs = (float*)p.d_coefs);
    MUST(poly_grad_of, pg, p.d_du = (void*)p.d_codes);

    he_weight_grad_plan w = {100, 40, 50, HE_BF16, HE_F32, 0, at(G), 40, (uint8_t*)at(2 * G), 64, (uint8_t*)at(3 * G), 1, at(4 * G), 50, at(5 * G), 1 << 30};
    MAY(weight_of, w, (void)p);
    MAY(weight_of, w, p.m = 0; p.d_dy = nullptr; p.d_codes = nullptr; p.d_exponents = nullptr; p.d_work = nullptr);
    MAY(weight_of, w, p.n = 0; p.d_dw = nullptr);
    MUST(weight_of, w, p.out_dtype = 7);
    MUST(weight_of, w, p.m = (1 << 21) + 1);
    MUST(weight_of, w, p.n = (1 << 17) + 1);
    MUST(weight_of, w, p.k = (1 << 17) + 1);
    MUST(weight_of, w, p.ld_codes = 56);
    MUST(weight_of, w, p.ld_dw = 49);
    MUST(weight_of, w, p.d_dw = nullptr);
    MUST(weight_of, w, p.d_dw = (void*)p.d_dy);
    MUST(weight_of, w, p.d_dw = at(4 * G + 2));
    MUST(weight_of, w, p.m = 1 << 20; p.work_bytes = weight_grad_work(&p) - 1);
    MUST(weight_of, w, p.m = 1 << 20; p.d_work = (void*)p.d_dw);

    he_logprobs_plan lp = {10, 100, 5, HE_F32, 1.0f, at(G), 100, (int32_t*)at(2 * G), (float*)at(3 * G), (float*)at(4 * G), (float*)at(5 * G), (int32_t*)at(6 * G), (float*)at(7 * G), at(8 * G), 1 << 20};
    MAY(logprobs_of, lp, (void)p);
    MAY(logprobs_of, lp, p.d_tokens = nullptr; p.d_logp = nullptr);
    MAY(logprobs_of, lp, p.k = 0; p.d_values = nullptr; p.d_index = nullptr);
    MAY(logprobs_of, lp, p.rows = 0; p.d_z = nullptr);
    MUST(logprobs_of, lp, p.k = 101);
    MUST(logprobs_of, lp, p.vocab = 200; p.k = 129);
    MUST(logprobs_of, lp, p.k = 0);
    MUST(logprobs_of, lp, p.d_index = nullptr);
    MUST(logprobs_of, lp, p.d_logp = nullptr);
    MUST(logprobs_of, lp, p.vocab = 0);
    MUST(logprobs_of, lp, p.vocab = (1 << 20) + 1);
    MUST(logprobs_of, lp, p.tau = 0);
    MUST(logprobs_of, lp, p.tau = 0x1p61f);
    MUST(logprobs_of, lp, p.ld_z = 99);
    MUST(logprobs_of, lp, p.d_entropy = p.d_logp);
    MUST(logprobs_of, lp, p.d_logp = (float*)p.d_tokens);
    MUST(logprobs_of, lp, p.d_values = (float*)p.d_z);

    he_logprobs_grad_plan g = {10, 100, HE_F32, 1.0f, at(G), 100, (int32_t*)at(2 * G), (float*)at(3 * G), (float*)at(4 * G), (float*)at(5 * G), at(6 * G), 100};
    MAY(refuse_logprobs_grad, g, (void)p);
    MAY(refuse_logprobs_grad, g, p.d_grad = (void*)p.d_z);
    MAY(refuse_logprobs_grad, g, p.d_tokens = nullptr; p.d_logp_weights = nullptr);
    MUST(refuse_logprobs_grad, g, p.d_tokens = nullptr);
    MUST(refuse_logprobs_grad, g, p.d_grad = (void*)p.d_z; p.ld_grad = 101);
    MUST(refuse_logprobs_grad, g, p.d_grad = (void*)p.d_stats);
    MUST(refuse_logprobs_grad, g, p.d_stats = nullptr);

    // cuts: every step of 32 rows belongs to one part, and none is empty
    const uint32_t sizes[] = {1, 2, 31, 32, 33, 100, 777, 1000, 4096, 20011, 65536, 1 << 17};
    for (uint32_t m : sizes)
        for (uint32_t n : sizes)
            for (uint32_t k : sizes) {
                for (int32_t t = 0; t < 3; t++) {
                const WeightCut c = weight_cut(m, n, k, t);
                const uint32_t steps = (m + 31) / 32;
                if (c.parts < 1 || c.parts > 65535 || c.per < 1 || (uint64_t)(c.parts - 1) * c.per >= steps || (uint64_t)c.parts * c.per < steps) { bad++; printf("cut of %u %u %u\n", m, n, k); }
                if (c.side != (n > 64 ? 128 : 64) && (c.side != 256 || n < 256)) { bad++; printf("tile of %u %u %u\n", m, n, k); }
                }
            }
    if (weight_cut(0, 5, 7, HE_F32).parts != 1 || weight_cut(0, 5, 7, HE_F32).per != 0) { bad++; printf("cut of no rows\n"); }
    for (uint32_t rows : sizes)
        for (uint32_t dim : sizes)
            if (dim <= HE_DIM_MAX && (layernorm_parts(rows, dim) < 1 || layernorm_parts(rows, dim) > rows || layernorm_parts(rows, dim) > 65535 || poly_groups(rows, dim, 1024) < 1)) { bad++; printf("parts of %u %u\n", rows, dim); }
    printf("%d bad\n", bad);
    return bad != 0;
}
'''


def test_refusals(tmp_path):
    src, exe = tmp_path / "checks.cc", tmp_path / "checks"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wno-unused-value", "-I", os.path.join(ROOT, "paper_2302_02407_amd", "csrc"), str(src), "-o", str(exe)], check=True, timeout=120)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout


BOUND = r"""
#include <stdio.h>
#include "checks.h"

int main() {
    int bad = 0;
    for (int32_t t = 0; t < 3; t++)
        for (uint64_t m = 1; m <= 1 << 21; m = m * 7 / 4 + 1)
            for (uint64_t n = 1; n <= 1 << 17; n = n * 5 / 4 + 1)
                for (uint64_t k = 1; k <= 1 << 17; k = k * 5 / 4 + 1) {
                    he_weight_grad_plan p = {};
                    p.m = m, p.n = n, p.k = k, p.dtype = t;
                    const uint64_t bytes = weight_grad_work(&p), parts = weight_cut(m, n, k, t).parts;
                    if (bytes > 1ull << 30 || bytes != (parts > 1 ? parts * n * ((k + 3) / 4 * 4) * 4 : 0)) bad++;
                }
    printf("%d bad\n", bad);
    return bad != 0;
}
"""


def on_host(tmp_path, program):
    """What a program says that is compiled for the host with the header of checks."""
    src, exe = tmp_path / "program.cc", tmp_path / "program"
    src.write_text(program)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", os.path.join(ROOT, "paper_2302_02407_amd", "csrc"), str(src), "-o", str(exe)], check=True, timeout=120)
    return subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)


def test_scratch_memory_of_a_weight_gradient_has_a_bound(tmp_path):
    r = on_host(tmp_path, BOUND)
    assert r.returncode == 0, r.stdout


PARTED = r"""
#include <stdio.h>
#include "checks.h"

int main() {
    int bad = 0;
    for (int32_t t = 0; t < 3; t++)
        for (uint32_t rows = 1; rows <= 600; rows++)
            for (uint32_t vocab = 1; vocab <= HE_VOCAB_MAX; vocab += 1 + vocab / 97) {
                const LogprobCut c = logprobs_cut(rows, vocab, t);
                const uint64_t last = vocab - (uint64_t)(c.parts - 1) * c.len;
                // every element in one part, and the last part not empty
                if (c.parts < 1 || (uint64_t)(c.parts - 1) * c.len >= vocab || (uint64_t)c.parts * c.len < vocab) bad++;
                // as many as the join takes; in each as many as can be asked for, and more than a wavefront's launch has
                if (c.parts > 1 && (c.parts > HE_JOIN_PARTS || last < HE_TOP_MAX || c.len < HE_TOP_MAX || (uint64_t)c.len * dtype_bytes(t) <= 4096 || c.len % 16)) bad++;
            }
    printf("%d bad\n", bad);
    return bad != 0;
}
"""


def test_parts_of_a_row_of_logits(tmp_path):
    r = on_host(tmp_path, PARTED)
    assert r.returncode == 0, r.stdout


CUTS = r"""
#include <stdio.h>
#include "checks.h"

int main() {
    const uint32_t want[][6] = {%s};                     // m, n, k, tile, parts, whether rows are asked for further ahead
    int bad = 0;
    for (auto& w : want) {
        const WeightCut c = weight_cut(w[0], w[1], w[2], HE_BF16);
        if (c.side != w[3] || c.parts != w[4] || c.ahead != (w[5] != 0)) { bad++; printf("%%u %%u %%u: %%u %%u %%d\n", w[0], w[1], w[2], c.side, c.parts, c.ahead); }
    }
    return bad != 0;
}
"""


def test_sizes_that_take_every_launch_of_a_weight_gradient(tmp_path):
    """Those that the tests on the GPU go by: kinds of tiles of bfloat16, whole and in parts, with rows asked for one step and four steps ahead."""
    from test_gpu_weight_grad import LAUNCHES
    r = on_host(tmp_path, CUTS % ", ".join("{%d, %d, %d, %d, %d, %d}" % row for row in LAUNCHES))
    assert r.returncode == 0, r.stdout


def test_every_operator_is_exported():
    for f in ("he_layernorm", "he_layernorm_grad", "he_poly_q8", "he_poly_grad_q8", "he_weight_grad_q8", "he_token_logprobs", "he_token_logprobs_grad",
              "he_work_layernorm_grad", "he_work_poly_grad_q8", "he_work_weight_grad_q8", "he_work_token_logprobs"):
        assert callable(getattr(B.HEContext, f)) and f in B.EXPORTS
