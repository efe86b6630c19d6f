"""CPU: the plans that the binding packs have the layout that a C compiler gives them."""
import os
import struct
import subprocess

import pytest

from paper_2302_02407_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
FIELDS = {
    "he_rmsnorm_plan": (B._RMSNORM, "rows dim dtype eps d_x ld_x d_residual ld_residual d_weight d_sum ld_sum d_codes ld_codes d_scales ld_scales"),
    "he_matmul_plan": (B._MATMUL, "m n k out_dtype fast_sums d_a ld_a d_a_scales ld_a_scales d_w ld_w d_w_scales ld_w_scales d_out ld_out"),
    "he_top_plan": (B._TOP, "rows vocab k dtype tau d_z ld_z d_values d_index d_rest"),
    "he_distill_plan": (B._DISTILL, "rows vocab k dtype tau alpha d_z ld_z d_values d_index d_rest d_labels d_loss d_stats d_row_weights d_grad ld_grad"),
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
    fields = fields.split()
    lines = "".join('    printf("%%zu\\n", offsetof(%s, %s));\n' % (name, f) for f in fields)
    src, exe = tmp_path / "plan.c", tmp_path / "plan"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "he_mi355x.h"\nint main(void) {\n%s    printf("%%zu\\n", sizeof(%s));\n    return 0;\n}\n' % (lines, name))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(HERE, "..", "include"), str(src), "-o", str(exe)], check=True, timeout=60)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True, timeout=60).stdout.split()]
    assert got[:-1] == offsets(fmt)
    assert struct.calcsize(fmt.format) <= got[-1] < struct.calcsize(fmt.format) + 8      # what is past the last field is not read


def test_every_operator_is_exported():
    for f in ("he_rmsnorm_q8", "he_matmul_q8", "he_ws_query_matmul_q8", "he_top_logits", "he_distill_loss", "he_distill_grad"):
        assert callable(getattr(B.HEContext, f))
