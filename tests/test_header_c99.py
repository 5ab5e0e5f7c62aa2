"""The C header in the strictest C that its declarations need, and a descriptor's last field by each of its names (no GPU needed)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
COMPILERS = [c for c in (shutil.which("gcc"), "/opt/rocm/llvm/bin/clang") if c and os.path.exists(c)]

PROGRAM = """
#include <vq.h>
static const vq_attn_desc in_order = {32, 8, 128, 16, 100, VQ_F16, 0.1f, 0};
static const vq_attn_desc by_name = {.heads = 32, .kv_heads = 8, .reserved = 0};
static const vq_attn_desc in_8_bits = {.heads = 32, .kv_heads = 8, .cache_dtype = VQ_E4M3};
typedef char same_size[sizeof(vq_attn_desc) == 32 ? 1 : -1];
int main(void) { return in_order.reserved != 0 || by_name.cache_dtype != 0 || in_8_bits.reserved != VQ_E4M3 || sizeof(same_size) != 1; }
"""


@pytest.mark.skipif(not COMPILERS, reason="no C compiler")
@pytest.mark.parametrize("standard", ["c99", "c11", "c17"])
@pytest.mark.parametrize("compiler", COMPILERS)
def test_strict_c(tmp_path, compiler, standard):
    source, program = tmp_path / "program.c", tmp_path / "program"
    source.write_text(PROGRAM)
    res = subprocess.run([compiler, f"-std={standard}", "-pedantic-errors", "-I", os.path.join(ROOT, "include"), str(source), "-o", str(program)],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    assert subprocess.run([str(program)]).returncode == 0
