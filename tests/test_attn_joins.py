"""Generated code of prompts' joins (no GPU needed): a sum over values is one product and one fused multiplication and addition, and which of the two products
is the fused one is the same in every build, as are, with it, the last bits of what calls return."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2402_15319_amd import build as vqbuild

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not available")


def registers(text):
    found = set()
    for m in re.finditer(r"\bv\[(\d+):(\d+)\]|\bv(\d+)\b", text):
        found |= {int(m[3])} if m[3] else set(range(int(m[1]), int(m[2]) + 1))
    return found


def fused_with_a_loaded_value(lines, load):
    """How many fused operations multiply a register as `load` left it."""
    loaded, count = set(), 0
    for line in lines:
        op, _, rest = line.split(";")[0].strip().partition(" ")
        ops = [x.strip() for x in rest.split(",")]
        if op == load:
            loaded |= registers(ops[0])
            continue
        if op.startswith(("v_fmac_f32", "v_fma_f32")):
            count += bool((registers(ops[1]) | registers(ops[2])) & loaded)
        if op.startswith("v_"):
            loaded -= registers(ops[0])
    return count


def test_the_count_tells_the_two_ways_apart():
    load = "ds_read_b128 v[4:7], v1 offset:1024"
    new = [load, "v_mul_f32_e32 v10, v2, v18", "v_fmac_f32_e32 v10, v3, v5"]
    old = [load, "v_mul_f32_e32 v5, v3, v5", "v_fmac_f32_e32 v5, v2, v18"]
    assert fused_with_a_loaded_value(new, "ds_read_b128") == 1
    assert fused_with_a_loaded_value(old, "ds_read_b128") == 0


SOURCES = ["vq_attn_prompt.hip", "vq_attn_prompt_256.hip", "vq_attn_prompt_window.hip", "vq_attn_prompt_window_256.hip", "vq_attn_prompt8.hip",
           "vq_attn_prompt8_256.hip"]


@pytest.mark.parametrize("source", SOURCES)
def test_which_product_is_fused(tmp_path, source):
    out = tmp_path / "code.s"
    cmd = [HIPCC, *(f for f in vqbuild.HIPCC_FLAGS if f != "-fPIC"), *vqbuild.SOURCE_FLAGS.get(source, []), "-S", "--cuda-device-only", "-o", str(out),
           os.path.join(vqbuild.CSRC, source)]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-2000:]
    kernels = re.findall(r"^(_ZN\S*prompt\S*_kernelILb\dELi(\d+)ELi(\d)E\S*):.*?\n(.*?)^\.Lfunc_end", out.read_text(), re.M | re.S)
    assert len(kernels) == (2 if "256" in source else 12)
    plain = "window" not in source and "prompt8" not in source
    for name, dim, teams, text in kernels:
        lines, dim = text.splitlines(), int(dim)
        sums = dim // 2                                                 # of a lane
        last = next(i for i, t in enumerate(lines) if "global_atomic_add" in t)
        # parts: behind the counter, up to the first value that is rounded
        end = next(i for i in range(last, len(lines)) if re.search(r"v_cvt_pk|v_cvt_f16|permlane", lines[i]))
        assert fused_with_a_loaded_value(lines[last:end], "global_load_dwordx2") == (sums if plain and dim in (64, 256) else 0), name
        if teams == "2":   # between the last barriers in front of it
            barriers = [i for i, t in enumerate(lines[:last]) if "s_barrier" in t]
            first = next(b for b in reversed(barriers) if sum("v_fmac_f32" in t for t in lines[b:last]) > sums // 2)
            assert fused_with_a_loaded_value(lines[first:last], "ds_read_b128") == (sums if plain else 24), name
