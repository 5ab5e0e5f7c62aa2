"""Generated code of attention of one new token, three tiles of heads of 128 to a workgroup (no GPU needed): a step gets two pieces of q from scratch, and with a
window one number more.  The address of V among them, which a step would wait for, costs 9 % (64 sequences, 48 heads to one key/value head)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2402_15319_amd import build as vqbuild

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not available")


@pytest.mark.parametrize("source, kernel, most", [("vq_attn_decode.hip", "decode_kernel", 2), ("vq_attn_decode_window.hip", "decode_window_kernel", 3)])
def test_a_step_of_three_tiles(tmp_path, source, kernel, most):
    out = tmp_path / "code.s"
    cmd = [HIPCC, *(f for f in vqbuild.HIPCC_FLAGS if f != "-fPIC"), *vqbuild.SOURCE_FLAGS.get(source, []), "-S", "--cuda-device-only", "-o", str(out),
           os.path.join(vqbuild.CSRC, source)]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-2000:]
    kernels = re.findall(rf"^(_ZN\S*{kernel}ILb\dELi128ELb\dELi4ELi3E\S*):.*?\n(.*?)^\.Lfunc_end", out.read_text(), re.M | re.S)
    assert len(kernels) == 4
    for name, text in kernels:
        lines, steps = text.splitlines(), 0
        for i, t in enumerate(lines):
            if not (t.startswith(".LBB") and "Loop Header" in t):
                continue
            label = re.escape(t.split(":")[0]) + r"\b"
            end = max((j for j in range(i + 1, len(lines)) if re.search(r"\bs_\w*branch\w* " + label, lines[j])), default=i)
            loop = lines[i:end]
            if sum("v_exp_f32" in x for x in loop) >= 24:                  # the weights of 3 x 8 tokens a lane
                steps += 1
                assert sum("v_mfma" in x for x in loop) == 48, name
                assert sum("scratch_load" in x for x in loop) <= most and not any("scratch_store" in x for x in loop), name
        assert steps == 1, name
