"""Generated code of prompts with a window over 16-bit pages (no GPU needed): a wave that takes values that are no numbers out of LDS says so in a
word first, and the waves look at these words behind their reads of values.  A wave that finds values gone relies on that order: it adds again what they were."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2402_15319_amd import build as vqbuild

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not available")


@pytest.mark.parametrize("source, instances", [("vq_attn_prompt_window.hip", 12), ("vq_attn_prompt_window_256.hip", 2)])
def test_the_word_is_written_before_the_values_and_read_behind_them(tmp_path, source, instances):
    out = tmp_path / "code.s"
    cmd = [HIPCC, *(f for f in vqbuild.HIPCC_FLAGS if f != "-fPIC"), *vqbuild.SOURCE_FLAGS.get(source, []), "-S", "--cuda-device-only", "-o", str(out),
           os.path.join(vqbuild.CSRC, source)]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-2000:]
    kernels = re.findall(r"^(_ZN\S*prompt_window_kernel\S*):.*?\n(.*?)^\.Lfunc_end", out.read_text(), re.M | re.S)
    assert len(kernels) == instances
    for name, text in kernels:
        lines = [t for t in (t.strip() for t in text.splitlines()) if t.startswith(("ds_", ".LBB", "; words: ", "s_barrier"))]
        written = [i for i, t in enumerate(lines) if t == "; words: written"]
        read = [i for i, t in enumerate(lines) if t == "; words: read"]
        assert written and len(read) == 1, name
        for i in written:
            block = max((j for j in range(i) if lines[j].startswith(".LBB")), default=0)
            before = [t for t in lines[block:i] if t.startswith("ds_write")]
            behind = next(t for t in lines[i:] if t.startswith("ds_write"))
            assert len(before) == 1 and before[0].startswith("ds_write_b32"), (name, before)
            assert behind.startswith("ds_write_b128"), (name, behind)
        assert next(t for t in lines[read[0]:] if t.startswith(("ds_", "s_barrier"))).startswith("ds_read"), name
