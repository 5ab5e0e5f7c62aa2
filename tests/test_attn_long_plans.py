"""The prompts of tests/test_gpu_attn_long.py are split into parts of more steps than a wave's 64 page numbers last for (no GPU needed)."""
import os
import shutil
import subprocess

import pytest

from test_gpu_attn_long import LONG

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not available")
def test_parts_of_many_steps(tmp_path):
    out = tmp_path / "attn_plan_print"
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           os.path.join(ROOT, "paper_2402_15319_amd", "csrc", "vq_attn_api.hip"),
           os.path.join(ROOT, "tests", "host", "attn_plan_print.cpp"), "-o", str(out)]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-3000:]
    seen = set()
    for heads, kv, dim, _, n_seqs, length, new in LONG:
        res = subprocess.run([str(out), *map(str, (heads, kv, dim, n_seqs, n_seqs * new, length))], capture_output=True, text=True, timeout=60)
        assert res.returncode == 0
        _, _, teams, steps, parts = map(int, res.stdout.split())
        assert steps > 64 * teams, (heads, kv, dim, n_seqs, length, res.stdout)
        seen.add((teams, parts > 1))
    assert seen >= {(1, False), (2, False), (1, True)}
