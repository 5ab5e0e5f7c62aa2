"""A workspace of attention over the paged cache serves every smaller batch (tests/host/attn_workspace_check.cpp, no GPU needed)."""
import os
import shutil
import subprocess

import pytest

import paper_2402_15319_amd as vq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not available")
def test_a_workspace_serves_every_smaller_batch(tmp_path):
    out = tmp_path / "attn_workspace_check"
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           os.path.join(ROOT, "paper_2402_15319_amd", "csrc", "vq_attn_api.hip"),
           os.path.join(ROOT, "tests", "host", "attn_workspace_check.cpp"), "-o", str(out)]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-3000:]
    res = subprocess.run([str(out)], capture_output=True, text=True, timeout=600)
    assert res.returncode == 0 and res.stdout.strip() == "workspace check ok", res.stdout[-2000:] + res.stderr[-2000:]


@pytest.mark.parametrize("heads, kv, large, small", [
    (32, 32, (4, 4, 4096), (1, 1, 4096)),            # fewer sequences are split into more parts
    (32, 32, (1, 4096, 12288), (1, 512, 8704)),      # a chunk of 512 behind 8,192 tokens, one of 4,096
    (32, 8, (1, 1, 1152), (1, 1, 1024)),             # shorter ones too
    (48, 1, (64, 64, 8192), (3, 3, 8192)),
    (32, 8, (8, 2000, 4096), (8, 8, 4096)),          # a step of single tokens behind prompts
])
def test_sizes_do_not_grow_as_batches_shrink(heads, kv, large, small):
    desc = vq.make_attn_desc(heads, kv, 128, 16, 10000)
    batch = lambda n_seqs, n_tokens, max_len: type("B", (), {"struct": vq.VQAttnBatch(n_seqs, n_tokens, 4096, max_len, 1 << 16, 1 << 16, 1 << 16)})  # noqa: E731
    assert vq.vq_attn_workspace_bytes(desc, batch(*large)) >= vq.vq_attn_workspace_bytes(desc, batch(*small))
