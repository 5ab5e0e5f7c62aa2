"""Registers and instances of the compiled attention and cache kernels (no GPU needed): what the launches count on."""
import re

from test_registers import pytestmark, resources  # noqa: F401


def _decode(resources):  # noqa: F811
    """{(bf16, head_dim, whole lines, waves, tiles): (vector registers, bytes of scratch)}"""
    found = {}
    for name, r in resources.items():
        m = re.search(r"decode_kernelILb(\d)ELi(\d+)ELb(\d)ELi(\d)ELi(\d)EE", name)
        if m and "DecodeArgs" in name:
            found[tuple(map(int, m.groups()))] = r
    return found


def test_every_instance_is_one_that_a_plan_names(resources):  # noqa: F811
    """8 waves take a sequence in one part, of more than 128 tokens and at most 32,768 values of a head's keys: none of 256 dimensions.  Several
    tiles share a workgroup of 4 waves up to 128 dimensions."""
    shapes = {(d, w, t) for d in (64, 96, 128) for w, t in ((4, 1), (8, 1), (4, 2), (4, 3))} | {(256, 4, 1)}
    assert set(_decode(resources)) == {(b, d, lines, w, t) for b in (0, 1) for lines in (0, 1) for d, w, t in shapes}


def test_scratch(resources):  # noqa: F811
    """None, but for three tiles of heads of 128 to a workgroup: two pieces of q (32 bytes) are read again in every step."""
    kernels = {n: r for n, r in resources.items() if re.search(r"decode_kernelILb.*DecodeArgs|prompt_kernel|append_|copy_kernel", n)}
    assert len(kernels) >= 4 * 13 + 2 * 7 + 7
    spilled = {n: r[1] for n, r in kernels.items() if r[1]}
    assert all(re.search(r"decode_kernelILb.ELi128ELb.ELi4ELi3EE", n) and b <= 80 for n, b in spilled.items()), spilled


def test_waves_that_share_a_simd(resources):  # noqa: F811
    """512 registers of a SIMD, in eights, and what the launch bounds promise: two workgroups of 4 waves to a compute unit, but for heads of 256."""
    for (_, d, _, waves, tiles), (registers, _) in _decode(resources).items():
        fit = 512 // (-(-registers // 8) * 8)
        assert fit >= (1 if d == 256 else 2), (d, waves, tiles, registers)
        if tiles == 1:
            assert fit >= {64: 4, 96: 4, 128: 3, 256: 1}[d], (d, waves, registers)
    for name, (registers, _) in resources.items():
        if "prompt_kernel" in name:
            assert registers <= (512 if "Li256" in name else 256), name
