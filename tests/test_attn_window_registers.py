"""Registers and instances of the kernels of windows and of pages in 8 bits (no GPU needed): what the launches count on."""
import re

from test_registers import pytestmark, resources  # noqa: F401


def _decode(resources, kernel):  # noqa: F811
    """{(bf16, head_dim, whole lines, waves, tiles): (vector registers, bytes of scratch)}"""
    found = {}
    for name, r in resources.items():
        m = re.search(kernel + r"ILb(\d)ELi(\d+)ELb(\d)ELi(\d)ELi(\d)EE", name)
        if m:
            found[tuple(map(int, m.groups()))] = r
    return found


def test_every_instance_is_one_that_a_plan_names(resources):  # noqa: F811
    shapes = {(d, w, t) for d in (64, 96, 128) for w, t in ((4, 1), (8, 1), (4, 2), (4, 3))} | {(256, 4, 1)}
    assert set(_decode(resources, "decode_window_kernel")) == {(b, d, lines, w, t) for b in (0, 1) for lines in (0, 1) for d, w, t in shapes}
    shapes -= {(96, 4, 3), (128, 4, 3)} | {(d, 8, 1) for d in (64, 96, 128)}
    assert set(_decode(resources, "decode8_kernel")) == {(b, d, lines, w, t) for b in (0, 1) for lines in (0, 1) for d, w, t in shapes}
    for kernel in ("prompt_window_kernel", "prompt8_kernel"):
        assert sum(kernel in n for n in resources) == 2 * 7
    assert sum("append8_few_kernel" in n for n in resources) == sum("append8_kernel" in n for n in resources) == 8


def test_scratch(resources):  # noqa: F811
    """None, but for three tiles of heads of 128 to a workgroup with a window, as without one (a window's bounds take 16 bytes more)."""
    kernels = {n: r for n, r in resources.items() if re.search(r"decode_window_kernel|decode8_kernel|prompt_window_kernel|prompt8_kernel|append8_", n)}
    spilled = {n: r[1] for n, r in kernels.items() if r[1]}
    assert all(re.search(r"decode_window_kernelILb.ELi128ELb.ELi4ELi3EE", n) and b <= 96 for n, b in spilled.items()), spilled


def test_waves_that_share_a_simd(resources):  # noqa: F811
    """As without a window, in 16 bits; in 8 bits heads of 96 and 128 have one wave fewer: twice as many tokens are under way in each."""
    for kernel, least in (("decode_window_kernel", {64: 4, 96: 3, 128: 3, 256: 1}), ("decode8_kernel", {64: 4, 96: 3, 128: 2, 256: 1})):
        for (_, d, _, waves, tiles), (registers, _) in _decode(resources, kernel).items():
            fit = 512 // (-(-registers // 8) * 8)
            assert fit >= (least[d] if tiles == 1 else 2), (kernel, d, waves, tiles, registers)
    for name, (registers, _) in resources.items():
        if "prompt_window_kernel" in name or "prompt8_kernel" in name:
            assert registers <= (512 if "Li256" in name else 256), name
