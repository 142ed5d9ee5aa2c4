"""What the compiler gave the kernels over pages, read from the metadata of the built library (no GPU needed), where splits and launch bounds count on it: three
workgroups of a tile of 16 on a CU (168 vector registers, a third of 160 KB of LDS), but for 4-bit codes of two groups with more than eight rows, and two of those
that turn rows on their way into pages (eight wavefronts each, 128 registers)."""
import re

from test_kernel_resources import kernels  # noqa: F401


def test_three_workgroups_of_a_tile_of_16_per_cu(kernels):  # noqa: F811
    seen = set()
    for name, f in kernels.items():
        at = re.search(r"paged_attention_kernelILi(\d+)ELi(\d+)ELb([01])ELi(\d)ELb([01])E", name)
        if not at:
            continue
        G, W, many, bits, eight = (int(x) for x in at.groups())
        seen.add((G, W, many, bits, eight))
        three = W == 16 and not (bits == 4 and G == 64 and not eight)
        assert int(f["vgpr_count"]) <= (168 if three else 256), (name, f["vgpr_count"])
        assert int(f["group_segment_fixed_size"]) <= 160 * 1024 // (3 if three else 1 if many else 2), (name, f["group_segment_fixed_size"])
    assert seen == {(G, W, many, bits, 0) for G in (64, 128) for W, many in ((16, 0), (32, 0), (32, 1)) for bits in (2, 4)} | {(64, 16, 0, 4, 1), (128, 16, 0, 4, 1)}


def test_two_workgroups_that_turn_rows_per_cu(kernels):  # noqa: F811
    found = [f for name, f in kernels.items() if "paged_turn_kernelI" in name]
    assert len(found) == 8
    for f in found:
        assert int(f["vgpr_count"]) <= 128 and int(f["group_segment_fixed_size"]) <= 160 * 1024 // 2
