"""The kernels of the products in 8-bit integers, the group norm and the clipped gradients in the built library: which there are,
and that none keeps anything in scratch memory."""
import re

from test_kernel_resources import scratch_bytes  # noqa: F401


def test_the_product_has_the_tiles_that_its_choice_counts_with(scratch_bytes):  # noqa: F811
    found = {tuple(map(int, m.groups())) for name in scratch_bytes for m in [re.search(r"k_i8_matmul_tiles.*?TileILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)E", name)] if m}
    assert {(16 * wm * mt, 16 * wn * nt, stages) for wm, wn, mt, nt, stages in found} == {(128, 128, 2), (128, 128, 4), (256, 256, 2)}


def test_nothing_in_scratch_memory(scratch_bytes):  # noqa: F811
    quiet = [k for k in scratch_bytes if re.search(r"k_i8_|k_group_norm_|k_clip_", k)]
    assert len(quiet) > 150
    assert not {k: scratch_bytes[k] for k in quiet if scratch_bytes[k]}
