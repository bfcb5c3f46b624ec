"""The block operators' kernels in the built library: which there are, and what the compiler made of them."""
import re

from test_kernel_resources import scratch_bytes  # noqa: F401


def _tiles(names):
    """(way, rows of b's blocks, rows of a tile, columns of a tile) of the product's tile kernels"""
    found = set()
    for name in names:
        m = re.search(r"k_f8_matmul_tilesILi\d+ELi(\d+)ELi(\d+)E.*?TileILi(\d+)ELi(\d+)ELi(\d+)E", name)
        if m:
            way, b_rows, wm, wn, mt = map(int, m.groups())
            found.add((way, b_rows, 16 * wm * mt, 64 * wn))
    return found


def test_the_product_has_the_tiles_that_its_choice_counts_with(scratch_bytes):  # noqa: F811
    """Ways 0 to 3: f32 scales, power-of-two scales, and both with f32 results.  128 x 128 everywhere; the large tile is 256 x 256,
    128 x 256 for f32 results with f32 scales, and not there for f32 scales of every row of b."""
    want = {(way, b_rows, 128, 128) for way in range(4) for b_rows in (1, 128)}
    want |= {(way, b_rows, 128 if way == 2 else 256, 256) for way in range(4) for b_rows in (1, 128)} - {(0, 1, 256, 256)}
    assert _tiles(scratch_bytes) == want


def test_kernels_that_keep_nothing_in_scratch_memory(scratch_bytes):  # noqa: F811
    """All of the quantizer's and the product's, the forward norms of up to 8192 channels (one group of 8 values a lane) and, in
    bf16 and f16, their gradients from 129 channels on."""
    quiet = [k for k in scratch_bytes if re.search(r"k_f8_|k_strip_sums|k_column_sums|k_fill_rows|k_block_normI.*Li1ELb", k)]
    quiet += [k for k in scratch_bytes if re.search(r"k_block_norm_backwardI(?!f).*Li(64|128|256|512|1024)ELi1ELb", k)]
    assert len(quiet) > 150
    assert not {k: scratch_bytes[k] for k in quiet if scratch_bytes[k]}


def test_scratch_memory_of_the_other_norms(scratch_bytes):  # noqa: F811
    """What rows of more than 8192 channels, f32 gradients and gradients of up to 128 channels keep there, at most."""
    at_most = [(r"k_block_normI.*Li1024ELi2ELb", 380), (r"k_block_norm_backwardI.*Li1024ELi2ELb", 704),
               (r"k_block_norm_backwardI.*Li16ELi1ELb", 116), (r"k_block_norm_backwardIff.*Li(64|128|256|512|1024)ELi1ELb", 32)]
    for pattern, limit in at_most:
        found = {k: v for k, v in scratch_bytes.items() if re.search(pattern, k)}
        assert found and max(found.values()) <= limit, found
