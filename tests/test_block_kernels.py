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
