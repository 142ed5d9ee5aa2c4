"""The rule that picks a tile of attention over 4-bit codes (host code, no GPU), where a row has two groups: its estimate has no term for the second one and lies below
what its comment measures by much the same share in tiles of either size, so that it still takes the quicker one."""
from nibble_tiles import tiles

# units, tokens of the longest chunk, heads a KV head, cached rows; us in tiles of 32 and of 256 rows
MEASURED = [(256, 96, 1, 4096, 118, 145), (256, 200, 1, 4096, 260, 198), (128, 128, 1, 8192, 133, 153), (128, 256, 1, 8192, 262, 219),
            (64, 256, 1, 8192, 131, 124), (4, 585, 7, 2048, 52, 62), (8, 1024, 4, 32768, 907, 761), (8, 584, 7, 32768, 896, 751)]


def test_what_the_rule_reckons_and_takes():
    for (*shape, us32, us256), (tile, _, cost32, cost256) in zip(MEASURED, tiles([(*m[:4], 64) for m in MEASURED])):
        assert 1.09 <= us32 / cost32 <= 1.31 and 1.12 <= us256 / cost256 <= 1.29, (shape, us32 / cost32, us256 / cost256)
        assert tile == (32 if us32 < us256 else 256), shape


def test_one_group():
    """... and what the comment says of one: the sizes, and the call that is well off the estimate but not near the border."""
    for (*shape, us32, us256), (tile, _, cost32, cost256) in zip(
            [(256, 96, 1, 4096, 100, 121), (256, 200, 1, 4096, 221, 165), (128, 128, 1, 8192, 110, 125), (128, 256, 1, 8192, 214, 191), (64, 256, 1, 8192, 112, 106),
             (8, 1024, 4, 32768, 744, 640)],
            tiles([(256, 96, 1, 4096, 128), (256, 200, 1, 4096, 128), (128, 128, 1, 8192, 128), (128, 256, 1, 8192, 128), (64, 256, 1, 8192, 128), (8, 1024, 4, 32768, 128)])):
        assert abs(cost32 / us32 - 1) <= 0.12 and abs(cost256 / us256 - 1) <= 0.06, (shape, cost32 / us32, cost256 / us256)
        assert tile == (32 if us32 < us256 else 256), shape
    tile, splits, cost32, cost256 = tiles([(128, 2048, 1, 8192, 128)])[0]
    assert (tile, splits) == (256, 1) and round(cost256) == 1659 and round(cost32) == 2228
