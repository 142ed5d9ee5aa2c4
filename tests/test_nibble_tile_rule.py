"""The rules that pick a tile and the splits of attention over 4-bit codes (host code, no GPU), at the shapes that their comments measure."""
from nibble_tiles import tiles

# units, tokens of the longest chunk, heads a KV head, cached rows, G; us in tiles of 32 and of 256 rows
MEASURED = [(256, 96, 1, 4096, 128, 100, 121), (256, 200, 1, 4096, 128, 221, 165), (128, 128, 1, 8192, 128, 110, 125), (128, 256, 1, 8192, 128, 214, 191),
            (64, 256, 1, 8192, 128, 112, 106), (4, 585, 7, 2048, 64, 53, 60), (8, 1024, 4, 32768, 128, 744, 640)]


def test_what_the_rule_reckons_and_takes():
    for (*shape, us32, us256), (tile, _, cost32, cost256) in zip(MEASURED, tiles([m[:5] for m in MEASURED])):
        assert abs(cost32 / us32 - 1) <= 0.2 and abs(cost256 / us256 - 1) <= 0.21, (shape, cost32, cost256)
        assert tile == (32 if us32 < us256 else 256), shape


def test_few_rows():
    assert [t[0] for t in tiles([(1, 1, 1, 0, 128), (512, 16, 1, 1 << 20, 64), (32, 4, 7, 16384, 64), (128, 4, 7, 16384, 64), (64, 32, 1, 8192, 128), (1, 33, 1, 0, 128)])] == \
        [16, 16, 32, 32, 16, 32]


def test_splits():
    """One token a sequence: the choices that the rule's comment measures."""
    assert [n for _, n, _, _ in tiles([(512, 1, 1, 16384, 128), (512, 1, 1, 4096, 128), (256, 1, 1, 16384, 128), (128, 1, 7, 32768, 64), (512, 1, 1, 8192, 64),
                                       (32, 1, 1, 640, 128),
                                       (128, 1, 7, 16384, 64), (512, 1, 1, 16384, 64), (256, 2, 8, 8192, 64)])] == [4, 1, 6, 6, 1, 5, 6, 3, 2]


def test_splits_of_short_calls():
    """No merge where a wavefront has two pairs of blocks at most, and one reading of partial sums where sixteen splits leave it one."""
    assert [n for _, n, _, _ in tiles([(32, 1, 1, 320, 128), (32, 1, 1, 479, 128), (32, 1, 1, 480, 128), (32, 16, 1, 432, 128), (8, 1, 1, 3000, 128),
                                       (8, 1, 1, 3839, 128), (8, 1, 1, 3840, 128)])] == [1, 1, 4, 1, 16, 16, 30]
