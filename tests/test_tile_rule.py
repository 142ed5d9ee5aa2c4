"""The rule that picks a tile of akvq_paged_attention (host code, no GPU) at the shapes that its comment measures: what it reckons for tiles of
32 and of 256 rows is within 19 % of both, and it takes the quicker one."""
from tile_rule import tiles

# units, tokens of the longest chunk, heads a KV head, cached rows; us in tiles of 32 and of 256 rows
MEASURED = [(256, 96, 1, 4096, 85, 97), (256, 200, 1, 4096, 188, 151), (128, 128, 1, 8192, 95, 112), (128, 256, 1, 8192, 185, 172),
            (64, 256, 1, 8192, 94, 102), (4, 585, 7, 2048, 39, 54), (4, 1024, 4, 32768, 320, 302), (4, 4096, 1, 64, 71, 59), (8, 2048, 1, 64, 42, 48)]


def test_what_the_rule_reckons_and_takes():
    for (*shape, us32, us256), (tile, cost32, cost256) in zip(MEASURED, tiles([m[:4] for m in MEASURED])):
        assert abs(cost32 / us32 - 1) <= 0.19 and abs(cost256 / us256 - 1) <= 0.19, (shape, cost32, cost256)
        assert tile == (32 if us32 < us256 else 256), shape


def test_few_rows():
    assert [t for t, _, _ in tiles([(1, 1, 1, 0), (512, 16, 1, 1 << 20), (8, 8, 4, 32768), (32, 8, 4, 32768), (1, 33, 1, 0), (256, 64, 1, 1 << 20)])] == \
        [16, 16, 16, 32, 32, 32]
    assert tiles([(1, 65535 * 32 + 1, 1, 0)])[0][0] == 256  # tiles are a grid dimension
