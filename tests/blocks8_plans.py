"""How the weights' gradient of a size runs: rows, n, k, then the tile (256 x 256, 256 x 128 or
128 x 128 of n x k), into how many shares the rows of a partial last round's tiles
are cut, the tiles of whole rounds, and all tiles.  Every kind of plan that small sizes reach,
with edges that no tile divides."""
TILES = [(256, 256), (256, 128), (128, 128)]

WEIGHT_GRADIENTS = [
    # a partial round, in one piece
    (70, 776, 8248, 0, 1, 0, 132), (70, 392, 8368, 1, 1, 0, 132), (70, 136, 264, 2, 1, 0, 6),
    # a partial round, in shares
    (7177, 272, 5536, 0, 5, 0, 44), (10947, 2056, 520, 1, 5, 0, 45), (8003, 1288, 1288, 1, 3, 0, 66), (1001, 520, 520, 2, 4, 0, 25),
    # one whole round
    (70, 3888, 4000, 0, 1, 256, 256), (70, 832, 8128, 1, 1, 256, 256), (70, 408, 8112, 2, 1, 256, 256),
    # a whole round and a rest in one piece
    (70, 2104, 7272, 0, 1, 256, 261), (70, 1592, 9256, 1, 1, 256, 511),
    # a whole round and a rest in shares, as fused projections of 2560 channels run
    (4001, 4232, 4104, 0, 5, 256, 289), (1501, 4232, 4104, 0, 3, 256, 289), (2003, 7680, 2560, 0, 3, 256, 300),
    (1922, 1624, 4712, 1, 8, 256, 259),
]


def workspace_bytes(plan):
    """What the shares' sums take: unequal to those of any other tile or number of shares of the size."""
    _, n, k, tile, shares, whole, tiles = plan
    return (tiles - whole) * shares * TILES[tile][0] * TILES[tile][1] * 4 if shares > 1 else 0
