"""Sizes of products that reach every tile shape of the linear layer: (rows, columns, length of the sum), and the tile that they are
cut into with operands of 2 or 4 bytes.  Sums of several slabs (128 bytes of a row) with something left over; whole ones too."""

HALF = {
    256: [(4099, 3080, 330), (3080, 4104, 320), (4099, 3079, 72)],
    128: [(2100, 2200, 330), (2177, 2049, 1025)],
    64: [(1100, 1000, 330), (1500, 1501, 200), (1027, 1100, 1024)],      # the first and last with slabs ahead where that goes
    32: [(600, 500, 330), (520, 530, 448)],
}
SPLIT_HALF = [(300, 500, 1100), (100, 120, 4099), (700, 33, 2048)]
SINGLE = {
    128: [(3700, 3701, 150), (3717, 3650, 128)],
    64: [(1100, 1000, 200), (1501, 1500, 161)],
    32: [(600, 500, 165)],
}
SPLIT_SINGLE = [(300, 500, 600), (100, 120, 2051)]
# both products of a gradient in one launch: (m, n, k), tile of both
PAIRS = [((520, 530, 512), 32), ((800, 808, 790), 64), ((1000, 777, 900), 64)]


def sizes(itemsize):
    """(rows, columns, sum, tile, split or not) of every product above for this type."""
    whole, split = (HALF, SPLIT_HALF) if itemsize == 2 else (SINGLE, SPLIT_SINGLE)
    return [(*s, tile, False) for tile, some in whole.items() for s in some] + [(*s, 32, True) for s in split]
