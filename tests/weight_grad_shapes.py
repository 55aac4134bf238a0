"""Rows, columns of dY and columns of X for the tests of the weight gradient that have to reach a particular form of it."""

SMALL = (70, 40, 200)                               # tiles of 128 x 128
FEW = (70, 5, 200)                                  # fewer than eight columns of dY
LARGE = [(1, 4099, 4100), (70, 4099, 4100), (333, 4001, 5003), (64, 4096, 4096)]         # tiles of 256 x 256, the rows in one piece
LARGE_SPLIT = [(3000, 2300, 2051), (8200, 2048, 2048)]                                   # and split
