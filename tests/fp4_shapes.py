"""Products of 4-bit floating point that reach every kind of output tile, in both formats, with rows of y that start on 16-byte
boundaries (N % 8 == 0) and others."""

# (channels, rows of x to a tile, runs of K, whether the product quantises x itself), M, N, K
PRODUCTS = [
    # up to sixteen rows, quantised by the product: whole K, two and four runs of it
    ((128, 16, 1, True), 16, 72, 192), ((128, 16, 1, True), 3, 9601, 800),
    ((128, 16, 2, True), 14, 40, 480), ((128, 16, 2, True), 4, 339, 480),
    ((128, 16, 4, True), 11, 200, 1024), ((128, 16, 4, True), 7, 45, 832),
    # up to sixteen rows, too long for that
    ((128, 64, 1, False), 13, 9600, 1312), ((128, 64, 1, False), 16, 9601, 1312),
    ((128, 64, 2, False), 13, 7688, 2848), ((128, 64, 2, False), 15, 7601, 2848),
    ((128, 64, 4, False), 16, 600, 8192), ((128, 64, 4, False), 9, 333, 8224),
    # tiles of 64 rows: whole K, in one round and in several, and two runs of it
    ((128, 64, 1, False), 99, 336, 544), ((128, 64, 1, False), 50, 24001, 544),
    ((128, 64, 2, False), 98, 296, 6528), ((128, 64, 2, False), 105, 305, 6496),
    # tiles of 128 rows: the same
    ((128, 128, 1, False), 1180, 2288, 320), ((128, 128, 1, False), 1432, 1859, 320),
    ((128, 128, 2, False), 333, 1560, 14240), ((128, 128, 2, False), 257, 1813, 14176),
    # pairs of CTAs; 192 rows to a tile: every second tile starts at row 64 of a row block
    ((256, 128, 1, False), 1943, 528, 7040), ((256, 128, 1, False), 1885, 543, 7456), ((256, 128, 1, False), 1604, 2656, 4384),
    ((256, 192, 1, False), 655, 3440, 800), ((256, 192, 1, False), 653, 3407, 800), ((256, 192, 1, False), 1307, 5208, 288), ((256, 192, 1, False), 901, 7193, 288),
    ((256, 256, 1, False), 774, 3608, 1312), ((256, 256, 1, False), 819, 3605, 1312), ((256, 256, 1, False), 1164, 5672, 800), ((256, 256, 1, False), 1162, 5659, 800),
]
# (channels, rows of x to a tile), rows of each matrix, N, K; the last of each kind has more tiles than the GPU takes at once
ROUTED = [
    ((128, 64), [64, 1, 0, 65, 30, 7, 128, 16], 264, 544), ((128, 64), [64, 1, 0, 65, 30, 7, 128, 16], 2440, 288),
    ((128, 128), [100, 0, 65, 129, 1, 128, 200], 264, 544), ((128, 128), [100, 0, 65, 129, 1, 128, 200], 2440, 288),
    ((256, 256), [300, 0, 700, 257, 1000], 328, 544), ((256, 256), [300, 0, 700, 257, 1000], 1333, 544), ((256, 256), [300, 0, 700, 257, 1000], 1672, 544),
]
