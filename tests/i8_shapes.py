"""Products of 8-bit integers that reach every kind of output tile, with rows of y that start on 16-byte boundaries (N % 8 == 0) and others."""

# (channels, rows of x to a tile, runs of K, whether the product quantises x itself), M, N, K
PRODUCTS = [
    # up to sixteen rows, quantised by the product: whole K, in one round and in several, two and four runs of it
    ((128, 16, 1, True), 3, 9602, 400), ((128, 16, 1, True), 7, 19136, 528), ((128, 16, 1, True), 1, 19934, 144),
    ((128, 16, 2, True), 9, 331, 208), ((128, 16, 2, True), 5, 4840, 1504),
    ((128, 16, 4, True), 16, 201, 1008), ((128, 16, 4, True), 2, 264, 7184),
    # up to sixteen rows, too long for that
    ((128, 64, 1, False), 13, 10165, 4176), ((128, 64, 1, False), 1, 19456, 4128), ((128, 64, 2, False), 13, 5583, 1200), ((128, 64, 2, False), 11, 4840, 1504),
    ((128, 64, 4, False), 15, 331, 1296), ((128, 64, 4, False), 4, 264, 7184),
    # tiles of 64 rows: whole K, in one round and in several, two and four runs of it
    ((128, 64, 1, False), 99, 337, 544), ((128, 64, 1, False), 37, 19344, 272),
    ((128, 64, 2, False), 23, 5165, 5968), ((128, 64, 2, False), 20, 5720, 5856), ((128, 64, 4, False), 33, 331, 4656), ((128, 64, 4, False), 70, 264, 6160),
    # tiles of 128 rows: the same
    ((128, 128, 1, False), 70, 10491, 304), ((128, 128, 1, False), 100, 19680, 144), ((128, 128, 1, False), 100, 20001, 144),
    ((128, 128, 2, False), 67, 6187, 7552), ((128, 128, 2, False), 69, 4752, 7312), ((128, 128, 4, False), 100, 2467, 10000), ((128, 128, 4, False), 1100, 264, 12880),
    # tiles of up to 240 rows, in two and four runs of K; several tiles, which start within a row block and may reach into a third one
    ((128, 240, 2, False), 150, 6517, 6064), ((128, 240, 2, False), 160, 6432, 6160), ((128, 240, 4, False), 200, 3107, 9856), ((128, 240, 4, False), 240, 2825, 10000),
    ((128, 240, 4, False), 400, 1544, 9104), ((128, 240, 4, False), 3700, 136, 12304),
    # pairs of CTAs; 192 rows to a tile: every second tile starts at row 64 of a row block
    ((256, 128, 1, False), 790, 15137, 448), ((256, 128, 1, False), 790, 15136, 448),
    ((256, 192, 1, False), 141, 14371, 800), ((256, 192, 1, False), 130, 13168, 688), ((256, 192, 1, False), 941, 14779, 144), ((256, 192, 1, False), 1341, 10304, 272),
    ((256, 256, 1, False), 218, 9583, 960), ((256, 256, 1, False), 198, 10032, 800), ((256, 256, 1, False), 395, 28319, 144), ((256, 256, 1, False), 414, 24064, 272),
]
# rows of each matrix, N, K; the last has more tiles than the GPU takes at once
ROUTED = [([64, 1, 0, 65, 30, 7, 128, 16], 264, 544), ([300, 0, 700, 257, 1000], 331, 528), ([300, 0, 700, 257, 1000], 1672, 272)]
