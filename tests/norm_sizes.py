"""Sizes that the tests share between the GPU, where the kernels run on them, and the CPU, where it is checked that they reach
every kernel."""

# weight gradient from a checkpoint: rows, in, out; out and in are no whole number of vectors, of tiles or of blocks of 32
WEIGHT_64x128 = [(16, 1030, 2051), (33, 2051, 1030), (70, 777, 2501), (97, 1501, 1503), (150, 2051, 1029), (20000, 300, 131), (3000, 513, 259)]
WEIGHT_128x256 = [(1, 4099, 4099), (33, 4099, 2051), (70, 2051, 4099), (97, 4097, 2049), (300, 4098, 2051), (40000, 1030, 515), (60000, 1025, 257)]

# maps whose groups fit a workgroup: pictures, pixels, channels, groups.  With few, several hundred and more than a thousand
# workgroups, since the number of pixels of a thread hangs on that.
RESIDENT = [
    (2, 4, 16, 4), (2, 49, 16, 4), (2, 100, 16, 4), (2, 169, 16, 4), (2, 300, 16, 4), (2, 600, 16, 4), (2, 841, 16, 4), (2, 1300, 16, 4),
    (2, 4000, 24, 3), (2, 169, 96, 8), (2, 3025, 64, 2), (16, 841, 16, 4), (37, 169, 384, 32), (64, 49, 130, 10), (64, 169, 128, 4),
    (64, 300, 128, 4), (64, 600, 128, 4), (64, 1300, 128, 4), (128, 49, 37, 37), (128, 500, 37, 37), (128, 841, 37, 37), (128, 2000, 40, 4),
    (256, 729, 256, 32), (300, 4, 16, 4), (300, 4, 256, 32), (300, 49, 256, 32), (300, 100, 24, 3), (300, 100, 256, 32), (300, 100, 384, 32),
    (300, 169, 130, 10), (300, 500, 16, 4), (300, 2000, 16, 4), (600, 49, 37, 37), (600, 49, 100, 5), (600, 100, 37, 37), (600, 169, 37, 37),
    (600, 169, 96, 32), (600, 300, 37, 37), (600, 500, 37, 37),
]
