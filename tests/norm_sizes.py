"""Sizes that the tests share between the GPU, where the kernels run on them, and the CPU, where it is checked that they reach
every kernel."""

# weight gradient from a checkpoint: rows, in, out; out and in are no whole number of vectors, of tiles or of blocks of 32
WEIGHT_64x128 = [(16, 1030, 2051), (33, 2051, 1030), (70, 777, 2501), (97, 1501, 1503), (150, 2051, 1029), (20000, 300, 131), (3000, 513, 259)]
WEIGHT_128x256 = [(1, 4099, 4099), (33, 4099, 2051), (70, 2051, 4099), (97, 4097, 2049), (300, 4098, 2051), (40000, 1030, 515), (60000, 1025, 257)]
