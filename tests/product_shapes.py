"""Products in every tile, in slices of k and in one piece, for the tests on the GPU (their
results) and on the host (which kernel they run)."""

# (m, n, k): tile of a bf16 result, of one under a mask, of a float32 result, of one that is added to; each in
# slices of k, the last one short; rows and columns that the tiles cut, or (n a multiple of four) whole vectors
SLICED = {
    (69, 2883, 11031): (128, 128, 128, 128),
    (2845, 67, 6703): (64, 64, 128, 128),
    (72, 2884, 11031): (128, 128, 128, 128),
    (899, 4371, 9765): (256, 256, 256, 256),
    (990, 4668, 10667): (256, 256, 256, 256),
    (300, 301, 6001): (64, 64, 64, 64),
}
KINDS = ("bf16", "masked", "float32", "added")

# (m, n, k): tile of all four, in one piece
WHOLE = {(65, 127, 129): 64, (2001, 2003, 1000): 128, (4090, 4081, 6001): 256}
