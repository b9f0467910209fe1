"""Sizes that reach every kernel of the 8-bit products and weight gradients,
tiles not divided, all in parts, and those of the last round in parts.

Each entry: (rows, columns, long axis) -> tile rows, tile columns, whole tiles,
parts, as planned on 256 CUs with the default workspace.  Rows and columns are
no multiples of the tile's; long axes are one block or slice, a few, and many
with a remainder.  tests/test_linear_choice.py holds the plans, without a GPU;
tests/test_gpu_linear_tiles.py runs the sizes.
"""

WORKSPACE = 64 << 20

# Products with bf16 results.
PRODUCT = {
    (17, 129, 100): (64, 128, 0, 1),
    (257, 383, 333): (64, 128, 0, 1),
    (63, 65, 2000): (64, 128, 0, 4),
    (65, 127, 8000): (64, 128, 0, 7),
    (8193, 129, 8000): (64, 128, 256, 7),
    (8191, 257, 129): (128, 128, 0, 1),
    (4097, 129, 8000): (128, 128, 0, 3),
    (777, 5000, 4096): (128, 128, 256, 4),
    (2900, 2049, 129): (128, 256, 0, 1),
    (4095, 2047, 2000): (128, 256, 0, 1),
    (777, 2560, 14336): (128, 256, 0, 3),
    (4097, 4000, 1333): (128, 256, 512, 2),
    (4097, 3000, 100): (256, 256, 0, 1),
    (4095, 4001, 640): (256, 256, 0, 1),
    (5000, 3333, 2000): (256, 256, 256, 2),
}

# Products with fp32 results, or fp32 sums.
EXACT = {
    (17, 129, 100): (64, 128, 0, 1),
    (257, 383, 333): (64, 128, 0, 1),
    (63, 65, 2000): (64, 128, 0, 4),
    (777, 5000, 1000): (64, 128, 512, 4),
    (6143, 257, 300): (128, 128, 0, 1),
    (4097, 129, 8000): (128, 128, 0, 3),
    (4095, 1025, 1333): (128, 128, 256, 2),
}

# Weight gradients (rows and columns of dW, tokens).
GRAD = {
    (63, 65, 1): (64, 64, 0, 1),
    (257, 383, 333): (64, 64, 0, 1),
    (63, 65, 2049): (64, 64, 0, 4),
    (65, 8193, 2049): (64, 64, 256, 4),
    (8193, 65, 1): (128, 128, 0, 1),
    (65, 8193, 33): (128, 128, 0, 1),
    (8193, 127, 65): (128, 128, 0, 1),
    (65, 4097, 16000): (128, 128, 0, 7),
    (2047, 2049, 600): (128, 128, 256, 3),
    (513, 7000, 31): (256, 256, 0, 1),
    (7000, 513, 33): (256, 256, 0, 1),
    (4097, 1023, 97): (256, 256, 0, 1),
    (4097, 1000, 4097): (256, 256, 0, 3),
    (2047, 8193, 300): (256, 256, 256, 2),
    (4095, 4097, 600): (256, 256, 256, 2),
}
