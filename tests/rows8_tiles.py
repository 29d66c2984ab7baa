"""Sizes that every tile of the products and of the weight gradients is chosen for, each ending inside a tile: what the choice has to be
(tests/test_rows8_shapes.py), and what is computed with it (tests/test_gpu_rows8_tiles.py)."""

# (rows, cols, outs): (tokens and channels of a tile, whether k is cut into pieces); tiles of 0 x 0 are the kernel for few tokens
PRODUCTS = {
    (16, 130, 1000): (0, 0, False), (32, 272, 700): (0, 0, False),
    (17, 131_000, 270): (64, 64, True), (40, 77, 333): (64, 64, False), (40, 4100, 700): (64, 64, True),
    (200, 208, 4100): (64, 128, False),
    (500, 77, 4100): (128, 128, False), (128, 8192, 8190): (128, 128, True), (500, 16_400, 2000): (128, 128, True), (300, 20_003, 520): (128, 128, True),
    (777, 208, 5000): (256, 128, False),
    (3585, 77, 3401): (256, 256, False), (3600, 400, 3700): (256, 256, False),
}

# (workers, rows of each, cols, outs): (input and output channels of a tile, whether the sum is cut into pieces), for any types and scales
WEIGHTS = {
    (2, 33, 130, 70): (64, False), (1, 9000, 130, 257): (64, True),
    (3, 300, 1800, 1810): (128, False), (2, 9000, 1000, 1032): (128, True),
    (1, 2040, 3600, 3700): (256, False), (2, 2100, 2600, 2576): (256, False),
}
