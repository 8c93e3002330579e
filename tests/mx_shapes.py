"""Sizes of the tests of layers with 4-bit floating point weights, and which kernel each is for (held to it by test_mx_choices.py)."""

# few rows, or small matrices: outputs that end inside a tile, runs of columns that end inside one
SHAPES = [(1, 8, 32), (1, 250, 256), (2, 33, 96), (15, 64, 128), (16, 31, 160), (17, 100, 512), (31, 257, 288), (33, 64, 1056), (48, 130, 544), (64, 96, 2080),
          (65, 250, 320), (97, 256, 576), (128, 514, 256), (129, 300, 352), (200, 129, 1120), (255, 513, 64), (256, 256, 32), (257, 258, 608), (300, 700, 800),
          (16, 4100, 4128), (1, 16500, 2176), (2, 14000, 2176), (9, 20000, 544), (5, 8200, 2080), (3, 8000, 2208)]

# (batch, rows, cols, rows of x to a tile, whether the columns are in parts: with x in bf16, in 4 bits)
LARGE = [(700, 2050, 800, 64, (False, False)), (2100, 514, 2336, 64, (True, False)), (60, 250, 14336, 64, (True, True)), (300, 250, 14336, 64, (True, True)),
         (4000, 1030, 288, 128, (False, False)), (1300, 4100, 1056, 128, (False, False)), (9000, 1030, 160, 256, (False, False)),
         (2000, 4100, 288, 256, (False, False)), (3000, 8200, 160, 256, (False, False)), (2050, 4100, 2336, 256, (False, False))]

# (tokens, experts, top_k, hidden, inner)
LAYERS = [(1, 4, 1, 32, 32), (3, 8, 2, 96, 64), (20, 8, 4, 160, 96), (33, 16, 4, 512, 256), (70, 4, 2, 288, 544), (300, 8, 2, 128, 160), (150, 2, 2, 256, 288),
          (600, 4, 2, 64, 32), (40, 64, 8, 2080, 96)]
# and the rows of a tile
LARGE_LAYERS = [(400, 8, 2, 1056, 1056, 64), (3000, 2, 1, 544, 544, 64), (3000, 3, 2, 1056, 1056, 128), (6000, 2, 2, 1056, 160, 128), (12000, 2, 2, 288, 160, 256),
                (12000, 3, 3, 544, 544, 256)]
