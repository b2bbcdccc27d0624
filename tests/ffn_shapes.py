"""Shapes (particles, rows, width, hidden) of the gated feed-forward block's tests, by what they lead the kernels to: test_ffn_rules.py says what that is and
sees to it that they do; the GPU tests run them."""

# Tiles, of every kind in every product, with three whole steps of 32 columns at least and a part of one in every part of the columns.
TILES = [(26, 68, 102, 1_101), (39, 34, 101, 1_118), (32, 35, 103, 402), (16, 2_626, 130, 100), (33, 201, 132, 1_396), (27, 386, 135, 100), (34, 35, 196, 520),
         (1, 68, 97, 101), (1, 66, 101, 264), (21, 1_414, 98, 131), (35, 1_257, 99, 99), (1, 33, 97, 102), (37, 110, 513, 106), (5, 5_520, 131, 104),
         (10, 102, 134, 1_221), (2, 5_372, 130, 963), (39, 132, 203, 100), (11, 1_386, 99, 105), (32, 100, 101, 293), (1, 2_119, 99, 1_351), (1, 103, 106, 100),
         (1, 270, 97, 103), (1, 101, 101, 136), (1, 264, 103, 129),
         # whole steps only
         (2, 128, 128, 160), (8, 256, 256, 384)]

# Few rows, with columns enough for every wave to work on several steps, the last one a part of one.
THIN = [(2, 5, 545, 683), (1, 16, 577, 775), (3, 1, 600, 700), (2, 17, 700, 557), (1, 32, 570, 641), (1, 50, 600, 553), (1, 64, 555, 560), (1, 9, 768, 576)]

# Few rows, backward: dx by a wave for every weight or in tiles, with the parameters' gradients and without them.
DX_OF_FEW_ROWS = [(3, 7, 100, 203), (2, 16, 16, 2_000), (5, 9, 190, 301), (2, 13, 70, 1_501), (2, 31, 61, 333), (1, 20, 15, 1_700), (40, 25, 129, 321), (1, 32, 90, 2_003),
                  (64, 3, 130, 260), (12, 1, 353, 1_001)]
