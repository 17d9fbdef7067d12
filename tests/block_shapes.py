"""Shapes (rows, d, ffn, out) at which the gated feed-forward block's products are compared with the oracle, by the path
that they are there for.  Which tile a product takes follows a rule on its sizes: when that rule changes, shapes are added
here until every tile is reached again."""

# Products in the tiles that go straight from memory into LDS: with rows, columns and summed elements that are no whole
# tiles or steps, and more steps than the tile has on their way
TILES = [(341, 344, 32, 336), (385, 264, 4864, 392), (769, 72, 328, 2616), (3281, 40, 200, 1184), (193, 40, 1568, 2656),
         (4101, 32, 960, 216), (193, 784, 4800, 56), (841, 352, 4680, 32), (400, 1720, 4624, 112), (360, 32, 3520, 2312),
         (3665, 40, 376, 2288), (2307, 56, 1888, 2216), (1793, 32, 4488, 360), (1497, 1264, 3296, 40), (168, 32, 336, 32),
         (328, 2336, 904, 56)]
# The gradient by x in those tiles: a sum of two terms, of which the second begins while loads are on their way
TWO_TERMS = [(128, 40, 320, 32), (264, 136, 192, 64), (648, 2992, 320, 96), (1184, 3216, 192, 256), (3336, 2344, 192, 40),
             (1624, 2504, 768, 128), (2568, 1544, 1088, 72)]
# Operands that go through registers: widths that are no whole pieces of eight, tiles of 64 and of 128, sums long enough
# for the steady loop of either
REGISTERS = [(17, 771, 257, 130), (300, 771, 1030, 771), (2051, 331, 2049, 2053), (2049, 2051, 519, 131), (531, 2053, 2051, 37)]
# Up to 16 rows, where the weights are streamed once: sums that pass one round of the workgroup's waves
TOKENS = [(1, 2048, 5632, 2048), (2, 515, 2049, 33), (5, 1100, 4103, 70), (13, 4096, 2112, 50), (16, 2600, 6200, 17)]
