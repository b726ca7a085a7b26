"""Sizes (rows, d_in, d_out) of the product of operands in 8 bits that tests have for the sake of one kernel, and what the plan has to make of them: the kernel, whether k is
split, and whether rows of these lengths side by side are laid out again.  A rule that moves one of them fails the CPU test of the plans, not only
the subject of a GPU test in silence."""
FRAGMENTS, SMALL, SMALL2, DIRECT, LARGE = range(5)

# tiles loaded into LDS by 32-bit offsets from the tile's first row, rows up to 2^23 - 16 bytes apart: sums split and in one, columns with a part of an eight, either operand
FAR = {(264, 32784, 264): (DIRECT, True, False), (264, 65552, 262): (DIRECT, True, False), (1500, 2048, 1504): (DIRECT, False, False),
       (59200, 1024, 256): (LARGE, False, False), (256, 1024, 59200): (LARGE, False, False)}
# operands in whole pieces of 16 bytes but for where they start or how far apart their rows are
ANYWHERE = {(2100, 1040, 2048): (DIRECT, False, False), (4096, 1024, 4096): (LARGE, False, False)}
# y over the residual: 128 x 128 in one sum, whole eights and a part of one, k that ends inside a tile
OVER = {(2900, 1040, 2050): (DIRECT, False, False), (1500, 2048, 1504): (DIRECT, False, False)}
# every kernel and its edges
KINDS = {(16, 512, 4000): (FRAGMENTS, False, False), (33, 512, 2000): (FRAGMENTS, False, False), (100, 640, 1250): (FRAGMENTS, False, False), (60, 1500, 8100): (SMALL2, True, False),
         (1000, 272, 1000): (FRAGMENTS, False, False), (500, 1027, 900): (SMALL2, True, False), (300, 3001, 200): (SMALL2, True, False), (2100, 4001, 2050): (DIRECT, False, True),
         (200, 4112, 4096): (DIRECT, True, False), (3900, 1088, 4090): (LARGE, False, False), (25000, 704, 5): (SMALL2, False, False), (60000, 1024, 5): (SMALL, False, False),
         (60000, 1024, 69): (DIRECT, False, False), (40000, 1024, 135): (DIRECT, False, False), (4000, 1001, 1000): (DIRECT, False, True), (8190, 1023, 2048): (LARGE, False, True),
         (1999, 2050, 2001): (DIRECT, False, True), (20000, 33, 2000): (DIRECT, False, True), (20000, 17, 2003): (SMALL, False, False)}
