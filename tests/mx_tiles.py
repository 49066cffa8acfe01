"""Shapes that between them take every kernel of the MXFP4 products: ``(m, rows,
n)`` by kind of activations and number of matrices, the kernel's place first.

Rows and tokens end inside a tile, n inside a stage, and n has more stages than
any kernel has in flight.
"""

HALF = {
    False: {-1: (3, 1001, 3456), 0: (9, 333, 3456), 1: (5, 9002, 3456), 2: (7, 17001, 1152), 3: (4101, 61, 1152),
            4: (19, 16401, 1152), 5: (33, 16390, 1152), 6: (59, 16404, 1152), 7: (3, 33001, 1152),
            8: (65, 33002, 1152)},
    True: {-1: (4, 501, 3456), 0: (10, 211, 3456), 1: (6, 4101, 3456), 2: (3, 9001, 1152), 3: (4101, 31, 1152),
           4: (21, 9003, 1152), 5: (37, 9002, 1152), 6: (61, 9001, 1152), 7: (5, 16403, 1152), 8: (66, 16390, 1152)},
}
MX = {
    False: {-1: (2, 999, 3456), 0: (11, 345, 3456), 1: (6, 9001, 3456), 2: (4101, 61, 1152), 3: (35, 9002, 1152),
            4: (9, 16390, 1152), 5: (67, 16401, 1152), 6: (131, 16403, 1152), 7: (257, 25001, 1152)},
    True: {-1: (1, 777, 3456), 0: (13, 222, 3456), 1: (7, 4103, 3456), 2: (19, 4102, 1152), 3: (41, 4101, 1152),
           4: (11, 9001, 1152), 5: (66, 9002, 1152), 6: (67, 16401, 1152), 7: (65, 25002, 1152)},
}
# n in parts over blocks
SPLIT = [(10, 100, 16384), (40, 64, 16640), (300, 64, 16512)]
EVERY = [(act, gated, tile, shape) for act, table in (("f16", HALF), ("bf16", HALF), ("a4", MX)) for gated in table
         for tile, shape in table[gated].items()]
