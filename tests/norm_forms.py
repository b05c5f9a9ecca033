"""Sizes of layer norm and of its backward pass that run every form of their kernels: lanes of a row, eights that a lane holds."""

# forward, few rows: a workgroup or a part of one to a row
FEW = [(3, 7), (5, 64), (4, 128), (6, 129), (5, 200), (5, 300), (5, 500), (6, 600), (9, 641), (5, 1001), (5, 1025), (5, 1801), (5, 2049), (5, 2561), (5, 3001), (5, 5121), (5, 8001),
       (5, 9001), (5, 10241), (5, 12001), (3, 14001), (2, 20480), (2, 20481), (300, 1025), (600, 5121)]
# forward, many rows: a wavefront or a part of one to a row
MANY_ROWS = 2053
MANY = [3, 8, 33, 65, 71, 129, 136, 193, 257, 321, 513, 641, 1001, 1025, 1033, 1543, 2049, 2561, 3585, 4099, 5121, 5130, 7171, 8199, 9223, 10300]
MANY_BF16 = [12289, 14337, 15361, 16391]
# backward
BACK = [(9, 3), (9, 65), (30, 129), (9, 136), (300, 200), (9, 257), (9, 300), (20, 500), (30, 521), (300, 647), (9, 1001), (7, 1033), (300, 1543), (9, 2049), (7, 2061), (40, 2567), (5, 3001),
        (9, 5121), (5, 8001), (40, 9001), (300, 10241), (7, 12001), (6, 14001), (5, 20480), (5, 20481), (2100, 65), (3000, 193), (600, 1025)]


def norm_calls(bf16):
    sizes = FEW + [(MANY_ROWS, K) for K in MANY + (MANY_BF16 if bf16 else [])]
    return [("norm", N, K, bf16, drop) for N, K in sizes for drop in (0, 1)]


def back_calls(bf16):
    return [("back", N, K, bf16, drop, *asked) for N, K in BACK for drop in (0, 1) for asked in ((1, 1), (1, 0), (0, 1))]
