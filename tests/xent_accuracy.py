"""How far a softmax cross entropy of packed operands may be from 64 bits, by the size that its rounding errors have on average, which says much less than the worst
case of long sums does, and which kernels a few sizes are there for."""
import numpy as np

# rows, columns, classes, bfloat16, edges of the scores' tiles and of the gradients' (x: with a joined block of up to 32 rows), the gradients' sums cut into parts
CASES = [
    (1055, 271, 1659, False, "64", "64", False), (3407, 555, 203, False, "64", "64", True), (1000, 1025, 1000, False, "64", "128", False),
    (1911, 1641, 230, False, "64", "128", True), (1989, 599, 2641, False, "128", "128", False), (2119, 3687, 1052, False, "128", "256", False),
    (1545, 3339, 2112, False, "128", "256x", False), (3219, 1433, 3434, False, "256", "256", False), (6720, 363, 3121, False, "256", "256", True),
    (4062, 538, 2576, False, "256x", "256x", True),
    (1483, 512, 650, True, "64", "64", False), (4305, 434, 176, True, "64", "64", True), (676, 1420, 1157, True, "64", "128", False),
    (2163, 1545, 208, True, "64", "128", True), (2426, 537, 880, True, "128", "64", False), (1875, 1820, 2333, True, "128", "256x", False),
    (9000, 4000, 300, True, "128", "256", True), (2229, 2293, 2723, True, "256", "256", False), (942, 980, 5618, True, "256", "256", True),
    (661, 532, 8728, True, "256x", "256x", True),
]

# The error of a result of n products, relative to all results' size in the mean square. Operands and G of 22 bits: 2^-23 / sqrt(3) each, products of pairs of terms left
# out: 2^-24; together below 2^-21.5. Sums in 32 bits, rounded once for 16 products: n / 16 roundings of 2^-25 of a partial sum, whose size grows
# with the square root of its length: 2^-25 sqrt(n / 32), for 9000 products 2^-21; three terms of each product: below 2^-20. Together below 2^-19; twice that is
# allowed. (One operand of 11 bits: 2^-12 / sqrt(3) = 2^-12.8, of the losses, of which the scores are a fifth, 2^-15.)
MEAN = 2.0 ** -18
# A single result, relative to the root of the sum of its products' squares: sixteen times that mean.
SINGLE = 2.0 ** -14
# Results of bfloat16: numbers that lie near the middle of two are rounded to the other one than the exact result is. With an error e before, a share e / d of numbers
# whose neighbours lie d apart is off by d: in the mean square d e, and d is at most 2^-7 of the number.
MEAN_BF16 = (2.0 ** -7 * MEAN) ** 0.5


def mean_error(have, want):
    have, want = np.asarray(have, dtype=np.float64), np.asarray(want, dtype=np.float64)
    return float(np.sqrt(((have - want) ** 2).sum() / (want ** 2).sum()))
