"""Attention calls whose partial results are joined over many parts: (query heads, kv heads, head dimension, new tokens, cached tokens,
parts that the longest slot is cut into at least, rows joined by a workgroup of their own)."""
JOINS = [
    (4, 1, 128, [1], [40000], 65, True),                     # more than 8 parts to each of the 8 groups that take them side by side
    (4, 2, 64, [1], [70001], 129, True),                     # ... of 16 groups, heads of 64
    (4, 2, 64, [1], [9000], 9, True),                        # fewer parts than groups
    (4, 1, 128, [1] * 70, [9 * i for i in range(69)] + [30011], 9, False),
    (8, 1, 64, [4, 1] * 32, [3 + i for i in range(63)] + [25000], 9, False),
    (24, 1, 64, [17], [20000], 9, True),                     # parts of the tile form
    (24, 1, 128, [21], [11003], 9, True),
    (8, 1, 128, [70], [12000], 9, False),
    (8, 2, 64, [100, 33], [17, 14500], 9, False),
]
