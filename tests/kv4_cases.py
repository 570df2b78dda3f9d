"""Calls of the attention over a 4-bit cache that between them take every kernel and way of
cutting it up (test_kv_plan.py holds them to that): rows and first positions of the
sequences, kv heads, query heads of each, and the page table's width where it is not the longest
sequence's."""

CASES = {
    "a token": ([1], [299], 8, 4, None),
    "100 tokens": ([1] * 100, [3 * i for i in range(100)], 8, 4, None),
    "a token, several splits": ([1], [2999], 8, 4, None),
    "a token, many splits": ([1], [33000], 8, 4, None),
    "tokens of a wide group": ([1, 1, 1], [40, 700, 3], 2, 16, None),
    "3 rows each": ([3] * 90, [60 + i for i in range(90)], 8, 4, None),
    "3 rows": ([3], [300], 8, 4, None),
    "3 rows, several splits": ([3], [3001], 8, 4, None),
    "3 rows, many splits": ([3], [40005], 8, 4, None),
    "a prompt of 40": ([40], [0], 8, 4, None),
    "64 rows, splits": ([64], [3005], 8, 4, None),
    "8 x 64 rows": ([64, 61, 64, 1, 60, 64, 33, 64], [1000 + i for i in range(8)], 8, 4, None),
    "4 x 30 rows, splits": ([30, 29, 30, 17], [8000, 8001, 100, 7999], 8, 4, None),
    "a prompt of 1,999": ([1999], [0], 8, 4, None),
    "ragged turns, splits": ([90, 150, 211], [3007, 5000, 7010], 8, 4, None),
    "prompt rows in a wide table, splits": ([128], [0], 8, 4, 8192),
}


def sizes(case):
    rows, first, hkv, group, pages = CASES[case]
    pages = pages or max(r + f + 15 for r, f in zip(rows, first)) // 16
    return len(rows), sum(rows), max(rows), hkv * group, hkv, pages
