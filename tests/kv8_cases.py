"""Calls of the attention over an 8-bit cache that take more than 64 steps a wave, and lists by every way
of cutting them up (test_kv8_cases.py holds them to that).  LONG is as in kv4_cases.py; LISTS: rows, the first one's
position, kv heads, query heads of each, entries of a list.  The sequences of LONG are one
stream, read at several places."""

LONG = {
    "128 tokens": ([1] * 128, [16000 - 3 * i for i in range(128)], 8, 4, None),
    "128 x 4 rows": ([4] * 128, [10000 - 5 * i for i in range(128)], 8, 4, None),
    "256 x 2 rows of a wide group": ([2] * 256, [9000 + 3 * i for i in range(256)], 8, 8, None),
    "300 x 7 rows": ([7] * 300, [9000 - i for i in range(300)], 8, 4, None),
    "130 x 20 rows": ([20] * 130, [10000 - 7 * i for i in range(130)], 8, 4, None),
    "30 x 300 rows": ([300] * 30, [9000 + 100 * i for i in range(30)], 8, 4, None),
    "a prompt of 16,384": ([16384], [0], 8, 4, None),
}

LISTS = {
    "a row, split": (1, 25000, 8, 4, 300),
    "a row, long": (1, 60000, 2, 4, 3000),
    "12 rows": (12, 9000, 8, 4, 64),
    "60 rows": (60, 9000, 8, 4, 40),
    "200 rows of a wide group": (200, 9000, 4, 16, 33),
    "300 rows of 41 heads": (60, 3000, 2, 41, 20),
    "500 rows of 129 blocks": (500, 9000, 8, 4, 129),
    "500 rows of 256 blocks": (500, 9000, 8, 4, 256),
    "500 rows of 300 blocks": (500, 9000, 8, 4, 300),
    "400 rows of 300 blocks, wide": (400, 9000, 8, 12, 300),
    "900 rows": (900, 2000, 8, 4, 17),
}


def sizes(rows, first, hkv, group, pages=None):
    return len(rows), sum(rows), max(rows), hkv * group, hkv, pages or (max(r + f for r, f in zip(rows, first)) + 15) // 16
