"""Calls that between them are taken by every form of the kernels for scores of pages and for attention over picked ones.

Attention: blocks of 2, 4 and 8 waves, up to eight query heads to a KV head and more, rows of a sequence of their own and several, lists
whole and split, both head dimensions.  name: n_q, n_kv, head_dim, contexts, rows (of each sequence), pages of a list.
"""
_SOME, _ROWS = [1500, 1290, 64, 700, 5, 1411], [4, 3, 1, 9, 2, 1]

CALLS = {
    # eight waves: lists of more than 16 pages that are not split, up to 256 blocks
    "eight-wide-128": (16, 1, 128, _SOME, None, 20),
    "eight-wide-64": (12, 1, 64, _SOME, None, 17),
    "eight-wide-128-rows": (16, 1, 128, _SOME, _ROWS, 31),
    "eight-wide-64-rows": (9, 1, 64, _SOME, _ROWS, 24),
    "eight-17-heads": (17, 1, 128, _SOME, None, 23),            # a second block of a row and KV head has one of them
    "eight-17-heads-rows": (34, 2, 64, _SOME, _ROWS, 18),
    "eight-40-heads": (40, 1, 128, _SOME, _ROWS, 19),
    "eight-wide-many": (16, 1, 128, [1500, 1290] + [130] * 148, None, 20),
    "eight-narrow-128": (8, 1, 128, _SOME, None, 20),
    "eight-narrow-64": (10, 2, 64, _SOME, None, 21),
    "eight-narrow-128-rows": (7, 1, 128, _SOME, _ROWS, 30),
    "eight-narrow-64-rows": (3, 3, 64, _SOME, _ROWS, 17),
    # four: shorter ones
    "four-wide-128": (12, 1, 128, _SOME, None, 16),
    "four-wide-64": (16, 1, 64, _SOME, None, 5),
    "four-wide-128-rows": (17, 1, 128, _SOME, _ROWS, 9),
    "four-wide-64-rows": (18, 2, 64, _SOME, _ROWS, 16),
    "four-narrow-128": (28, 4, 128, _SOME, None, 16),
    "four-narrow-64": (8, 1, 64, _SOME, None, 3),
    "four-narrow-128-rows": (2, 2, 128, _SOME, _ROWS, 16),
    "four-narrow-64-rows": (14, 2, 64, _SOME, _ROWS, 7),
    # two: 512 blocks and more, of rows that may share pages
    "two-wide-128": (72, 8, 128, [700, 130], [40, 24], 6),
    "two-wide-64": (128, 8, 64, [700, 130], [40, 24], 7),
    "two-narrow-128": (56, 8, 128, [700, 130], [40, 24], 6),
    "two-narrow-64": (16, 8, 64, [700, 130], [40, 24], 18),
    # split: up to 128 blocks, lists of 32 pages and more
    "split-wide-128": (16, 1, 128, [2900, 130], None, 40),
    "split-wide-64": (40, 2, 64, [2900, 130], None, 33),
    "split-wide-128-rows": (17, 1, 128, [2900, 130], [3, 2], 45),
    "split-wide-64-rows": (9, 1, 64, [2900, 130], [3, 2], 32),
    "split-narrow-128": (28, 4, 128, [2900, 130], None, 41),
    "split-narrow-64": (4, 2, 64, [2900, 130], None, 32),
    "split-narrow-128-rows": (8, 1, 128, [2900, 130], [3, 2], 34),
    "split-narrow-64-rows": (14, 2, 64, [2900, 130], [3, 2], 45),
}

# The same without the length of a list: as many pages as the longest context has, all listed.  Eight waves, for where the softmax is hard.
HARD = {
    "eight-wide-128": (16, 1, 128, [1400, 700, 130, 1], [1, 1, 1, 1]),
    "eight-wide-64": (12, 1, 64, [1400, 1100, 65], [1, 1, 1]),
    "eight-wide-128-rows": (17, 1, 128, [1300, 700, 64], [2, 5, 1]),
    "eight-wide-64-rows": (9, 1, 64, [1100, 130, 30], [3, 2, 7]),
    "eight-narrow-128-rows": (7, 1, 128, [1400, 130], [9, 2]),
}

# Scores: a row of each sequence, whose wave has 16 pages or 64, and up to 16 query heads to a KV head or more; rows that share ranges,
# of 32 pages to a wave or 64, and every way that the heads of a row lie in a product's rows.
# name: n_q, n_kv, head_dim, contexts, rows, rows and columns of the call (the sequences' rows come first)
_LONG, _SHORT = [1500, 4097, 64, 1, 700, 3000], [900, 40, 0, 3, 64, 700, 1]
_MANY = [130, 40, 0, 3, 1, 65, 0]
SCORES = {
    "walk-16-128": (28, 4, 128, _LONG, None, 6, 65),
    "walk-16-64": (14, 2, 64, _LONG, None, 6, 70),
    "walk-64-128": (28, 4, 128, _LONG, None, 700, 65),
    "walk-64-64": (14, 2, 64, _LONG, None, 700, 100),
    "walk-heads-128": (34, 2, 128, _LONG, None, 6, 65),
    "walk-heads-64": (40, 1, 64, _LONG, None, 2000, 65),
    "rows-32-128": (28, 4, 128, _SHORT, _MANY, 239, 15),
    "rows-32-64": (14, 2, 64, _SHORT, _MANY, 1700, 15),
    "rows-64-128": (28, 4, 128, _SHORT, _MANY, 3000, 300),
    "rows-64-64": (14, 2, 64, _SHORT, _MANY, 3000, 1000),
    "rows-64-1-head": (2, 2, 64, _SHORT, _MANY, 3000, 1000),
    "rows-64-2-heads": (4, 2, 64, _SHORT, _MANY, 3000, 1000),
    "rows-64-3-heads": (3, 1, 128, _SHORT, _MANY, 4000, 900),
    "rows-64-5-heads": (10, 2, 64, _SHORT, _MANY, 3000, 1000),
    "rows-64-12-heads": (12, 1, 128, _SHORT, _MANY, 4000, 900),
    "rows-64-40-heads": (40, 1, 64, _SHORT, _MANY, 4000, 900),
}
