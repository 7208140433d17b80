"""Inputs of paged attention by the path that their plan takes: tests/test_paged_plan.py holds them to it (no GPU), and
tests/test_gpu_paged_paths.py runs them.

dtype, Dh, the shape of a block, how a row's ranges of keys are joined ("one": there is one; "last": by the block that finishes
last; "later": in a launch of their own), whether blocks look at all items' lengths, form, B, H, Hkv, M, S, page size."""

# what the blocks of a row tile leave in the handle for each other is back to zero behind the call
JOINED_BY_THE_LAST_BLOCK = [
    ("bf16", 64, 0, "last", 0, "chunk", 3, 3, 3, 1, 6807, 32),
    ("bf16", 64, 0, "last", 1, "tree", 7, 3, 3, 1, 5909, 64),
    ("bf16", 64, 1, "last", 0, "tree", 3, 4, 4, 1, 5364, 32),
    ("bf16", 64, 1, "last", 1, "chunk", 11, 2, 2, 1, 5861, 64),
    ("bf16", 64, 2, "last", 0, "tree", 1, 96, 24, 61, 3070, 64),
    ("bf16", 64, 2, "last", 1, "chunk", 34, 1, 1, 33, 1479, 128),
    ("bf16", 128, 0, "last", 0, "tree", 3, 3, 3, 1, 5516, 256),
    ("bf16", 128, 0, "last", 1, "chunk", 2, 8, 8, 1, 6163, 16),
    ("bf16", 128, 1, "last", 0, "chunk", 10, 1, 1, 1, 6704, 256),
    ("bf16", 128, 1, "last", 1, "tree", 8, 2, 2, 1, 6781, 16),
    ("bf16", 128, 2, "last", 0, "chunk", 1, 32, 16, 130, 1659, 16),
    ("bf16", 128, 2, "last", 1, "tree", 17, 12, 4, 16, 1551, 32),
    ("bf16", 128, 3, "last", 0, "chunk", 1, 96, 24, 199, 2042, 32),
    ("bf16", 128, 3, "last", 1, "tree", 18, 6, 3, 129, 1918, 64),
    ("bf16", 128, 4, "last", 1, "chunk", 5, 32, 16, 33, 3546, 64),
    ("f32", 64, 0, "last", 0, "tree", 6, 2, 2, 1, 5408, 64),
    ("f32", 64, 0, "last", 1, "chunk", 9, 3, 3, 1, 4901, 128),
    ("f32", 64, 1, "last", 0, "chunk", 9, 9, 3, 6, 1187, 64),
    ("f32", 64, 1, "last", 1, "tree", 6, 2, 2, 129, 883, 128),
    ("f32", 128, 0, "last", 0, "chunk", 6, 1, 1, 1, 5385, 128),
    ("f32", 128, 0, "last", 1, "tree", 6, 2, 2, 1, 5425, 256),
    ("f32", 128, 1, "last", 0, "chunk", 2, 24, 24, 17, 748, 256),
    ("f32", 128, 1, "last", 1, "tree", 5, 2, 2, 129, 1138, 16),
]

# one range: which item a block takes goes by the lengths
LONGEST_FIRST = [
    ("bf16", 64, 0, "one", 1, "chunk", 11, 24, 24, 1, 929, 16),
    ("bf16", 64, 1, "one", 1, "chunk", 17, 24, 8, 11, 1858, 32),
    ("bf16", 64, 2, "one", 1, "chunk", 35, 24, 8, 11, 898, 64),
    ("bf16", 64, 3, "one", 1, "chunk", 23, 32, 16, 36, 471, 256),
    ("bf16", 64, 4, "one", 1, "chunk", 34, 32, 8, 25, 650, 128),
    ("bf16", 128, 1, "one", 1, "tree", 30, 3, 3, 129, 1663, 256),
    ("bf16", 128, 2, "one", 1, "tree", 34, 24, 8, 16, 886, 16),
    ("bf16", 128, 3, "one", 1, "tree", 22, 8, 8, 129, 265, 32),
    ("bf16", 128, 4, "one", 1, "chunk", 38, 3, 3, 257, 214, 32),
    ("f32", 64, 0, "one", 1, "tree", 34, 12, 4, 16, 1848, 32),
    ("f32", 64, 1, "one", 1, "tree", 29, 3, 3, 129, 753, 64),
    ("f32", 128, 0, "one", 1, "tree", 43, 9, 3, 16, 903, 128),
    ("f32", 128, 1, "one", 1, "tree", 11, 8, 8, 129, 806, 256),
]

# every other shape with every way of joining that it is chosen with
OTHERS = [
    ("bf16", 64, 0, "later", 0, "chunk", 3, 6, 3, 7, 6972, 128),
    ("bf16", 64, 0, "one", 0, "tree", 17, 16, 16, 1, 258, 256),
    ("bf16", 64, 1, "later", 0, "tree", 5, 2, 2, 16, 6640, 128),
    ("bf16", 64, 1, "later", 1, "chunk", 5, 4, 4, 29, 6383, 256),
    ("bf16", 64, 1, "one", 0, "tree", 1, 1, 1, 1, 228, 16),
    ("bf16", 64, 2, "later", 0, "tree", 5, 3, 1, 16, 6507, 256),
    ("bf16", 64, 2, "later", 1, "chunk", 4, 9, 3, 11, 5554, 16),
    ("bf16", 64, 2, "one", 0, "tree", 43, 9, 3, 16, 220, 32),
    ("bf16", 64, 3, "one", 0, "tree", 28, 8, 8, 129, 240, 128),
    ("bf16", 64, 4, "later", 0, "chunk", 2, 4, 2, 34, 5471, 16),
    ("bf16", 64, 4, "later", 1, "chunk", 4, 4, 2, 33, 5592, 32),
    ("bf16", 64, 4, "one", 0, "tree", 27, 12, 4, 61, 200, 64),
    ("bf16", 128, 0, "later", 0, "tree", 4, 2, 2, 16, 6142, 32),
    ("bf16", 128, 0, "later", 1, "chunk", 2, 8, 8, 11, 6180, 64),
    ("bf16", 128, 0, "one", 0, "tree", 30, 8, 8, 1, 210, 128),
    ("bf16", 128, 1, "later", 0, "chunk", 10, 1, 1, 8, 6625, 32),
    ("bf16", 128, 1, "later", 1, "tree", 2, 8, 8, 16, 6776, 64),
    ("bf16", 128, 1, "one", 0, "chunk", 1, 1, 1, 1, 330, 128),
    ("bf16", 128, 2, "later", 0, "chunk", 7, 3, 1, 11, 4942, 64),
    ("bf16", 128, 2, "later", 1, "tree", 3, 12, 4, 16, 5242, 128),
    ("bf16", 128, 2, "one", 0, "chunk", 34, 16, 4, 9, 222, 256),
    ("bf16", 128, 3, "later", 0, "chunk", 1, 96, 24, 18, 6267, 128),
    ("bf16", 128, 3, "later", 1, "tree", 15, 6, 3, 61, 4062, 256),
    ("bf16", 128, 3, "one", 0, "chunk", 11, 72, 24, 23, 291, 16),
    ("bf16", 128, 4, "later", 0, "tree", 1, 48, 24, 61, 3540, 128),
    ("bf16", 128, 4, "later", 1, "chunk", 4, 8, 4, 34, 2046, 256),
    ("bf16", 128, 4, "one", 0, "tree", 44, 2, 2, 129, 203, 16),
    ("f32", 64, 0, "later", 0, "tree", 4, 3, 3, 16, 6667, 256),
    ("f32", 64, 0, "one", 0, "chunk", 1, 4, 1, 1, 243, 16),
    ("f32", 64, 1, "later", 0, "chunk", 2, 9, 3, 6, 5637, 256),
    ("f32", 64, 1, "later", 1, "tree", 11, 1, 1, 61, 3841, 16),
    ("f32", 64, 1, "one", 0, "chunk", 45, 3, 3, 17, 100, 32),
    ("f32", 128, 0, "later", 0, "chunk", 5, 4, 1, 1, 6733, 16),
    ("f32", 128, 0, "later", 1, "tree", 2, 1, 1, 129, 3491, 32),
    ("f32", 128, 0, "one", 0, "chunk", 1, 1, 1, 1, 114, 64),
    ("f32", 128, 1, "later", 0, "chunk", 1, 8, 8, 17, 6189, 32),
    ("f32", 128, 1, "later", 1, "tree", 6, 1, 1, 61, 5332, 64),
    ("f32", 128, 1, "one", 0, "chunk", 33, 12, 4, 6, 197, 128),
]

# lengths of batches of single tokens, 8 heads over 2 of 128
TOKENS = [[3000], [1500, 2900]]

PATHS = JOINED_BY_THE_LAST_BLOCK + LONGEST_FIRST + OTHERS
