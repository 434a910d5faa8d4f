"""Steps of the attention that reach each of its kernels, for the tests that check
the choice (CPU) and the results (GPU).

(head_dim, page, key heads, group, lengths, new rows, kernel without the head size,
the joining kernel or None): sequences of about the largest length, one of them short
or without rows where there are several."""

ROWS, TILE, JOIN = "kv_attention_rows_kernel<%d,", "kv_attention_tile_kernel<%d,", "kv_attention_join_kernel<%d,"

EVERY = [
    # 16 rows: eight waves, four, in up to eight and in more pieces
    *[(d, 32, 2, 3, [100, 33], [1, 2], ROWS + "1,8,false>", None) for d in (64, 128, 256)],
    (64, 16, 1, 3, [100, 1, 0, 77] * 12, [1, 1, 0, 2] * 12, ROWS + "1,4,false>", None),
    (128, 32, 32, 2, [100, 65], [1, 1], ROWS + "1,4,false>", None),
    (256, 32, 16, 2, [100, 65], [1, 1], ROWS + "1,4,false>", None),
    (64, 64, 32, 4, [5000, 700], [1, 1], ROWS + "1,4,true>", JOIN + "1,1>"),
    (128, 32, 16, 3, [5000, 1400], [1, 1], ROWS + "1,4,true>", JOIN + "1,1>"),
    (256, 16, 1, 5, [600], [2], ROWS + "1,4,true>", JOIN + "1,1>"),
    *[(d, 32, 1, 4, [6000, 900], [1, 2], ROWS + "1,4,true>", JOIN + "1,4>") for d in (64, 128, 256)],
    # 32 rows
    *[(d, 16, 2, 3, [100, 50], [9, 13], ROWS + "2,4,false>", None) for d in (64, 128, 256)],
    (64, 32, 2, 1, [5000, 3300], [300, 290], ROWS + "2,4,true>", JOIN + "2,1>"),
    *[(d, 32, 1, 3, [1500], [9], ROWS + "2,4,true>", JOIN + "2,1>") for d in (128, 256)],
    *[(d, 64, 1, 3, [5000], [9], ROWS + "2,4,true>", JOIN + "2,4>") for d in (64, 128, 256)],
    # 128 rows
    (64, 32, 16, 8, [300, 0, 220], [200, 0, 180], TILE + "false>", None),
    (128, 32, 16, 8, [300, 0, 220], [200, 0, 180], TILE + "false>", None),
    (256, 32, 8, 8, [100, 90], [70, 75], TILE + "false>", None),
    (64, 64, 1, 8, [16000], [8187], TILE + "true>", JOIN + "8,1>"),
    (128, 64, 4, 4, [30000], [3900], TILE + "true>", JOIN + "8,1>"),
    (256, 32, 8, 8, [600, 400], [70, 66], TILE + "true>", JOIN + "8,1>"),
    (64, 64, 2, 64, [87000], [548], TILE + "true>", JOIN + "8,4>"),
    (128, 64, 1, 64, [60000], [1000], TILE + "true>", JOIN + "8,4>"),
    (256, 32, 1, 3, [5000], [1100], TILE + "true>", JOIN + "8,4>"),
]


def names(step):
    """The step's kernels, as the library calls them."""
    return [k % step[0] for k in step[6:8] if k is not None]


def name(step):
    return "_".join(n.replace("kv_attention_", "").replace("_kernel", "") for n in names(step)) + "_%d" % step[4][0]
