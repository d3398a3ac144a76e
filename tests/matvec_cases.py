"""Shapes that reach every instance of the packed products' kernel: for each format and (tiles a
workgroup takes, copy, rows) of the launch rules a call of each kind (dense M rows, or rows per expert)
that takes it, with N no multiple of the tile, K past its last whole slice where the format has such K,
and row counts that are not the most a workgroup takes.  test_matvec_plan_cpu checks which instance each
takes; test_gpu_matvec runs them."""

# fmt, instance, rows (M of a dense call, or a list of rows per expert), N, K
VARIANTS = [
    ("nvfp4", (1, "cached", "all"), 7, 1001, 1056),
    ("nvfp4", (1, "cached", "small"), 3, 1001, 1056),
    ("nvfp4", (1, "cached", "twice"), [11, 0, 30, 9], 77, 1056),
    ("nvfp4", (1, "streamed", "all"), 11, 18090, 1888),
    ("nvfp4", (1, "streamed", "small"), 1, 9125, 3744),
    ("nvfp4", (1, "streamed", "small"), [1, 0, 4, 0, 1, 2, 0, 0] * 8, 5481, 96),
    ("nvfp4", (1, "streamed", "twice"), [13, 2, 0, 9] * 16, 661, 864),
    ("nvfp4", (1, "words", "all"), 13, 333, 1072),
    ("nvfp4", (1, "words", "small"), 2, 333, 1072),
    ("nvfp4", (1, "words", "twice"), [12, 17, 0], 45, 1072),
    ("nvfp4", (2, "cached", "all"), 49, 8501, 160),
    ("nvfp4", (2, "cached", "small"), [1, 2, 0, 1] * 32, 645, 96),
    ("nvfp4", (2, "cached", "twice"), [9, 4, 2, 7, 0] * 12, 885, 160),
    ("nvfp4", (2, "streamed", "all"), 10, 5145, 6752),
    ("nvfp4", (2, "streamed", "all"), [3, 3, 0, 2, 2, 3, 1, 4], 18817, 224),
    ("nvfp4", (2, "streamed", "small"), [1, 0, 2, 1] * 15, 1449, 416),
    ("nvfp4", (2, "streamed", "twice"), [30, 11, 0, 50, 9, 16] * 10, 927, 608),
    ("nvfp4", (2, "words", "all"), 49, 8501, 176),
    ("nvfp4", (2, "words", "small"), [1, 2, 0, 1] * 4, 5415, 48),
    ("nvfp4", (2, "words", "twice"), [9, 4, 2, 7, 0] * 12, 885, 176),
    ("mxfp4", (1, "cached", "all"), 15, 1001, 1056),
    ("mxfp4", (1, "cached", "twice"), [11, 0, 30, 9], 77, 1056),
    ("mxfp4", (1, "streamed", "all"), 2, 11181, 3040),
    ("mxfp4", (2, "streamed", "all"), [2, 1], 7441, 2272),
    ("mxfp4", (1, "streamed", "twice"), [70, 63], 5589, 3040),
    ("mxfp4", (2, "cached", "all"), 63, 8501, 96),
    ("mxfp4", (2, "cached", "twice"), [9, 4, 2, 7, 0] * 12, 885, 160),
    ("mxfp4", (2, "streamed", "all"), 8, 24405, 1376),
    ("mxfp4", (2, "streamed", "all"), [2, 3, 0, 1] * 32, 483, 608),
    ("mxfp4", (2, "streamed", "twice"), [30, 11, 0, 50, 9, 16] * 10, 975, 608),
    ("q4k", (1, "cached", "all"), 5, 1001, 1280),
    ("q4k", (1, "cached", "all"), [40, 9, 0, 64, 1], 77, 1280),
    ("q4k", (1, "streamed", "all"), 2, 5053, 6912),
    ("q4k", (1, "streamed", "all"), [3, 2, 0, 5, 1, 7, 0, 6] * 16, 43, 6912),
    ("q4k", (2, "cached", "all"), 52, 7271, 256),
    ("q4k", (2, "cached", "all"), [9, 4, 2, 7, 0] * 12, 469, 256),
    ("q4k", (2, "streamed", "all"), 16, 19077, 1792),
    ("q4k", (2, "streamed", "all"), [17, 2, 0, 33, 16] * 2, 16393, 256),
]


def instances():
    """Every instance of the kernel: what qf_matvec.hip compiles for a format."""
    out = set()
    for fmt, copies, rows in (("nvfp4", ("cached", "streamed", "words"), ("all", "small", "twice")),
                              ("mxfp4", ("cached", "streamed"), ("all", "twice")), ("q4k", ("cached", "streamed"), ("all",))):
        out |= {(fmt, (nt, c, r)) for nt in (1, 2) for c in copies for r in rows}
    return out


SPARE = 3                                                          # rows of no expert after the last one's


def sizes(rows):
    """grouped, E, R of a case's rows."""
    return (True, len(rows), sum(rows) + SPARE) if isinstance(rows, list) else (False, 1, rows)
