"""Sizes at which the attention over what a place sees takes its tiled kernel, for test_span_tiled_gpu.py;
test_span_plan.py holds them to it without a GPU."""
WIDTHS = list(range(32, 161, 8))
RULES = [(1, 0, 0), (1, 1, 0), (1, 64, 0), (1, 65, 1), (1, 200, 64), (1, 1000, 100), (0, 0, 0), (0, 130, 0), (0, 50, 70), (7, 0, 0),
         (7, 20, 3), (64, 128, 65), (90, 180, 90), (1 << 30, 0, 0), (2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1)]
# (B, H, Hk, Lq, tokens before them)
USUAL = (5, 8, 8, 200, 60)
MANY = (33, 8, 8)                   # with the lengths of LENGTHS
LENGTHS = [(33, 0), (33, 31), (64, 0), (65, 0), (65, 63), (127, 1), (128, 1), (129, 0), (257, 190)]
GROUPS = [(9, 4, 2, 230, 30), (20, 5, 1, 90, 110), (17, 6, 2, 90, 110), (20, 7, 1, 70, 130), (9, 32, 2, 30, 170), (7, 33, 3, 40, 160), (3, 130, 1, 25, 175),
          (40, 40, 20, 17, 50)]
RAGGED = (8, 40, 20, 40, 260)
INFINITE = (1, 64, 32, 260, 0)
PAGES = (2, 32, 16, 150, 700)
PARTS = [(4, 16, 8, 129, 2871, (1, 1500, 300)), (2, 4, 4, 1100, 900, (1, 0, 0)), (2, 4, 2, 1100, 1900, (0, 0, 0))]
FAR = (1, 16, 4, 600, 100)          # tokens at the end of tensors past 32 bits
FAR_DENSE = (1, 4, 1, 2100, (1 << 24) - 1900)
LARGE = (3, 12, 12, 250, 0)         # of unusual scores
CAUSAL = (2, 2, 2, 2100, 0)         # in parts, one pass or two of the card


def cases():
    """((B, H, Hk, Lq, far), rule, widths, kinds) of every tiled call of the GPU tests."""
    plain, window = (1, 0, 0), (1, 100, 5)
    yield USUAL, window, WIDTHS, "dp"
    for rule in RULES:
        yield USUAL, rule, [64], "dp"
    for length in LENGTHS:
        for rule in (plain, (0, 40, 2)):
            yield MANY + length, rule, [40, 128], "dp"
    for group in GROUPS:
        yield group, (1, 90, 4), [40, 128], "dp"
    for rule in (plain, (1, 70, 9), (0, 0, 0), (5, 64, 64)):
        yield RAGGED, rule, [64, 128], "dp"
    for rule in (plain, (1, 64, 0), (1, 40, 31), (0, 100, 33)):
        yield INFINITE, rule, [40, 64, 128, 136], "dp"
    for rule in (plain, (1, 130, 70)):
        yield PAGES, rule, [64, 128], "p"
    for part in PARTS:
        yield part[:5], part[5], [40, 64, 128, 160], "dp"
    yield FAR, plain, [128], "p"
    yield FAR_DENSE, (1, 150, 0), [128], "d"
    for rule in (plain, (1, 90, 20)):
        yield LARGE, rule, [40, 64, 128, 136], "dp"
    yield CAUSAL, plain, [64, 128], "dp"
