"""Sizes of the tests of grouped products and adapters: beside those with a reason of their own, sizes that between them take every form of
every product that sizes of up to 16384 rows and 4096 channels take (test_group_plans_host.py draws such sizes and fails for a form that is not
among these)."""
import random

# rows, groups, c_in, c_out
GROUP_FORMS = [(3, 1, 16, 16), (681, 1, 16, 24), (141, 35, 488, 16), (2, 1, 80, 472), (290, 22, 1248, 16), (2335, 24, 16, 16), (317, 22, 16, 1080),
               (138, 1, 16, 624), (151, 1, 600, 24), (7550, 5, 392, 16), (101, 3, 1704, 712), (2108, 63, 24, 528), (2281, 20, 149, 18), (1267, 1, 2853, 139),
               (2385, 45, 240, 216), (138, 1, 2168, 1760), (174, 7, 481, 3782)]
# rows, requests, rank, c_in, c_out
ADAPTER_FORMS = [(2, 2, 2, 24, 16), (750, 1, 8, 16, 16), (1, 1, 8, 928, 880), (139, 1, 8, 16, 672), (151, 1, 16, 712, 16), (18, 2, 32, 975, 2169),
                 (7932, 3, 16, 16, 144), (7779, 4, 64, 144, 16), (104, 11, 16, 3656, 24), (138, 1, 32, 1040, 1512), (127, 127, 8, 16, 3080),
                 (33, 2, 16, 3576, 912), (7165, 5, 16, 400, 16), (5485, 5, 8, 16, 536), (3162, 3, 64, 1184, 136), (3158, 2, 64, 136, 1256)]


def spread(rows, runs, seed):
    """`rows` over `runs`, unevenly; some of many may be empty."""
    rng = random.Random(seed)
    weight = [rng.expovariate(1.0) for _ in range(runs)]
    sizes = [0] * runs
    for k in rng.choices(range(runs), weight, k=rows):
        sizes[k] += 1
    return sizes


def plan_keys(dc, rows, runs, rank, c_in, c_out, dtype):
    """What tells the forms of a call's products apart (of a gradient of adapters the tile's columns are the rank's)."""
    out = set()
    for part in (dc.GROUP_FORWARD, dc.GROUP_DX, dc.GROUP_DW):
        p = dc.group_plan(rows, runs, c_in, c_out, rank, dtype, part)
        out.add((rank > 0, dtype, part, p.form, 0 if rank and part == dc.GROUP_DW else p.tile_cols, p.split > 1))
    return out
