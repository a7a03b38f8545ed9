"""Sizes of the tests of grouped products and adapters: beside those with a reason of their own, sizes that between them take every form of
every product that sizes of up to 16384 rows and 4096 channels take (test_group_plans_host.py draws such sizes and fails for a form that is not
among these)."""
import random

# rows, groups, c_in, c_out
GROUP_FORMS = [(3, 1, 16, 16), (2, 1, 73, 67), (681, 1, 16, 24), (4, 1, 16, 472), (9, 1, 544, 17), (164, 10, 2264, 16), (2, 1, 16, 33),
               (8, 1, 23, 22), (2, 1, 37, 20), (17, 1, 19, 24), (8, 2, 24, 18), (38, 3, 17, 18), (12, 2, 26, 24), (132, 10, 16, 2064),
               (266, 30, 1768, 16), (136, 1, 29, 597), (218, 64, 88, 72), (1042, 24, 16, 1446), (156, 40, 27, 33), (2122, 17, 18, 20),
               (70, 22, 19, 100), (101, 18, 18, 132), (370, 62, 18, 46), (1998, 2, 1448, 80), (53, 6, 16, 840), (2942, 31, 232, 224),
               (26, 11, 16, 675), (150, 32, 20, 175), (2047, 2, 144, 1712), (2231, 42, 16, 136), (2281, 20, 149, 18), (229, 2, 1195, 1602),
               (2026, 2, 1913, 133)]
# rows, requests, rank, c_in, c_out
ADAPTER_FORMS = [(2, 2, 2, 24, 16), (750, 1, 8, 16, 16), (1, 1, 16, 834, 913), (138, 2, 27, 585, 17), (1, 1, 1, 20, 115), (4, 1, 8, 24, 16),
                 (4, 1, 8, 19, 32), (7, 1, 8, 27, 22), (1, 1, 16, 22, 16), (14, 2, 8, 25, 32), (45, 1, 32, 16, 21), (6, 4, 9, 56, 22),
                 (179, 2, 8, 16, 1312), (3122, 1, 128, 16, 16), (143, 1, 8, 1296, 16), (3485, 3, 16, 415, 18), (1181, 7, 8, 17, 68),
                 (7932, 3, 16, 16, 144), (3862, 7, 16, 16, 39), (49, 1, 32, 2680, 1536), (18, 2, 32, 975, 2169), (104, 11, 16, 3656, 24),
                 (138, 1, 32, 1040, 1512), (7165, 5, 16, 400, 16), (5485, 5, 8, 16, 536), (127, 127, 8, 16, 3080), (3162, 3, 64, 1184, 136),
                 (3158, 2, 64, 136, 1256)]


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
        key = (rank > 0, dtype, part, p.form, 0 if rank and part == dc.GROUP_DW else p.tile_cols, p.split > 1)
        out.add(key + (c_in % 4 == 0, c_out % 4 == 0) if p.form == dc.GROUP_FMAS else key)
    return out
