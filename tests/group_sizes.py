"""Sizes of the tests of grouped products and adapters: beside those with a reason of their own, sizes that between them take every form of
every product that sizes of up to 16384 rows and 4096 channels take (test_group_plans_host.py draws such sizes and fails for a form that is not
among these)."""
import random

# rows, groups, c_in, c_out
GROUP_FORMS = [(4, 1, 16, 16), (844, 1, 16, 24), (19, 1, 16, 16), (35, 1, 16, 568), (40, 1, 536, 16), (1, 1, 464, 488), (49, 1, 16, 928), (351, 7, 2128, 16),
               (28, 2, 528, 1512), (1500, 2, 136, 1281), (1774, 26, 1156, 79), (1339, 7, 184, 2512), (4769, 4, 408, 432), (19, 27, 131, 667), (1466, 3, 2000, 144)]
# rows, requests, rank, c_in, c_out
ADAPTER_FORMS = [(1, 1, 2, 16, 40), (550, 1, 38, 24, 16), (27, 1, 8, 24, 16), (1, 1, 8, 616, 528), (40, 4, 8, 552, 16), (70, 2, 8, 17, 484), (138, 2, 8, 824, 16),
                 (167, 2, 32, 16, 632), (23, 1, 8, 524, 626), (3104, 8, 59, 592, 72), (3215, 2, 128, 72, 688), (4840, 4, 8, 672, 16), (4360, 10, 8, 16, 784),
                 (3078, 3, 8, 16, 1400), (1118, 6, 28, 3880, 16), (165, 1, 16, 1760, 2080)]


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
