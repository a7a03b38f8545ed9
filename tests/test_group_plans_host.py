"""Which forms grouped products and adapters take, without a GPU: plans are in range, and every form that drawn sizes take is one that a GPU
test takes."""
import ctypes as C
import math
import random

import pytest

pytest.importorskip("torch")

from paper_2301_12187_b200 import dc
from tests.group_sizes import ADAPTER_FORMS, GROUP_FORMS, plan_keys


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def width(rng):
    v = log_int(rng, 16, 4096)
    return v if rng.random() < 0.2 else max(8, v // 8 * 8)


def covered():
    keys = set()
    for dtype in (dc.BF16, dc.F32):
        for rows, runs, c_in, c_out in GROUP_FORMS:
            keys |= plan_keys(dc, rows, runs, 0, c_in, c_out, dtype)
        for rows, runs, rank, c_in, c_out in ADAPTER_FORMS:
            keys |= plan_keys(dc, rows, runs, rank, c_in, c_out, dtype)
    return keys


def test_drawn_sizes_take_tested_forms():
    rng, have = random.Random(11), covered()
    for _ in range(3000):
        rows, c_in, c_out, dtype = log_int(rng, 1, 16384), width(rng), width(rng), rng.choice([dc.BF16, dc.F32])
        new = plan_keys(dc, rows, log_int(rng, 1, 64), 0, c_in, c_out, dtype)
        runs = rows if rows <= 128 and rng.random() < 0.6 else min(rows, log_int(rng, 1, 12))
        new |= plan_keys(dc, rows, runs, rng.choice([8, 16, 32, 64, 128, rng.randint(1, 100)]), c_in, c_out, dtype)
        assert new <= have, (rows, c_in, c_out, dtype, new - have)


def test_plans_are_in_range():
    rng = random.Random(3)
    for _ in range(2000):
        args = (log_int(rng, 1, 1 << 30), log_int(rng, 1, 1 << 20), log_int(rng, 1, 1 << 20), log_int(rng, 1, 1 << 20), rng.choice([0, 0, rng.randint(1, 128)]),
                rng.choice([dc.BF16, dc.F32]))
        for part in range(3):
            p = dc.group_plan(*args, part)
            if p.form == dc.GROUP_FMAS:
                assert p.tile_cols in (4, 8, 16) and part != dc.GROUP_DW and args[5] == dc.F32
                continue
            assert p.form in (dc.GROUP_TILES, dc.GROUP_PAIRS, dc.GROUP_FEW_ROWS) and 16 <= p.tile_cols <= 256 and p.tile_cols % 16 == 0, args
            assert 1 <= p.split <= 8 and 1 <= p.stages <= 8, (args, part, p.stages)
            if p.form == dc.GROUP_PAIRS:
                assert p.tile_cols == 256 and p.split == 1
            if p.form == dc.GROUP_FEW_ROWS:
                assert p.tile_cols <= 64 and part != dc.GROUP_DW and args[5] == dc.BF16


def test_plan_query_refuses():
    f, p = dc.lib().dc_group_plan_query, dc.GroupPlan()

    def call(rows=8, runs=2, c_in=8, c_out=8, rank=0, dtype=dc.BF16, part=0, plan=p):
        return f(rows, runs, c_in, c_out, rank, dtype, part, C.byref(plan) if plan is not None else None)

    assert call() == dc.OK and call(rank=128) == dc.OK
    assert call(rows=0) == dc.ERR_INVALID_ARG and call(runs=0) == dc.ERR_INVALID_ARG and call(rank=-1) == dc.ERR_INVALID_ARG
    assert call(part=3) == dc.ERR_INVALID_ARG and call(part=-1) == dc.ERR_INVALID_ARG and call(dtype=2) == dc.ERR_INVALID_ARG and call(plan=None) == dc.ERR_INVALID_ARG
    assert call(rank=129) == dc.ERR_UNSUPPORTED and call(rows=(1 << 30) + 1) == dc.ERR_UNSUPPORTED and call(runs=(1 << 20) + 1) == dc.ERR_UNSUPPORTED
