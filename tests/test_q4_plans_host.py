"""Which ways through the 4-bit products the GPU tests take, held to those that the estimate picks over sizes drawn at random."""
import numpy as np
import pytest

pytest.importorskip("torch")

from paper_2301_12187_b200 import dc
from tests import test_gpu_q4 as forms
from tests import test_gpu_q4_plans as plans


def reached():
    ways = {}
    for shapes, forward in ((forms.FORMS + forms.PRODUCTS + forms.NARROW + plans.PRODUCTS, False), (forms.FORWARD_FORMS + plans.FORWARDS, True)):
        for shape in shapes:
            for fmt in (dc.MX4, dc.NV4):
                for dtype in (dc.F32, dc.BF16):
                    ways.setdefault(plans.way(*shape, fmt, dtype, forward), shape)
    return ways


def drawn(n, seed):
    """Rows up to 200000, half of them few; 1 to 16384 columns, most of the outputs a multiple of 8."""
    r = np.random.default_rng(seed)
    for _ in range(n):
        rows = int(np.exp(r.uniform(0, np.log(200000 if r.random() < 0.7 else 64))))
        c_in, c_out = (int(np.exp(r.uniform(0, np.log(16384)))) for _ in range(2))
        yield rows, c_in, max(8, c_out // 8 * 8) if r.random() < 0.7 else c_out


def test_the_gpu_tests_take_every_way_that_is_picked():
    have = reached()
    missing = {}
    for shape in drawn(8000, 5):
        for fmt in (dc.MX4, dc.NV4):
            for dtype in (dc.F32, dc.BF16):
                for forward in (False, True):
                    way = plans.way(*shape, fmt, dtype, forward)
                    if "apart" not in way[0]:     # (the same products as without quantising)
                        if way not in have:
                            missing.setdefault(way, (shape, fmt, dtype))
    assert not missing, "\n".join("%s: %s" % (s, ", ".join(w)) for w, s in missing.items())


def test_pairs_walk_over_several_tiles():
    """With 256 and with 128 columns, in both formats, with ragged rows too; and some so many that each accumulator is used three times or more."""
    for fmt in ("mx4", "nv4"):
        for columns, accumulators in (("two scale tiles", "1 accumulators"), ("one scale tile", "2 accumulators")):
            for rows in ("rows of 16 bytes", "ragged rows"):
                assert any(w[0] == "pairs" and w[1] == fmt and w[2] == columns and w[4] == accumulators and w[7] == rows and w[8] == "many tiles" for w in reached()), \
                    (fmt, columns, rows)
