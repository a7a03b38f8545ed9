"""Adapters whose tensors others have taken the place of since: each call looks at those that are there.  Without a GPU."""
import pytest

torch = pytest.importorskip("torch")

from paper_2301_12187_b200 import dc
from tests.test_group_host import cpu  # noqa: F401


def test_tensors_in_the_place_of_an_adapters_own_are_looked_at(cpu):  # noqa: F811
    z = torch.zeros
    off, which, ws = z(3, dtype=torch.int32), z(2, dtype=torch.int32), z(256, dtype=torch.uint8)
    saved = z(4 * 96, dtype=torch.uint8)

    def forward(ad):
        dc.adapter_forward(z(4, 8), z(6, 8), ad, off, which, None, 0, None, saved, z(4, 6), ws)

    def backward(ad):
        dc.adapter_backward(z(4, 6), z(4, 8), z(6, 8), ad, off, which, saved, z(4, 8), z(3, 4, 8), z(3, 6, 4), ws)

    fresh = lambda: dc.Adapters(z(3, 4, 8), z(3, 6, 4), z(3))
    for name, t in (("a", z(2, 4, 8)), ("a", z(3, 2, 8)), ("a", z(3, 4, 16)[:, :, ::2]), ("a", z(3, 4, 6)), ("b", z(2, 6, 4)), ("b", z(3, 5, 4)),
                    ("b", z(3, 6, 4, dtype=torch.bfloat16)), ("b", z(3, 4, 6).transpose(1, 2)), ("scale", z(2)), ("scale", z(3, dtype=torch.bfloat16))):
        for call in (forward, backward):
            ad = fresh()
            setattr(ad, name, t)
            with pytest.raises(ValueError):
                call(ad)
    # others that belong together: of their sizes
    ad = fresh()
    ad.a, ad.b, ad.scale = z(5, 20, 8, dtype=torch.bfloat16), z(5, 7, 20, dtype=torch.bfloat16), None
    ad.check()
    assert (ad.count, ad.rank, ad.c_in, ad.c_out, ad.dtype) == (5, 20, 8, 7, dc.BF16)
    assert (ad.c.count, ad.c.rank, ad.c.scale) == (5, 20, None) and ad.saved(3).numel() == dc.adapter_saved_bytes(3, 20, dc.BF16)
