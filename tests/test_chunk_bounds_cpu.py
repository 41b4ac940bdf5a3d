"""The bounds that attention of new tokens is held to can fail: an output of zeros, or one that lacks a range of its keys, is outside them, however long
the context."""
import pytest
import torch

from chunk_bounds import row
from chunk_util import Batch


def _long(cache, dtype):
    return Batch(new=[1, 4, 2], past=[9000, 5001, 1300], cache=cache, dtype=dtype, page=64, seed=5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("cache", ["16", "4"])
@pytest.mark.parametrize("how", [dict(parts=2), dict(parts=1)])
def test_wrong_outputs_are_outside(how, cache, dtype):
    b = _long(cache, dtype)
    faint = 0.0 if dtype == torch.bfloat16 else 2.0 ** -38 if how["parts"] == 2 else 2.0 ** -25
    for band in ({}, dict(sink=5, window=4000)):
        for i in (0, 1, 4, 6):
            for h in (0, 5):
                o, lse, tol, tol_z = row(b, i, h, faint=faint, **how, **band)
                assert (o.abs() > tol).any()                      # zeros (a row passes only if all of its 128 dims do)
                whole, s = b.table.clone(), next(s for s in range(3) if b.off[s] <= i < b.off[s + 1])
                last = (b.ctx[s] - 1) // b.page
                b.table[s, max(0, last - 3):last - 1] = -1        # two pages of 64
                part, lse_part, _, _ = row(b, i, h, faint=faint, **how, **band)
                b.table = whole
                assert ((part - o).abs() > tol).any() and abs(lse_part - lse) > tol_z
