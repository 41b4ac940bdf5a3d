"""Attention of new tokens where a range of keys has to be taken again: what comes of it is as exact as what does not."""
import math

import pytest
import torch

import test_gpu_chunk_wide as wide
from chunk_bounds import check_rows
from chunk_util import Batch
from test_gpu_chunk import DT
from test_gpu_chunk_references import alike, put

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("cache", ["16", "4"])
@pytest.mark.parametrize("why", ["lost_page", "not_finite"])
def test_few_rows_beside_a_chunk(why, cache, dtype):
    """Tiles of up to 32 rows in a call that takes wide ones: their probabilities stay in two parts."""
    b = Batch(new=[3, 70, 1], past=[700, 300, 2500], cache=cache, dtype=DT[dtype], seed=31)
    u = alike(b, 32)
    put(b, 0, slice(None), 0.1 * torch.randn((2, b.n_pages, b.page, 128), generator=torch.Generator().manual_seed(33)))
    for s in range(3):                                            # (the largest score is the first one)
        page, slot = b.spot(s, 0)
        put(b, 0, (slice(None), page, slot), 2.0 * 128 ** 0.5 * u / u.square().sum(1, keepdim=True))
    x = torch.einsum("hpsd,hd->hps", b.rows[0].double(), u.double()) * 128.0 ** -0.5
    p = torch.exp(x - x.flatten(1).amax(1)[:, None, None])
    put(b, 1, slice(None), torch.where(p.to(b.dtype).double() > p, 1.0, -1.0)[..., None].expand(*p.shape, 128).float())
    if why == "lost_page":
        b.table[:, 3::4] = -1
    else:                                                         # V of the last token of two sequences, which one row of each sees
        for s, pos in ((0, 702), (1, 369)):
            page, slot = b.spot(s, pos)
            b.rows[1][:, page, slot] = math.nan
            if cache == "4":
                b.scale[1][:, page, slot] = 255
    names = wide._launches(lambda: wide.run(b))
    assert "chunk_again" in names, names
    faint = 0.0 if dtype == "bf16" else 2.0 ** -38
    for which, how in (("all", {}), ("local", dict(sink=40, window=400))):
        out, lse, _ = wide.run(b, which, **how)
        few, many = [0, 1, 73] if why == "not_finite" else [0, 1, 2, 73], range(3, 72, 6)
        check_rows(b, out, lse, [(i, h) for i in few for h in range(8)], parts=2, faint=faint, **how)
        check_rows(b, out, lse, [(i, h) for i in many for h in range(8)], faint=2.0 ** 13 * faint, **how)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("cache", ["16", "4"])
@pytest.mark.parametrize("sink", [0, 20])
def test_pages_that_nobody_sees(sink, cache, dtype):
    """Pages between the sink and the first window are given back, as a server does with them: their tiles of keys, which the window's edge and the sink
    share with what is seen, are not taken again -- the results are those of before to the bit (sink 20: every row sees its reference)."""
    b = Batch(new=[70, 2], past=[1000, 777], cache=cache, dtype=DT[dtype], seed=34)
    how = dict(sink=sink, window=300)
    whole = [run(b, "local", **how)[:2] for run in (wide.run_small, wide.run)]
    for s in range(2):
        first = max(0, b.ctx[s] - b.new[s] - 300 + 1)
        b.table[s, -(-sink // b.page):first // b.page] = -1
    assert (b.table[0, :44] == -1).sum() >= 40
    faint = 0.0 if dtype == "bf16" else 2.0 ** -25
    for (out0, lse0), run in zip(whole, (wide.run_small, wide.run)):
        out, lse, _ = run(b, "local", **how)
        check_rows(b, out, lse, [(i, h) for i in range(0, 72, 5) for h in range(8)], faint=faint, **how)
        same = bool((out == out0).all()) and bool((lse == lse0).all())
        assert same or sink == 0
