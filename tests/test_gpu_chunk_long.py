"""Long contexts in ranges, against bounds that do not grow with them."""
import pytest
import torch

import test_gpu_chunk_wide as wide
from chunk_bounds import check_rows
from test_chunk_bounds_cpu import _long
from test_gpu_chunk import DT, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("cache", ["16", "4"])
def test_tiles_of_few_rows(cache, dtype):
    b = _long(cache, DT[dtype])
    b.expected = lambda *a: {}
    for call in (run, wide.run):                                  # (few rows are taken alike under either's bounds)
        for which, how in (("all", {}), ("local", dict(sink=5, window=4000))):
            out, lse, _ = call(b, which, **how)
            check_rows(b, out, lse, [(i, h) for i in range(7) for h in range(8)], parts=2, faint=0.0 if dtype == "bf16" else 2.0 ** -38, **how)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("cache", ["16", "4"])
@pytest.mark.parametrize("sink", [0, 5])
def test_wide_tiles(sink, cache, dtype):
    b = wide.Batch(new=[40, 70], past=[9000, 5001], cache=cache, dtype=DT[dtype], page=64, seed=6)
    b.expected = lambda *a: {}
    for which, how in (("all", {}), ("local", dict(sink=sink, window=4000))):
        out, lse, _ = wide.run(b, which, **how)
        check_rows(b, out, lse, [(i, h) for i in range(0, 110, 3) for h in range(8)], faint=0.0 if dtype == "bf16" else 2.0 ** -25, **how)
