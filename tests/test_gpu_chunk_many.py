"""New tokens of more sequences than a wave has lanes, over contexts that are cut into ranges: the plan comes from memory, and partial results, their
merge and what is taken again go by it."""
import random

import pytest
import torch

import test_gpu_chunk_wide as wide
from chunk_bounds import check_rows
from chunk_util import Batch
from test_gpu_append import Case
from test_gpu_chunk import DT, MARK, run
from paper_2605_16928_amd import rtp

pytestmark = pytest.mark.gpu


def _served(b, out, lse, which, ret, rows, **how):
    heads = range(b.hq) if which == "all" else [h for h in range(b.hq) if h not in ret]
    check_rows(b, out, lse, [(i, h) for i in rows for h in heads], **how)
    assert which == "all" or (out[:b.total, list(ret)] == MARK).all()


@pytest.mark.parametrize("lost", [False, True], ids=["plain", "taken_again"])
@pytest.mark.parametrize("cache,dtype", [("16", "bf16"), ("4", "bf16"), ("16", "fp16"), ("4", "fp16")])
@pytest.mark.parametrize("bounds", ["narrow", "wide"])
def test_a_hundred_sequences_in_ranges(bounds, cache, dtype, lost):
    """100 sequences, some without new tokens, six of them with 2000 to 6000 tokens; the launches that cut them have to be there."""
    rng = random.Random(41)
    new = [rng.choice([0, 1, 1, 1, 2, 5]) for _ in range(100)]
    past = [rng.randint(0, 60) for _ in range(100)]
    for b, (n, p) in {3: (1, 6000), 17: (4, 2000), 40: (1, 3100), 63: (2, 4500), 64: (1, 5003), 99: (3, 2222)}.items():
        new[b], past[b] = n, p
    if bounds == "wide":
        new[40], new[99] = 40, 30                                 # (160 and 120 rows to a KV head)
    b = Batch(new=new, past=past, cache=cache, dtype=DT[dtype], page=64, seed=42)
    if lost:
        b.table[[3, 17, 40, 63, 64, 99], 20] = -1
    rows = sorted({i for s in (0, 1, 2, 3, 17, 40, 41, 62, 63, 64, 65, 98, 99) for i in list(range(b.off[s], b.off[s + 1]))[:3] + [b.off[s + 1] - 1]
                   if b.off[s] <= i < b.off[s + 1]} | set(range(0, b.total, 7)))
    faint = 0.0 if dtype == "bf16" else 2.0 ** -25
    b.expected = lambda *a: {}
    call = run if bounds == "narrow" else wide.run
    for which, ret, how in (("all", (), {}), ("local", (1, 4), dict(sink=20, window=1500))):
        names = wide._launches(lambda: call(b, which, ret, **how))
        assert "plan" in names and "merge" in names, names
        out, lse, _ = call(b, which, ret, **how)
        _served(b, out, lse, which, ret, rows, faint=faint, **how)
        assert (out[b.total:] == MARK).all()
    if bounds == "narrow":                                        # (the plan begins with the ranges of the longest sequence)
        ws = torch.zeros(1 << 26, dtype=torch.uint8, device="cuda")
        again, lse2, _ = run(b, which, ret, ws=ws, **how)
        assert torch.equal(again, out) and torch.equal(lse2, lse) and int(ws[:4].view(torch.int32)) > 1


@pytest.mark.parametrize("cache", ["16", "4"])
def test_more_sequences_than_the_plan_has_threads(cache):
    """1500 sequences (the plan's loops come round), 5000 (three steps of every search): single tokens and none, a few long contexts."""
    for B in (1500, 5000):
        rng = random.Random(B)
        new, past = [rng.choice([0, 1, 1]) for _ in range(B)], [rng.randint(0, 20) for _ in range(B)]
        for s in (0, 1023, 1024, B - 1):
            new[s], past[s] = 1, rng.randint(1500, 3000)
        b = Batch(new=new, past=past, hq=4, hkv=1, cache=cache, seed=B)
        rows = sorted({b.off[s] for s in (0, 1023, 1024, B - 1)} | set(range(0, b.total, 37)) | {b.total - 1})
        b.expected = lambda *a: {}
        for which, ret, how in (("all", (), {}), ("local", (2,), dict(sink=3, window=900))):
            names = wide._launches(lambda: run(b, which, ret, **how))
            assert "plan" in names, names
            out, lse, _ = run(b, which, ret, **how)
            _served(b, out, lse, which, ret, rows, **how)


def test_append_to_thousands_of_sequences():
    for B in (1500, 5000):
        rng = random.Random(B)
        c = Case([rng.choice([0, 1, 1, 2]) for _ in range(B)], [rng.randint(0, 40) for _ in range(B)], hq=4, hkv=1, seed=B)
        c.check(*c.call())


def test_thousands_of_sequences_without_new_tokens():
    """One token among 5000 sequences, at either end and in the middle."""
    for at in (0, 2500, 4999):
        new = [0] * 5000
        new[at] = 1
        b = Batch(new=new, past=[3] * 5000, hq=4, hkv=1, seed=at)
        b.expected = lambda *a: {}
        out, lse, _ = run(b)
        check_rows(b, out, lse, [(0, h) for h in range(4)])
        assert (out[1:] == MARK).all()
