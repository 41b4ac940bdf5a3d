"""fp16 attention of new tokens where a row's probabilities are small beside the reference of its exponentials, against bounds that go by them."""
import math

import pytest
import torch

from chunk_bounds import check_rows
from chunk_util import Batch
from test_gpu_chunk import run

pytestmark = pytest.mark.gpu


def alike(b, seed=0):
    """One query per KV head, of which every key of a cache has nearly the same logit; returns it, [KV heads, 128]."""
    g = torch.Generator().manual_seed(seed)
    u = torch.randn((b.hkv, 128), generator=g)
    b.q[:] = u.repeat_interleave(b.hq // b.hkv, 0).to(b.dtype)
    return u.to(b.dtype).float()


def put(b, w, where, x):
    """K (w = 0) or V of the tokens (KV head, page, slot) `where`: x [..., 128], through the 4-bit format where the cache has it."""
    if b.kind == "4":
        from oracle import kv4_oracle as k4
        code, scale = k4.quantise(x.double().numpy())
        b.code[w][where], b.scale[w][where] = torch.from_numpy(code).to(b.code.dtype), torch.from_numpy(scale).to(b.scale.dtype)
        x = torch.from_numpy(k4.values(code, scale))
    b.rows[w][where] = x.to(b.dtype)


def against(b, u, reference, step):
    """Values of +1 and -1, by whether a probability of the key beside `reference` (a logit per KV head) is rounded up or down to `step`: errors
    that do not average."""
    x = torch.einsum("hpsd,hd->hps", b.rows[0].double(), u.double()) * 128.0 ** -0.5
    p = torch.exp(x - reference.double()[:, None, None]) / step
    put(b, 1, slice(None), torch.where(torch.round(p) > p, 1.0, -1.0)[..., None].expand(*p.shape, 128).float())


@pytest.mark.parametrize("cache", ["16", "4"])
def test_a_strong_key_in_front_of_the_window(cache):
    """2048 tokens are 256 wide tiles, whose keys are not cut.  The token in front of the first window lies in the first tile of keys of the first
    64 queries, two of which see another key of that tile: the others' reference is a logit 13 above all that they see, and a probability
    against it a few steps of fp16."""
    window, past = 8192, 8192 + 128 + 61
    b = Batch(new=[2048], past=[past], hq=32, hkv=8, dtype=torch.float16, page=64, cache=cache, seed=21)
    u = alike(b)
    put(b, 0, slice(None), 0.05 * torch.randn((8, b.n_pages, b.page, 128), generator=torch.Generator().manual_seed(22)))
    page, slot = b.spot(0, past - window)
    put(b, 0, (slice(None), page, slot), 12.9 * 128 ** 0.5 * u / u.square().sum(1, keepdim=True))
    strong = (b.rows[0][:, page, slot].double() * u.double()).sum(1) * 128.0 ** -0.5
    assert 11.5 < strong.min() < strong.max() < 13.5
    against(b, u, strong, 2.0 ** -24)
    b.expected = lambda *a: {}                                    # (65536 rows; some of them are looked at below)
    out, lse, _ = run(b, "local", sink=0, window=window)
    rows = [(t, h) for t in (0, 1, 2, 3, 31, 62, 63, 64, 100, 2047) for h in (0, 5, 31)]
    check_rows(b, out, lse, rows, sink=0, window=window, faint=2.0 ** -25, off_reference=2.0 ** -12)


@pytest.mark.parametrize("again", [False, True], ids=["plain", "taken_again"])
@pytest.mark.parametrize("cache", ["16", "4"])
def test_a_dominant_key_without_a_value(cache, again):
    _dominant(5, cache, again)


@pytest.mark.parametrize("cache", ["16", "4"])
@pytest.mark.parametrize("pos", [63, 64, 127, 128, 3000])
def test_a_dominant_key_anywhere(pos, cache):
    _dominant(pos, cache, False)


def _dominant(pos, cache, again):
    """One of a context's tokens has nearly all of the softmax and a value of 0, as the first token of a prompt often has: the outputs are
    sums of probabilities 16 below it, 2^-23 of it each.  Wide tiles, whose keys are not cut; with a page that is not there they are taken again."""
    b = Batch(new=[2048], past=[6000], hq=32, hkv=8, dtype=torch.float16, page=64, cache=cache, seed=23)
    u = alike(b, 24)
    put(b, 0, slice(None), 0.05 * torch.randn((8, b.n_pages, b.page, 128), generator=torch.Generator().manual_seed(25)))
    page, slot = b.spot(0, pos)
    put(b, 0, (slice(None), page, slot), 16.0 * 128 ** 0.5 * u / u.square().sum(1, keepdim=True))
    strong = (b.rows[0][:, page, slot].double() * u.double()).sum(1) * 128.0 ** -0.5
    assert 14.0 < strong.min() < strong.max() < 17.0
    against(b, u, strong, 2.0 ** -24)
    put(b, 1, (slice(None), page, slot), torch.zeros((8, 128)))
    if again:
        b.table[0, 70] = -1
    b.expected = lambda *a: {}
    out, lse, _ = run(b)
    check_rows(b, out, lse, [(t, h) for t in (0, 1, 63, 64, 1000, 2047) for h in (0, 5, 31)], faint=2.0 ** -37)


@pytest.mark.parametrize("again", [False, True], ids=["plain", "taken_again"])
@pytest.mark.parametrize("cache", ["16", "4"])
@pytest.mark.parametrize("new", [1, 3, 6])
def test_dominant_keys_in_tiles_of_few_rows(new, cache, again):
    """Every 32nd token has nearly all of the softmax and a value of 0; the others' probabilities are 2^-26 of theirs."""
    b = Batch(new=[new], past=[1500], dtype=torch.float16, cache=cache, seed=26 + new)
    u = alike(b, 27)
    put(b, 0, slice(None), torch.zeros((2, b.n_pages, b.page, 128)))
    put(b, 1, slice(None), torch.full((2, b.n_pages, b.page, 128), 1024.0))
    for pos in range(7, b.ctx[0], 32):
        page, slot = b.spot(0, pos)
        put(b, 0, (slice(None), page, slot), 18.0 * 128 ** 0.5 * u / u.square().sum(1, keepdim=True))
        put(b, 1, (slice(None), page, slot), torch.zeros((2, 128)))
    if again:
        b.table[0, 40] = -1
    out, lse, _ = run(b)
    check_rows(b, out, lse, [(t, h) for t in range(new) for h in range(8)], parts=2, faint=2.0 ** -38)
