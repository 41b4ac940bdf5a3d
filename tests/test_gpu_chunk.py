"""Attention of batches of new tokens over paged caches, on the GPU, against the definition in 64 bits."""
import math

import pytest
import torch

from chunk_util import Batch, check
from paper_2605_16928_amd import rtp

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
MARK = 7.0


def _layer(b, ret=(), sink=4, window=64):
    return rtp.layer_desc(b.hq, b.hkv, list(ret), sink, window, kv_dtype=rtp.RTP_DTYPE_FP16 if b.dtype == torch.float16 else rtp.RTP_DTYPE_BF16)


def run(b, which="all", ret=(), sink=4, window=64, lse=True, prepared=None, ws=None):
    """(out, lse, expected) of one call."""
    layer = _layer(b, ret, sink, window)
    q, cache, chunk = prepared or b.device()
    out = torch.full((b.total + 2, b.hq, 128), MARK, dtype=b.dtype, device="cuda")
    z = torch.full((b.total + 2, b.hq), MARK, dtype=torch.float32, device="cuda") if lse else None
    four = "_kv4" if b.kind == "4" else ""
    sizes = (chunk.B, chunk.total_q, chunk.max_q, chunk.max_ctx)
    if which == "local":
        ws = ws if ws is not None else torch.empty(rtp.rtp_local_attn_chunk_workspace_bytes(layer, *sizes), dtype=torch.uint8, device="cuda")
        getattr(rtp, "rtp_local_attn_chunk" + four)(layer, q, q.stride(0), cache, chunk, out, z, ws)
        want = b.expected([h for h in range(b.hq) if h not in ret], sink, window)
    else:
        heads = rtp.RTP_HEADS_ALL if which == "all" else rtp.RTP_HEADS_RETRIEVAL
        ws = ws if ws is not None else torch.empty(rtp.rtp_dense_attn_chunk_workspace_bytes(layer, *sizes, heads), dtype=torch.uint8, device="cuda")
        getattr(rtp, "rtp_dense_attn_chunk" + four)(layer, q, q.stride(0), cache, chunk, heads, out, z, ws)
        want = b.expected(range(b.hq) if which == "all" else ret)
    torch.cuda.synchronize()
    return out, z, want


SHAPES = {
    "one": dict(new=[1], past=[0]),
    "one_long": dict(new=[1], past=[1300]),
    "prompt": dict(new=[77], past=[0]),
    "chunk": dict(new=[70], past=[333]),
    "ragged": dict(new=[3, 0, 65, 1, 0, 17], past=[200, 50, 1, 130, 0, 64]),
    "steps": dict(new=[1] * 9, past=[0, 1, 15, 16, 17, 63, 64, 65, 500]),
}


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("cache", ["16", "4"])
@pytest.mark.parametrize("name", list(SHAPES))
def test_dense(name, cache, dtype):
    b = Batch(**SHAPES[name], dtype=DT[dtype], cache=cache, seed=len(name))
    out, lse, want = run(b)
    check(b, want, out, lse, MARK)


@pytest.mark.parametrize("cache", ["16", "4"])
@pytest.mark.parametrize("sink,window", [(4, 64), (0, 1), (17, 5), (0, 100), (3, 0), (64, 128), (1000, 8)])
@pytest.mark.parametrize("name", ["one_long", "chunk", "ragged"])
def test_local(name, sink, window, cache):
    b = Batch(**SHAPES[name], cache=cache, seed=3)
    out, lse, want = run(b, "local", ret=[1, 4], sink=sink, window=window)
    check(b, want, out, lse, MARK)


@pytest.mark.parametrize("hq,hkv", [(8, 8), (4, 2), (8, 2), (16, 2), (12, 3), (128, 128)])
@pytest.mark.parametrize("which,ret", [("all", []), ("ret", [0, 3]), ("local", [0, 3]), ("local", [])])
def test_head_layouts(hq, hkv, which, ret):
    b = Batch(new=[5, 1, 34], past=[40, 100, 0], hq=hq, hkv=hkv, seed=hq + hkv)
    out, lse, want = run(b, which, ret, sink=2, window=30)
    check(b, want, out, lse, MARK)


@pytest.mark.parametrize("heads", [1, 2, 3, 4, 5, 6, 7, 8])
def test_any_number_of_served_heads(heads):
    """A KV head with 1 to 8 served heads: whole and partly filled tiles."""
    b = Batch(new=[90, 1], past=[10, 30], hq=16, hkv=2, seed=heads)
    ret = list(range(heads)) + [8]
    for which in ("ret", "local"):
        out, lse, want = run(b, which, ret, window=50)
        check(b, want, out, lse, MARK)


@pytest.mark.parametrize("page", [16, 32, 128, 256])
@pytest.mark.parametrize("order", ["heads", "pages", "tokens", "interleaved"])
def test_pages_and_layouts(page, order):
    b = Batch(new=[20, 3], past=[300, 77], page=page, order=order, seed=page)
    out, lse, want = run(b, lse=order != "pages")
    check(b, want, out, lse, MARK)


@pytest.mark.parametrize("which", ["all", "local"])
def test_many_sequences(which):
    """More than a wave has lanes: the plan comes from memory."""
    new = [(7 * i) % 5 for i in range(150)]
    b = Batch(new=new, past=[(13 * i) % 90 for i in range(150)], hq=4, hkv=1, seed=2)
    out, lse, want = run(b, which, window=20)
    check(b, want, out, lse, MARK)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("cache", ["16", "4"])
def test_long_contexts_in_ranges(cache, dtype):
    b = Batch(new=[1, 4, 2], past=[9000, 5001, 63], cache=cache, dtype=DT[dtype], page=64, seed=5)
    out, lse, want = run(b)
    check(b, want, out, lse, MARK)
    out, lse, want = run(b, "local", ret=[0], sink=5, window=4000)
    check(b, want, out, lse, MARK)


@pytest.mark.parametrize("cache", ["16", "4"])
@pytest.mark.parametrize("what", ["nan", "inf"])
def test_what_a_row_does_not_see_does_not_change_it(cache, what):
    """NaN and infinities in later tokens of the chunk, in slots behind the context, in pages that are not named, and before the window."""
    b = Batch(new=[40, 2], past=[100, 30], cache=cache, seed=6)
    plain, plain_lse, _ = run(b)
    x = math.nan if what == "nan" else math.inf
    seen = torch.zeros((b.n_pages, b.page), dtype=torch.bool)
    for s, n in enumerate(b.ctx):
        for t in range(n):
            seen[b.spot(s, t)] = True

    def spoil(where):
        for w in (0, 1):
            b.rows[w][:, where] = x
        if cache == "4":
            b.scale[:, :, where] = 255
    spoil(~seen)
    out, lse, want = run(b)
    check(b, want, out, lse, MARK)
    assert torch.equal(out, plain) and torch.equal(lse, plain_lse)
    late = torch.zeros_like(seen)
    late[b.spot(0, 125)] = True                        # rows 0 .. 24 of the first sequence are before it
    spoil(late)
    out, lse, want = run(b)
    hurt = {k: v for k, v in want.items() if 25 <= k[0] < 40}
    check(b, {k: v for k, v in want.items() if k not in hurt}, out, lse)
    if cache == "4" or what == "nan":
        assert all(torch.isnan(out[k]).all() for k in hurt)
    # before the window: position 125 is out of sight from 125 + 10 on
    out, lse, want = run(b, "local", sink=2, window=10)
    check(b, {k: v for k, v in want.items() if not 25 <= k[0] < 35}, out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("cache", ["16", "4"])
@pytest.mark.parametrize("new", [3, 5, 40])
def test_infinite_values_reach_the_rows_that_see_them(new, cache, dtype):
    """V of the last token of a draft, a short run and a chunk, infinite in three of four blocks; in 4 bits by a scale that the 16-bit type does not
    hold six times."""
    b = Batch(new=[new, 1], past=[100, 30], cache=cache, dtype=DT[dtype], seed=14 + new)
    page, slot = b.spot(0, b.ctx[0] - 1)
    b.rows[1][:, page, slot, 32:] = math.inf
    if cache == "4":
        b.code[1][:, page, slot, 32:] = 7
        b.scale[1][:, page, slot, 1:] = 253 if dtype == "bf16" else 141
    for which, kw in (("all", {}), ("local", dict(sink=3, window=30))):
        out, lse, want = run(b, which, **kw)
        hit = {k: v for k, v in want.items() if k[0] == new - 1}
        check(b, {k: v for k, v in want.items() if k not in hit}, out, lse)
        for k, (o, z, tol, tol_z) in hit.items():
            got = out[k].double().cpu()
            assert (got[32:] == math.inf).all()
            assert ((got[:32] - o[:32]).abs() <= tol[:32]).all() and abs(float(lse[k]) - z) <= tol_z


def test_large_logits_and_references():
    """Scores far from those of a range's first tile: sums that 32 bits do not hold against one reference."""
    for dtype in (torch.bfloat16, torch.float16):
        b = Batch(new=[30], past=[400], dtype=dtype, seed=7, gain=30.0)
        out, lse, want = run(b)
        check(b, want, out, lse, MARK)


def test_pages_that_are_not_there_are_left_out():
    b = Batch(new=[9, 3], past=[150, 40], seed=8)
    b.table[0, 2], b.table[0, 5], b.table[1, 0], b.table[1, 1], b.table[1, 2] = -1, b.n_pages, 1 << 30, -5, -1
    out, lse, want = run(b)
    check(b, want, out, lse, MARK)
    assert float(lse[b.off[1], 0]) == -math.inf
    out, lse, want = run(b, "local", sink=33, window=20)
    check(b, want, out, lse, MARK)


def test_positions_before_the_first_and_behind_the_table():
    b = Batch(new=[10, 4], past=None, ctx=[6, 40], seed=9)           # four rows have no position
    out, lse, want = run(b)
    check(b, want, out, lse, MARK)
    assert torch.isinf(lse[:4]).all() and (out[:4] == 0).all()
    q, cache, chunk = b.device()
    cache.pt_stride, chunk.max_ctx = 2, 32                           # (a table of 32 tokens; its second row is the first's third and fourth entry)
    b.table = b.table.flatten()[:4].view(2, 2)
    out, lse, want = run(b, prepared=(q, cache, chunk))
    check(b, want, out, lse, MARK)


@pytest.mark.parametrize("cache", ["16", "4"])
@pytest.mark.parametrize("new", [3, 40])
@pytest.mark.parametrize("sink,window", [(0, 8), (4, 16), (20, 200), (40, 0)])
def test_windows_behind_the_end_of_the_table(sink, window, new, cache):
    """Contexts that are longer than the table: what it does not hold is left out, and a band that lies behind it is empty."""
    b = Batch(new=[new, 1], past=[300, 500], seed=12, cache=cache)
    q, c, chunk = b.device()
    c.pt_stride, chunk.max_ctx = 2, 32
    b.table = b.table.flatten()[:4].view(2, 2)
    out, lse, want = run(b, "local", sink=sink, window=window, prepared=(q, c, chunk))
    check(b, want, out, lse, MARK)


@pytest.mark.parametrize("cache", ["16", "4"])
@pytest.mark.parametrize("new", [7, 40])
def test_the_largest_sinks_and_windows(new, cache):
    most = 2 ** 31 - 1
    b = Batch(new=[new, 1, 2], past=None, ctx=[new - 3, 700, 150], seed=13, cache=cache)       # (three rows have no position)
    for sink, window in ((0, most), (most, 0), (most, most)):
        out, lse, want = run(b, "local", sink=sink, window=window)
        check(b, want, out, lse, MARK)


def test_bounds_may_be_larger_than_what_is_there():
    b = Batch(new=[6, 1, 0], past=[70, 300, 9], seed=10)
    q, cache, chunk = b.device()
    exact, _, _ = run(b)
    big = rtp.rtp_chunk(chunk.q_offset, chunk.ctx_len, 3, b.total + 2, 1000, 16 * cache.pt_stride)
    big._keepalive = chunk._keepalive
    out, lse, want = run(b, prepared=(q, cache, big))
    check(b, want, out, lse, MARK)


def test_the_same_twice_and_from_a_graph():
    """Results do not depend on the run, nor on what the workspace held, nor on being replayed."""
    b = Batch(new=[33, 1, 5], past=[700, 3000, 90], seed=11)
    layer = _layer(b)
    q, cache, chunk = b.device()
    ws = torch.full((rtp.rtp_dense_attn_chunk_workspace_bytes(layer, 3, b.total, 33, 4096, rtp.RTP_HEADS_ALL),), 255, dtype=torch.uint8, device="cuda")
    out, lse, want = run(b, prepared=(q, cache, chunk), ws=ws)
    check(b, want, out, lse, MARK)
    for seed in (0, 90):
        ws.fill_(seed)
        again, lse2, _ = run(b, prepared=(q, cache, chunk), ws=ws)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
    o, z = torch.zeros_like(out), torch.zeros_like(lse)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        rtp.rtp_dense_attn_chunk(layer, q, q.stride(0), cache, chunk, rtp.RTP_HEADS_ALL, o, z, ws)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rtp.rtp_dense_attn_chunk(layer, q, q.stride(0), cache, chunk, rtp.RTP_HEADS_ALL, o, z, ws)
    for k in range(3):
        o.zero_()
        ws.fill_(k)
        chunk._keepalive[1][1] -= 7                                   # (contexts are the device's: the replay sees new ones)
        graph.replay()
        torch.cuda.synchronize()
        b.ctx[1] -= 7
        eager, lse3, want = run(b, prepared=(q, cache, chunk))
        check(b, want, o, z)
        assert torch.equal(o[:b.total], eager[:b.total]) and torch.equal(z[:b.total], lse3[:b.total])


@pytest.mark.parametrize("cache", ["16", "4"])
def test_rows_in_front_of_the_first_sequence(cache):
    """Offsets that begin behind the first row: the rows in front belong to no sequence.  Two sequences read the same pages."""
    b = Batch(new=[6, 0, 40], past=[70, 30, 300], cache=cache, seed=17)
    b.table[1, :6], b.ctx[1], b.new[1] = b.table[0, :6], 70, 2               # (one prompt, two drafts: the second's are the first's last ones)
    b.off, b.total = [2, 8, 10, 50], 50
    b.q = torch.randn((52, b.hq, 128), generator=torch.Generator().manual_seed(18)).to(b.dtype)
    q, c, chunk = b.device()
    out, lse, want = run(b, prepared=(q, c, chunk))
    check(b, want, out, lse, MARK)
    out, lse, want = run(b, "local", ret=[1], sink=3, window=40, prepared=(q, c, chunk))
    check(b, want, out, lse, MARK)
