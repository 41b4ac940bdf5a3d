"""Calls over new tokens that their documentation allows and that nothing else makes: queries that are not numbers, caches beyond 32-bit
offsets, a whole step in one graph."""
import math

import pytest
import torch

import test_gpu_chunk_wide as wide
from chunk_bounds import check_rows
from chunk_util import Batch
from test_gpu_append import near, turned
from test_gpu_chunk import DT, MARK, run
from paper_2605_16928_amd import rtp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("cache", ["16", "4"])
@pytest.mark.parametrize("call", [run, wide.run], ids=["narrow", "wide"])
def test_queries_that_are_not_numbers(call, cache, dtype):
    """One head of one token: its row alone is not a number."""
    b = Batch(new=[40, 2], past=[300, 30], cache=cache, dtype=DT[dtype], seed=61)
    hurt = [(11, 3), (41, 6)]
    for value in (math.nan, math.inf):
        for i, h in hurt:
            b.q[i, h, 5] = value
        b.expected = lambda *a: {}
        for which, how in (("all", {}), ("local", dict(sink=3, window=50))):
            out, lse, _ = call(b, which, **how)
            rows = [(i, h) for i in (0, 10, 11, 12, 39, 40, 41) for h in range(8) if (i, h) not in hurt]
            check_rows(b, out, lse, rows, faint=0.0 if dtype == "bf16" else 2.0 ** -25, **how)
            for i, h in hurt:
                assert not torch.isfinite(out[i, h]).any() or value == math.inf
                assert not torch.isfinite(lse[i, h])


def _far(rows, page_stride):
    """The same pools with pages so many elements apart."""
    hkv, n_pages, page = rows.shape[1:4]
    out = []
    for w in (0, 1):
        store = torch.empty((n_pages - 1) * page_stride + hkv * page * 128, dtype=rows.dtype, device="cuda")
        x = store.as_strided((hkv, n_pages, page, 128), (page * 128, page_stride, 128, 1))
        x.copy_(rows[w])
        out.append(x)
    return out


@pytest.mark.parametrize("call", [run, wide.run], ids=["narrow", "wide"])
def test_caches_beyond_32_bits(call):
    """Pages 2^28 elements apart: the last ones lie 12 GiB behind the first."""
    b = Batch(new=[40, 1], past=[200, 90], hq=4, hkv=1, seed=63)
    K, V = _far(b.rows, 1 << 28)
    q, _, chunk = b.device()
    cache = rtp.kv_cache(K, V, b.table.cuda())
    for which, how in (("all", {}), ("local", dict(sink=3, window=50))):
        out, lse, want = call(b, which, prepared=(q, cache, chunk), **how)
        check_rows(b, out, lse, [(i, h) for i in range(0, 41, 4) for h in range(4)], **how)


def test_append_beyond_32_bits():
    b = Batch(new=[40, 7], past=[200, 90], hq=4, hkv=1, seed=64)
    K, V = _far(b.rows, 1 << 28)
    freq = (1e4 ** (-torch.arange(64) / 64)).float()
    layer = rtp.layer_desc(4, 1, [], 4, 64)
    qkv = torch.randn((47, 6, 128), generator=torch.Generator().manual_seed(65)).bfloat16()
    x, (_, _, chunk) = qkv.cuda(), b.device()
    rtp.rtp_kv_append(layer, rtp.kv_cache(K, V, b.table.cuda()), chunk, rtp.rope_desc(freq.cuda()), None, 0, x[:, 4:5], 768, x[:, 5:], 768, None, 0)
    for s in range(2):
        pos = torch.arange(b.ctx[s] - b.new[s], b.ctx[s])
        at, slot, mine = b.table[s, pos // 16].long().cuda(), (pos % 16).cuda(), slice(b.off[s], b.off[s + 1])
        want, size = turned(qkv[mine, 4:5], pos, freq, False, 1.0)
        near(K[0, at, slot], want[:, 0], size[:, 0], torch.bfloat16)
        assert torch.equal(V[0, at, slot].cpu(), qkv[mine, 5])


def test_a_step_from_a_graph():
    """Rotation, storing and both kinds of attention of a step, captured once: every replay takes the lengths, tokens and pages of the moment."""
    b = Batch(new=[30, 1, 0], past=[100, 400, 50], seed=66)
    layer = rtp.layer_desc(8, 2, [1, 6], 4, 40)
    q, cache, chunk = b.device()
    K, V, table = cache._keepalive
    freq = (1e4 ** (-torch.arange(64) / 64)).float()
    rope = rtp.rope_desc(freq.cuda())
    qkv = torch.zeros((b.total, 12, 128), dtype=torch.bfloat16, device="cuda")
    rotated, out, lse = torch.zeros_like(qkv[:, :8]).contiguous(), torch.zeros((b.total, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((b.total, 8), device="cuda")
    most = rtp.rtp_chunk(chunk.q_offset, chunk.ctx_len, 3, b.total, b.total, table.shape[1] * 16)
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (
        rtp.rtp_dense_attn_chunk_workspace_bytes(layer, 3, b.total, b.total, most.max_ctx, rtp.RTP_HEADS_RETRIEVAL),
        rtp.rtp_local_attn_chunk_workspace_bytes(layer, 3, b.total, b.total, most.max_ctx))]

    def step():
        rtp.rtp_kv_append(layer, cache, most, rope, qkv[:, :8], 1536, qkv[:, 8:10], 1536, qkv[:, 10:], 1536, rotated, 1024)
        rtp.rtp_dense_attn_chunk(layer, rotated, 1024, cache, most, rtp.RTP_HEADS_RETRIEVAL, out, lse, ws[0])
        rtp.rtp_local_attn_chunk(layer, rotated, 1024, cache, most, out, lse, ws[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    off, ctx = chunk._keepalive
    g = torch.Generator().manual_seed(67)
    for new, lens in (([30, 1, 0], [130, 401, 50]), ([0, 30, 1], [130, 380, 51]), ([1, 1, 1], [17, 33, 1])):
        b.new, b.ctx, b.off = new, lens, [0, new[0], new[0] + new[1], sum(new)]
        off.copy_(torch.tensor(b.off, dtype=torch.int32))
        ctx.copy_(torch.tensor(lens, dtype=torch.int32))
        fresh = torch.randn(qkv.shape, generator=g).bfloat16()
        qkv.copy_(fresh)
        for x in (out, lse):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        b.rows, b.q = torch.stack([K, V]).cpu(), rotated.cpu()
        for s in range(3):
            pos, mine = torch.arange(lens[s] - new[s], lens[s]), slice(b.off[s], b.off[s + 1])
            at, slot = b.table[s, pos // 16].long(), pos % 16
            near(b.q[mine], *turned(fresh[mine, :8], pos, freq, False, 1.0), torch.bfloat16)
            want, size = turned(fresh[mine, 8:10], pos, freq, False, 1.0)
            near(b.rows[0][:, at, slot], want.transpose(0, 1), size.transpose(0, 1), torch.bfloat16)
            assert torch.equal(b.rows[1][:, at, slot].transpose(0, 1), fresh[mine, 10:])
        rows = range(0, b.off[3], 3)
        check_rows(b, out, lse, [(i, h) for i in rows for h in (1, 6)], parts=2)
        check_rows(b, out, lse, [(i, h) for i in rows for h in (0, 2, 7)], parts=2, sink=4, window=40)
        assert (out[b.off[3]:] == 0).all() and (lse[b.off[3]:] == 0).all()
