"""Attention of batches of new tokens in tiles of 256 rows: the cases of test_gpu_chunk.py under bounds of so many tokens that the calls take those
tiles, which their own bounds are too small for."""
import pytest
import torch

import test_gpu_chunk as small
from chunk_util import Batch, check
from paper_2605_16928_amd import rtp
from test_gpu_chunk import (test_any_number_of_served_heads, test_dense, test_head_layouts, test_infinite_values_reach_the_rows_that_see_them,  # noqa: F401
                            test_large_logits_and_references, test_local, test_long_contexts_in_ranges, test_many_sequences, test_pages_and_layouts,
                            test_pages_that_are_not_there_are_left_out, test_positions_before_the_first_and_behind_the_table,
                            test_the_largest_sinks_and_windows, test_what_a_row_does_not_see_does_not_change_it, test_windows_behind_the_end_of_the_table)

pytestmark = pytest.mark.gpu
run_small = small.run


def run(b, which="all", ret=(), sink=4, window=64, lse=True, prepared=None):
    q, cache, chunk = prepared or b.device()
    n = 18000 if b.hq <= 16 else 5000
    many = torch.zeros((n, b.hq, 128), dtype=b.dtype, device="cuda")
    many[:b.total] = q[:b.total]
    big = rtp.rtp_chunk(chunk.q_offset, chunk.ctx_len, chunk.B, n, n, chunk.max_ctx)
    big._keepalive = chunk._keepalive
    total, b.total = b.total, n - 2
    try:
        out, z, want = run_small(b, which, ret, sink, window, lse, (many, cache, big))
    finally:
        b.total = total
    assert (out[total + 2:] == small.MARK).all() and (z is None or (z[total + 2:] == small.MARK).all())
    return out[:total + 2], None if z is None else z[:total + 2], want


@pytest.fixture(autouse=True)
def many_tokens(monkeypatch):
    monkeypatch.setattr(small, "run", run)


def _launches(call):
    rtp.rtp_profile_start(64)
    call()
    torch.cuda.synchronize()
    return " ".join(name for name, _ in rtp.rtp_profile_stop())


@pytest.mark.parametrize("cache", ["16", "4"])
def test_either_kind_of_tile(cache):
    """Few tokens go in tiles of 32 rows, over long contexts in ranges of them; under bounds of many tokens in wide ones."""
    b = Batch(new=[40, 2], past=[100, 30], cache=cache, seed=6)
    assert "narrow" in _launches(lambda: run_small(b)) and "chunk_attn" in _launches(lambda: run(b))
    b = Batch(new=[150], past=[20000], hq=4, hkv=1, page=64, cache=cache, seed=15)
    for call in (run_small, run):
        out, lse, want = call(b, which="ret", ret=[0, 2])
        check(b, want, out, lse, small.MARK)


@pytest.mark.parametrize("cache", ["16", "4"])
@pytest.mark.parametrize("spoiled", [False, True], ids=["plain", "taken_again"])
def test_from_a_graph(spoiled, cache):
    """Replays see the device's contexts of the moment, whatever the workspace held, also where tiles are taken again."""
    b = Batch(new=[33, 1, 70], past=[700, 3000, 90], cache=cache, seed=16)
    if spoiled:
        b.table[0, 3] = -1
    layer = rtp.layer_desc(b.hq, b.hkv, [], 4, 64)
    q, c, chunk = b.device()
    n = 18000
    many = torch.zeros((n, b.hq, 128), dtype=b.dtype, device="cuda")
    many[:b.total] = q[:b.total]
    big = rtp.rtp_chunk(chunk.q_offset, chunk.ctx_len, chunk.B, n, n, chunk.max_ctx)
    attend = rtp.rtp_dense_attn_chunk if cache == "16" else rtp.rtp_dense_attn_chunk_kv4
    ws = torch.empty(rtp.rtp_dense_attn_chunk_workspace_bytes(layer, 3, n, n, chunk.max_ctx, rtp.RTP_HEADS_ALL), dtype=torch.uint8, device="cuda")
    outs = [(torch.zeros((n, b.hq, 128), dtype=b.dtype, device="cuda"), torch.zeros((n, b.hq), device="cuda")) for _ in range(2)]

    def call(out, lse):
        attend(layer, many, many.stride(0), c, big, rtp.RTP_HEADS_ALL, out, lse, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(*outs[0])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*outs[0])
    for k in range(3):
        for x in outs[0]:
            x.zero_()
        ws.fill_(85 * k)
        chunk._keepalive[1][1] -= 7
        b.ctx[1] -= 7
        graph.replay()
        torch.cuda.synchronize()
        call(*outs[1])
        check(b, b.expected(range(b.hq)), outs[0][0][:b.total], outs[0][1][:b.total])
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
