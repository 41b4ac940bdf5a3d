"""Refusals of the calls over new tokens in a paged cache, all on the host."""
import ctypes as C
import math
import random

import pytest
import torch

from paper_2605_16928_amd import rtp

A = 0x10000  # a fake, well-aligned, non-NULL "device pointer": argument checks fail before any use


def _layer(**kw):
    d = dict(n_q_heads=8, n_kv_heads=2, ret_heads=[0, 4], sink=4, window=64)
    d.update(kw)
    return rtp.layer_desc(**d)


def _cache(**kw):
    d = dict(K=A, V=A, row_stride=128, page_stride=64 * 128, head_stride=100 * 64 * 128, page_table=A, pt_stride=32, page_size=64, n_pages=100)
    d.update(kw)
    return rtp.rtp_kv_cache(**d)


def _cache4(**kw):
    d = dict(codes=A, code_page_stride=64 * 128, code_head_stride=100 * 64 * 128, scales=A, scale_page_stride=64 * 8,
             scale_head_stride=100 * 64 * 8, page_table=A, pt_stride=32, page_size=64, n_pages=100)
    d.update(kw)
    return rtp.rtp_kv4_cache(**d)


def _chunk(**kw):
    d = dict(q_offset=A, ctx_len=A, B=3, total_q=50, max_q=20, max_ctx=2048)
    d.update(kw)
    return rtp.rtp_chunk(**d)


class Ws:                                      # a workspace that is large enough
    nbytes = 1 << 40

    @staticmethod
    def data_ptr():
        return A


QKV = 12 * 128


def _calls(layer=None, cache=None, chunk=None, cache4=None):
    layer, cache, chunk, cache4 = layer or _layer(), cache or _cache(), chunk or _chunk(), cache4 or _cache4()
    rope = rtp.rtp_rope(A, 128, 0, 0.0)
    attn = dict(layer=layer, q=A, q_stride=QKV, cache=cache, chunk=chunk, out=A + (1 << 30), lse=None, ws=Ws(), stream=0)
    return {
        "append": (rtp.rtp_kv_append, dict(layer=layer, cache=cache, chunk=chunk, rope=rope, q=A, q_stride=QKV, k=A + 2048, k_stride=QKV,
                                           v=A + 2560, v_stride=QKV, q_out=A + (1 << 30), q_out_stride=1024, stream=0)),
        "dense": (rtp.rtp_dense_attn_chunk, dict(attn, heads=rtp.RTP_HEADS_ALL)),
        "local": (rtp.rtp_local_attn_chunk, attn),
        "dense4": (rtp.rtp_dense_attn_chunk_kv4, dict(attn, cache=cache4, heads=rtp.RTP_HEADS_RETRIEVAL)),
        "local4": (rtp.rtp_local_attn_chunk_kv4, dict(attn, cache=cache4)),
    }


def _refused(code, call, **k):
    with pytest.raises(rtp.RtpError) as e:
        call(**k)
    assert e.value.code == code, str(e.value)
    assert rtp.rtp_last_error() != ""
    return str(e.value)


@pytest.mark.parametrize("name", ["append", "dense", "local", "dense4", "local4"])
def test_layers_and_batches_are_checked(name):
    for bad, code in ((dict(head_dim=64), -2), (dict(n_q_heads=32), -2), (dict(ret_heads=[4, 0]), -1), (dict(kv_dtype=2), -2)):
        call, args = _calls(layer=_layer(**bad))[name]
        _refused(code, call, **args)
    for bad, code in ((dict(q_offset=None), -1), (dict(ctx_len=None), -1), (dict(B=0), -1), (dict(B=65536), -2), (dict(total_q=-1), -1),
                      (dict(total_q=(1 << 24) + 1), -2), (dict(max_q=0), -1), (dict(max_ctx=0), -1), (dict(max_ctx=(1 << 30) + 1), -2),
                      (dict(max_ctx=32 * 64 + 1), -1)):
        call, args = _calls(chunk=_chunk(**bad))[name]
        _refused(code, call, **args)


@pytest.mark.parametrize("name", ["append", "dense", "local"])
@pytest.mark.parametrize("field,value", [
    ("K", None), ("V", None), ("page_table", None), ("page_size", 8), ("page_size", 48), ("page_size", 1 << 21), ("n_pages", 0), ("pt_stride", 0),
    ("K", A + 8), ("V", A + 2), ("row_stride", 120), ("row_stride", 132), ("row_stride", 1 << 25), ("page_stride", 64 * 128 + 4),
    ("page_stride", 63 * 128), ("page_stride", -64 * 128), ("head_stride", 99 * 64 * 128), ("head_stride", -128), ("head_stride", 0), ("head_stride", 64),
    ("page_stride", 1 << 41)])
def test_caches_are_checked(name, field, value):
    call, args = _calls(cache=_cache(**{field: value}))[name]
    _refused(rtp.RTP_ERR_INVALID_ARG, call, **args)


@pytest.mark.parametrize("name,field,value,code", [
    ("append", "k", None, -1), ("append", "v", None, -1), ("append", "q_out", None, -1), ("append", "q", A + 2, -1), ("append", "k", A + 8, -1),
    ("append", "q_out", A + (1 << 30) + 8, -1), ("append", "q_stride", 1016, -1), ("append", "q_stride", 1028, -1), ("append", "k_stride", 248, -1),
    ("append", "v_stride", QKV + 4, -1), ("append", "q_out_stride", 1000, -1), ("append", "q_out", A + 16, -1), ("append", "q_out", A + 1024, -1),
    ("append", "q_out", A, -1),
    ("dense", "q", None, -1), ("dense", "out", None, -1), ("dense", "q", A + 8, -1), ("dense", "out", A + (1 << 30) + 4, -1), ("dense", "q_stride", 1020, -1),
    ("dense", "q_stride", 512, -1), ("dense", "out", A, -1), ("dense", "out", A + 4096, -1), ("dense", "heads", 2, -1), ("dense", "lse", A + 2, -1),
    ("dense", "ws", None, -3), ("local", "ws", None, -3), ("local", "q_stride", -QKV, -1), ("dense4", "heads", -1, -1), ("local4", "out", None, -1)])
def test_arguments_are_checked(name, field, value, code):
    call, args = _calls()[name]
    args = dict(args)
    args[field] = value
    _refused(code, call, **args)


def test_rotations_are_checked():
    call, args = _calls()["append"]
    for rope, code in ((rtp.rtp_rope(None, 128, 0, 0.0), -1), (rtp.rtp_rope(A, 0, 0, 0.0), -2), (rtp.rtp_rope(A, 24, 0, 0.0), -2),
                       (rtp.rtp_rope(A, 144, 1, 0.0), -2), (rtp.rtp_rope(A, 64, 0, -1.0), -1), (rtp.rtp_rope(A, 64, 0, float("nan")), -1),
                       (rtp.rtp_rope(A, 64, 0, float("inf")), -1)):
        _refused(code, call, **dict(args, rope=rope))


def test_workspaces():
    lib, layer, cache = rtp.lib(), _layer(), _cache(pt_stride=1 << 20)
    vp = C.c_void_p
    for heads in (rtp.RTP_HEADS_ALL, rtp.RTP_HEADS_RETRIEVAL):
        for B, total, most, ctx in ((1, 1, 1, 100000), (100, 100, 1, 100000), (3, 5000, 4000, 1 << 20), (70, 300, 9, 64)):
            size = rtp.rtp_dense_attn_chunk_workspace_bytes(layer, B, total, most, ctx, heads)
            # a smaller call never asks for more
            for d in ((1, 1, 1, 1), (B, total // 2 or 1, most, ctx), (B, total, max(1, most // 3), ctx), (B, total, most, ctx // 2)):
                assert rtp.rtp_dense_attn_chunk_workspace_bytes(layer, *d, heads) <= size
            chunk = _chunk(B=B, total_q=total, max_q=most, max_ctx=ctx)

            def call(ws, n):
                return lib.rtp_dense_attn_chunk(C.byref(layer), vp(A), QKV, C.byref(cache), C.byref(chunk), heads, vp(A + (1 << 40)), None, vp(ws), n, None)
            if size > 256:
                assert call(A, size - 1) == call(A + 128, size) == call(0, size) == rtp.RTP_ERR_WORKSPACE
    for B, total, most, ctx in ((0, 1, 1, 1), (1, 0, 1, 1), (1, 1, 0, 1), (1, 1, 1, 0), (1 << 20, 1, 1, 1), (1, 1 << 30, 1, 1), (1, 1, 1, 1 << 40)):
        assert rtp.rtp_local_attn_chunk_workspace_bytes(layer, B, total, most, ctx) == 256
    # nothing to do, and nothing is asked for
    nothing = _chunk(total_q=0)
    assert lib.rtp_dense_attn_chunk(C.byref(layer), vp(A), QKV, C.byref(cache), C.byref(nothing), 0, vp(A + (1 << 40)), None, None, 0, None) == rtp.RTP_OK
    for lay, fn, extra in ((_layer(ret_heads=[]), lib.rtp_dense_attn_chunk, (1,)), (_layer(ret_heads=list(range(8))), lib.rtp_local_attn_chunk, ())):
        assert fn(C.byref(lay), vp(A), QKV, C.byref(cache), C.byref(_chunk()), *extra, vp(A + (1 << 40)), None, None, 0, None) == rtp.RTP_OK
    call, args = _calls(chunk=nothing)["append"]
    call(**args)


def test_descriptors_of_tensors():
    K, V = torch.zeros((2, 5, 16, 128), dtype=torch.bfloat16), torch.zeros((2, 5, 16, 128), dtype=torch.bfloat16)
    table = torch.zeros((3, 4), dtype=torch.int32)
    c = rtp.kv_cache(K, V, table)
    assert (c.row_stride, c.page_stride, c.head_stride, c.pt_stride, c.page_size, c.n_pages) == (128, 2048, 10240, 4, 16, 5)
    pages = torch.zeros((5, 16, 2, 128), dtype=torch.float16).permute(2, 0, 1, 3)
    c = rtp.kv_cache(pages, pages, table)
    assert (c.row_stride, c.page_stride, c.head_stride) == (256, 4096, 128)
    for bad in ((K, V[:1], table), (K, V.half(), table), (K.float(), V.float(), table), (K, pages.bfloat16(), table), (K[..., :64], V[..., :64], table),
                (K, V, table.long()), (K, V, table[0]), (K, V, table[:, ::2]), (K[:, :0], V[:, :0], table), (K, V.to("meta"), table)):
        with pytest.raises(rtp.RtpError):
            rtp.kv_cache(*bad)
    off, ctx = torch.zeros(4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    assert rtp.chunk_desc(off, ctx, 5, 3, 9).B == 3
    for bad in ((off[:3], ctx), (off.long(), ctx), (off, ctx.long()), (off[None], ctx), (off.to("meta"), ctx)):
        with pytest.raises(rtp.RtpError):
            rtp.chunk_desc(*bad, 5, 3, 9)
    for bad in (torch.zeros(4, dtype=torch.float64), torch.zeros((2, 4)), torch.zeros(8)[::2]):
        with pytest.raises(rtp.RtpError):
            rtp.rope_desc(bad)
    assert rtp.rope_desc(torch.zeros(32), True, 2.0).rotary_dim == 64


def test_calls_over_more_than_the_tensors_hold():
    K = torch.zeros((1, 5, 16, 128), dtype=torch.bfloat16)
    few_heads = rtp.kv_cache(K, K, torch.zeros((3, 200), dtype=torch.int32))
    few_seqs = rtp.kv_cache(K.expand(2, 5, 16, 128).contiguous(), K.expand(2, 5, 16, 128).contiguous(), torch.zeros((2, 200), dtype=torch.int32))
    for cache in (few_heads, few_seqs):
        for name in ("append", "dense", "local"):
            call, args = _calls(cache=cache)[name]
            with pytest.raises(rtp.RtpError) as e:
                call(**args)
            assert "a cache of" in str(e.value)


class Rows:
    """A tensor that says nothing of its device."""

    def __init__(self, t):
        self.shape, self.stride, self.element_size, self.data_ptr, self.numel, self.is_contiguous = t.shape, t.stride, t.element_size, (lambda: A), t.numel, t.is_contiguous


def test_tensors_lie_as_the_calls_take_them():
    """Tokens as far apart as the call says; outputs contiguous, log-sums contiguous in 32 bits."""
    fused, plain, short = (torch.zeros(n, dtype=torch.bfloat16) for n in ((50, 12, 128), (50, 8, 128), (49, 8, 128)))
    q = fused[:, :8]
    lse = torch.zeros((50, 8))
    for name in ("dense", "local", "dense4", "local4"):
        call, args = _calls()[name]
        for bad in (dict(q=Rows(q), q_stride=1024), dict(q=Rows(plain)), dict(q=Rows(short), q_stride=1024), dict(q=Rows(q.transpose(1, 2))), dict(q=Rows(q[:, :4])),
                    dict(q=Rows(q.float())), dict(out=Rows(q)), dict(out=Rows(short)), dict(out=Rows(torch.zeros((8, 50, 128), dtype=torch.half).transpose(0, 1))),
                    dict(lse=Rows(lse.half())), dict(lse=Rows(lse[:49])), dict(lse=Rows(torch.zeros((8, 50)).T)), dict(lse=Rows(torch.zeros((50, 12))[:, :8]))):
            with pytest.raises(rtp.RtpError, match="expected"):
                call(**dict(args, **bad))
    call, args = _calls()["append"]
    for bad in (dict(q=Rows(plain)), dict(k=Rows(plain[:, :2])), dict(v=Rows(fused[:, 10:]), v_stride=256), dict(q_out=Rows(q)), dict(k=Rows(fused[:, 8:])),
                dict(v=Rows(fused[:49, 10:]))):
        with pytest.raises(rtp.RtpError, match="expected"):
            call(**dict(args, **bad))


def test_a_workspace_serves_every_smaller_call():
    """Whichever tiles the smaller bounds are taken in."""
    rng = random.Random(4)
    for _ in range(400):
        hq, hkv = rng.choice([(8, 2), (32, 8), (64, 8), (16, 16), (4, 1)])
        layer = _layer(n_q_heads=hq, n_kv_heads=hkv, ret_heads=sorted(rng.sample(range(hq), 2)), window=rng.choice([0, 16, 500, 8192]))
        bounds = [int(2 ** rng.uniform(0, top)) for top in (8, 13, 12, 18)]
        less = [int(2 ** rng.uniform(0, math.log2(n))) for n in bounds]
        for size in (lambda *b: rtp.rtp_local_attn_chunk_workspace_bytes(layer, *b), lambda *b: rtp.rtp_dense_attn_chunk_workspace_bytes(layer, *b, 0),
                     lambda *b: rtp.rtp_dense_attn_chunk_workspace_bytes(layer, *b, 1)):
            assert size(*less) <= size(*bounds), (hq, hkv, less, bounds)
