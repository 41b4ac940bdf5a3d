"""The 4-bit format's oracle and the page model, pinned by hand; the entry points' refusals, all on the host."""
import ctypes as C

import numpy as np
import pytest

from oracle import kv4_oracle as k4
from pages_model import Pages
from paper_2605_16928_amd import rtp

A = 0x10000  # a fake, well-aligned, non-NULL "device pointer": argument checks fail before any use


# ---- oracle -----------------------------------------------------------------------------------------------------------------------
def _one_block(values):
    x = np.zeros(128)
    x[:len(values)] = values
    code, s = k4.quantise(x)
    return code[:len(values)].tolist(), int(s[0]) - 127, k4.values(code, s)[:len(values)].tolist()


def test_quantise_by_hand():
    # the largest magnitude sits in [3.5, 7) units of the block
    assert _one_block([6.0, 0.5, -1.0, 0.0]) == ([7, 1, 10, 0], 0, [6.0, 0.5, -1.0, 0.0])
    assert _one_block([6.99, 3.0])[1] == 0 and _one_block([7.0, 3.0])[1] == 1 and _one_block([3.5, 1.0])[1] == 0
    assert _one_block([3.49, 1.0])[1] == -1
    # halfway goes to the even code: 0.25 -> 0, 0.75 -> 1, 1.25 -> 1, 1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4
    assert _one_block([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])[2][1:] == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0]
    assert _one_block([-6.0, 0.26, -1.26, 5.01])[2] == [-6.0, 0.5, -1.5, 6.0]
    # each block has its own scale
    x = np.zeros(128)
    x[0], x[32], x[64] = 6.0, 6.0 * 2 ** -9, 1.0
    assert (k4.quantise(x)[1].astype(int) - 127).tolist() == [0, -9, -2, -125]
    assert np.array_equal(k4.values(*k4.quantise(x)), x)
    # what is not finite makes its block NaN, nothing else
    x[33] = np.inf
    v = k4.values(*k4.quantise(x))
    assert np.isnan(v[32:64]).all() and np.isfinite(v[:32]).all() and np.isfinite(v[64:]).all()


def test_quantise_is_within_half_a_step_and_idempotent():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((500, 128)) * np.exp(3 * rng.standard_normal((500, 1)))
    code, s = k4.quantise(x)
    v = k4.values(code, s)
    unit = np.repeat(np.exp2(s.astype(float) - 127), 32, axis=-1)
    a = np.abs(v) / unit
    step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))          # (the wider side: a value at 2 or 4 may come from above)
    assert (np.abs(v - x) <= step / 2 * unit).all()
    again = k4.values(*k4.quantise(v))
    np.testing.assert_array_equal(again, v)


def test_attend_and_positions_by_hand():
    q, k = np.zeros(128), np.zeros((3, 128))
    q[0], k[:, 0] = 2.0, [0.0, np.log(2.0), np.log(4.0)]
    v = np.eye(3, 128)
    out, lse, _, _ = k4.attend(q, k, v, 0.5)
    np.testing.assert_allclose(out[:3], np.array([1, 2, 4]) / 7, rtol=1e-12)
    assert abs(lse - np.log(7.0)) < 1e-12
    assert k4.attend(q, k[:0], v[:0], 0.5)[1] == -np.inf
    assert k4.local_positions(10, 2, 3).tolist() == [0, 1, 7, 8, 9]
    assert k4.local_positions(3, 4, 2).tolist() == [0, 1, 2] and k4.local_positions(6, 4, 5).tolist() == [0, 1, 2, 3, 4, 5]


def test_page_model_by_hand():
    m = Pages(3, 4, 8, 16)
    assert m.extend([0, 1], [0, 0], [33, 16]) == ([(-1, -1)] * 2, [0, 4])
    assert m.table.tolist() == [[0, 1, 2, -1], [3, -1, -1, -1], [-1] * 4]
    m.fork([0], [2], [33])
    assert m.refs.tolist() == [2, 2, 2, 1, 0, 0, 0, 0]
    assert m.extend([2, 0], [33, 33], [34, 33]) == ([(2, 4), (-1, -1)], [0, 3])
    assert m.table[2].tolist() == [0, 1, 4, -1] and m.refs.tolist() == [2, 2, 1, 1, 1, 0, 0, 0]
    assert m.extend([1], [16], [16 * 5 + 1])[1][0] == 2 + 0        # a row of 4 entries: two do not fit
    m.truncate([0], [16])
    assert m.refs.tolist() == [2, 1, 0, 1, 1, 0, 0, 0]
    assert m.compact() == ([(4, 2)], [4, 1])
    assert m.table.tolist() == [[0, -1, -1, -1], [3, -1, -1, -1], [0, 1, 2, -1]]


# ---- refusals ---------------------------------------------------------------------------------------------------------------------
def _layer(**kw):
    d = dict(n_q_heads=8, n_kv_heads=2, ret_heads=[0, 4], sink=4, window=64)
    d.update(kw)
    return rtp.layer_desc(**d)


def _cache(**kw):
    d = dict(codes=A, code_page_stride=64 * 128, code_head_stride=100 * 64 * 128, scales=A, scale_page_stride=64 * 8,
             scale_head_stride=100 * 64 * 8, page_table=A, pt_stride=16, page_size=64, n_pages=100)
    d.update(kw)
    return rtp.rtp_kv4_cache(**d)


BAD_CACHES = [("codes", None), ("scales", None), ("page_table", None), ("page_size", 8), ("page_size", 48), ("page_size", 1 << 21),
              ("n_pages", 0), ("pt_stride", 0), ("codes", A + 8), ("scales", A + 4), ("code_page_stride", 64 * 128 + 8),
              ("scale_head_stride", 100 * 64 * 8 + 4), ("code_page_stride", 64 * 128 - 16), ("code_page_stride", -64 * 128),
              ("code_head_stride", 99 * 64 * 128), ("scale_page_stride", 0), ("scale_head_stride", 64 * 8), ("code_head_stride", 0)]


def _refused(code, call, *a, **k):
    with pytest.raises(rtp.RtpError) as e:
        call(*a, **k)
    assert e.value.code == code, str(e.value)
    assert rtp.rtp_last_error() != ""


def _calls(layer=None, cache=None):
    layer, cache = layer or _layer(), cache or _cache()
    big = 1 << 30

    class Ws:                                  # a workspace that is large enough
        nbytes = big

        @staticmethod
        def data_ptr():
            return A
    return {
        "append": (rtp.rtp_kv4_append, dict(layer=layer, cache=cache, k=A, v=A, batch_stride=2560, token_stride=256, head_stride=128,
                                            start=A, count=A, B=3, T=10, stream=0)),
        "read": (rtp.rtp_kv4_read, dict(layer=layer, cache=cache, start=A, count=A, B=3, T=10, k=A, v=A, batch_stride=2560,
                                        token_stride=256, head_stride=128, stream=0)),
        "sparse": (rtp.rtp_sparse_attn_decode_kv4, dict(layer=layer, q=A, cache=cache, sel_idx=A, sel_stride=2000, sel_count=A,
                                                        max_sel=2000, B=3, out=A, lse=None, ws=Ws(), stream=0)),
        "local": (rtp.rtp_local_attn_kv4, dict(layer=layer, q=A, cache=cache, ctx_len=A, B=3, max_ctx=1024, out=A, lse=None, ws=Ws(),
                                               stream=0)),
        "dense": (rtp.rtp_dense_attn_kv4, dict(layer=layer, q=A, cache=cache, ctx_len=A, B=3, max_ctx=1024, out=A, lse=None, ws=Ws(),
                                               stream=0)),
    }


@pytest.mark.parametrize("name", ["append", "read", "sparse", "local", "dense"])
def test_cache_and_layer_are_checked(name):
    for field, value in BAD_CACHES:
        call, args = _calls(cache=_cache(**{field: value}))[name]
        _refused(rtp.RTP_ERR_INVALID_ARG, call, **args)
    call, args = _calls(cache=_cache(code_page_stride=1 << 37, code_head_stride=64 * 128))[name]
    _refused(rtp.RTP_ERR_UNSUPPORTED, call, **args)
    for bad, code in ((dict(head_dim=64), rtp.RTP_ERR_UNSUPPORTED), (dict(n_q_heads=32), rtp.RTP_ERR_UNSUPPORTED),
                      (dict(ret_heads=[4, 0]), rtp.RTP_ERR_INVALID_ARG), (dict(kv_dtype=2), rtp.RTP_ERR_UNSUPPORTED)):
        call, args = _calls(layer=_layer(**bad))[name]
        _refused(code, call, **args)


@pytest.mark.parametrize("name,field,value,code", [
    ("append", "k", None, -1), ("append", "v", A + 2, -1), ("append", "start", None, -1), ("append", "B", 0, -1), ("append", "T", -1, -1),
    ("append", "token_stride", 4, -1), ("append", "head_stride", -128, -1), ("append", "B", 1 << 30, -2),
    ("read", "k", None, -1), ("read", "v", A + 8, -1), ("read", "token_stride", 120, -1), ("read", "batch_stride", 1, -1), ("read", "T", 0, -1),
    ("sparse", "q", None, -1), ("sparse", "out", A + 8, -1), ("sparse", "sel_idx", None, -1), ("sparse", "sel_count", None, -1),
    ("sparse", "max_sel", 0, -1), ("sparse", "max_sel", (1 << 26) + 1, -1), ("sparse", "sel_stride", 1999, -1), ("sparse", "B", 0, -1),
    ("sparse", "B", 513, -2), ("sparse", "ws", None, -3),
    ("local", "q", A + 2, -1), ("local", "ctx_len", None, -1), ("local", "max_ctx", 0, -1), ("local", "max_ctx", 1025, -1),
    ("local", "B", -1, -1), ("local", "B", 1 << 20, -2),
    ("dense", "out", None, -1), ("dense", "ctx_len", None, -1), ("dense", "max_ctx", (1 << 26) + 1, -1), ("dense", "max_ctx", 1025, -1),
    ("dense", "ws", None, -3), ("dense", "B", 1 << 20, -2)])
def test_arguments_are_checked(name, field, value, code):
    call, args = _calls(cache=_cache(pt_stride=16))[name]
    if name in ("local", "dense") and field == "ws":
        args["max_ctx"], args["cache"] = 100000, _cache(pt_stride=2000)
    args[field] = value
    if field == "max_sel" and value > 2000:
        args["sel_stride"] = value
    _refused(code, call, **args)


def test_workspaces_are_checked():
    lib, layer, cache = rtp.lib(), _layer(), _cache(pt_stride=20000)
    vp = C.c_void_p
    for size, call in ((rtp.rtp_dense_attn_kv4_workspace_bytes(layer, 2, 1000000),
                        lambda ws, n: lib.rtp_dense_attn_kv4(C.byref(layer), vp(A), C.byref(cache), vp(A), 2, 1000000, vp(A), None, vp(ws), n, None)),
                       (rtp.rtp_sparse_attn_decode_kv4_workspace_bytes(layer, 2, 50000),
                        lambda ws, n: lib.rtp_sparse_attn_decode_kv4(C.byref(layer), vp(A), C.byref(cache), vp(A), 50000, vp(A), 50000, 2,
                                                                     vp(A), None, vp(ws), n, None))):
        assert size > 256
        assert call(A, size - 1) == rtp.RTP_ERR_WORKSPACE and call(A + 128, size) == rtp.RTP_ERR_WORKSPACE
        assert call(0, size) == rtp.RTP_ERR_WORKSPACE and b"workspace" in lib.rtp_last_error()
    # sizes of nonsense are small, not an error
    for B, n in ((1 << 30, 1000), (1 << 29, 1 << 40), (2, 1 << 40), (-1, 5), (4, 0)):
        assert rtp.rtp_dense_attn_kv4_workspace_bytes(layer, B, n) == 256 and rtp.rtp_local_attn_kv4_workspace_bytes(layer, B, n) == 256
        assert rtp.rtp_sparse_attn_decode_kv4_workspace_bytes(layer, B, n) == 256
    assert rtp.rtp_dense_attn_kv4_workspace_bytes(layer, 0, 100) == 256
    assert rtp.rtp_sparse_attn_decode_kv4_workspace_bytes(_layer(ret_heads=[]), 4, 100) == 256
    # no retrieval head / no local head: nothing to do, and nothing is asked for
    none = _layer(ret_heads=[])
    assert lib.rtp_sparse_attn_decode_kv4(C.byref(none), vp(A), C.byref(cache), vp(A), 4, vp(A), 4, 1, vp(A), None, None, 0, None) == rtp.RTP_OK
    every = _layer(ret_heads=list(range(8)))
    assert lib.rtp_local_attn_kv4(C.byref(every), vp(A), C.byref(cache), vp(A), 1, 64, vp(A), None, None, 0, None) == rtp.RTP_OK


def _map(**kw):
    d = dict(page_table=A, pt_stride=100, page_refs=A, n_seqs=4, n_pages=1000, page_size=64)
    d.update(kw)
    return rtp.rtp_page_map(**d)


class _Ws:
    nbytes = 1 << 20

    @staticmethod
    def data_ptr():
        return A


def _page_calls(m):
    return {
        "init": (rtp.rtp_kv_pages_init, dict(map=m, stream=0)),
        "extend": (rtp.rtp_kv_pages_extend, dict(map=m, seq=A, old_len=A, new_len=A, n=4, copy_src=A, copy_dst=A, status=A, ws=_Ws(), stream=0)),
        "fork": (rtp.rtp_kv_pages_fork, dict(map=m, src_seq=A, dst_seq=A, len=A, n=4, stream=0)),
        "truncate": (rtp.rtp_kv_pages_truncate, dict(map=m, seq=A, keep_len=None, n=4, stream=0)),
        "compact": (rtp.rtp_kv_pages_compact, dict(map=m, move_src=A, move_dst=A, status=A, ws=_Ws(), stream=0)),
    }


@pytest.mark.parametrize("name", ["init", "extend", "fork", "truncate", "compact"])
def test_page_maps_are_checked(name):
    for field, value, code in [("page_table", None, -1), ("page_refs", None, -1), ("pt_stride", 0, -1), ("n_seqs", 0, -1), ("n_pages", -1, -1),
                               ("page_size", 60, -1), ("page_size", 4, -1), ("n_pages", (1 << 26) + 1, -2), ("pt_stride", (1 << 26) + 1, -2)]:
        call, args = _page_calls(_map(**{field: value}))[name]
        _refused(code, call, **args)


@pytest.mark.parametrize("name,field,value,code", [
    ("extend", "seq", None, -1), ("extend", "old_len", None, -1), ("extend", "new_len", None, -1), ("extend", "copy_src", None, -1),
    ("extend", "copy_dst", None, -1), ("extend", "status", None, -1), ("extend", "n", 0, -1), ("extend", "n", 4097, -2), ("extend", "ws", None, -3),
    ("fork", "src_seq", None, -1), ("fork", "dst_seq", None, -1), ("fork", "len", None, -1), ("fork", "n", 65536, -1), ("fork", "n", 0, -1),
    ("truncate", "seq", None, -1), ("truncate", "n", 0, -1), ("truncate", "n", 65536, -1),
    ("compact", "move_src", None, -1), ("compact", "move_dst", None, -1), ("compact", "status", None, -1), ("compact", "ws", None, -3)])
def test_page_arguments_are_checked(name, field, value, code):
    call, args = _page_calls(_map())[name]
    args[field] = value
    _refused(code, call, **args)


def test_page_copies_are_checked():
    lib, vp = rtp.lib(), C.c_void_p

    def call(n_pools=1, n_pages=100, n=4, src=A, dst=A, **kw):
        d = dict(base=A, page_stride=4096, head_stride=409600, page_bytes=4096, n_heads=2)
        d.update(kw)
        pools = (rtp.rtp_page_pool * 1)(rtp.rtp_page_pool(**d))
        return lib.rtp_kv_pages_copy(pools, n_pools, n_pages, vp(src), vp(dst), n, None, None)
    for kw in (dict(src=None), dict(dst=None), dict(n_pools=0), dict(n_pages=0), dict(n=0), dict(base=None), dict(base=A + 8),
               dict(page_stride=4104), dict(head_stride=409608), dict(page_bytes=4100), dict(page_bytes=0), dict(page_bytes=(1 << 32) + 16),
               dict(n_heads=0), dict(n_heads=65536), dict(page_stride=4080), dict(head_stride=4096 * 99), dict(page_stride=-4096)):
        assert call(**kw) == rtp.RTP_ERR_INVALID_ARG and lib.rtp_last_error() != b"", kw
    assert lib.rtp_kv_pages_copy(None, 1, 100, vp(A), vp(A), 4, None, None) == rtp.RTP_ERR_INVALID_ARG


def test_descriptors_from_tensors():
    import torch
    codes = torch.zeros((2, 10, 16, 128), dtype=torch.uint8)
    scales = torch.zeros((2, 10, 128), dtype=torch.uint8)
    table = torch.zeros((3, 5), dtype=torch.int32)
    c = rtp.kv4_cache(codes, scales, table)
    assert (c.code_page_stride, c.code_head_stride, c.scale_page_stride, c.scale_head_stride) == (2048, 20480, 128, 1280)
    assert (c.pt_stride, c.page_size, c.n_pages) == (5, 16, 10)
    major = rtp.kv4_cache(codes.view(10, 2, 16, 128).transpose(0, 1), scales, table)
    assert (major.code_page_stride, major.code_head_stride) == (4096, 2048)
    for bad in ((codes[..., :64], scales, table), (codes.short(), scales, table), (codes, scales[:, :9], table), (codes, scales[..., :64], table),
                (codes, scales, table[:, :4]), (codes, scales, table.long()), (codes, scales, table[0]), (codes.transpose(2, 3), scales, table)):
        with pytest.raises(rtp.RtpError):
            rtp.kv4_cache(*bad)
    m = rtp.page_map(table, torch.zeros(10, dtype=torch.int32), 16)
    assert (m.pt_stride, m.n_seqs, m.n_pages, m.page_size) == (5, 3, 10, 16)
    with pytest.raises(rtp.RtpError):
        rtp.page_map(table[:, 1:], torch.zeros(10, dtype=torch.int32), 16)
    p = rtp.page_pools([codes, torch.zeros((10, 2, 8, 16), dtype=torch.bfloat16).transpose(0, 1)])
    assert (p[0].page_bytes, p[0].n_heads, p[1].page_stride, p[1].head_stride, p[1].page_bytes) == (2048, 2, 512, 256, 256) and p.n_pools == 2
    with pytest.raises(rtp.RtpError):
        rtp.page_pools([codes[:, :, :, ::2]])


@pytest.mark.parametrize("strides", [(0, 256, 128), (2560, 0, 128), (2560, 256, 0), (2560, 128, 128), (2560, 256, 120), (2432, 256, 128),
                                     (1280, 128, 1152), (1 << 62, 1 << 62, 128)])
def test_read_refuses_rows_that_overlap(strides):
    call, args = _calls()["read"]                       # 3 sequences of 10 tokens and 2 heads
    args.update(zip(("batch_stride", "token_stride", "head_stride"), strides))
    _refused(rtp.RTP_ERR_INVALID_ARG, call, **args)


def test_descriptors_refuse_other_types_devices_and_pools_that_are_too_small():
    import torch
    codes, scales = torch.zeros((2, 10, 16, 128), dtype=torch.uint8), torch.zeros((2, 10, 128), dtype=torch.uint8)
    table, refs = torch.zeros((3, 5), dtype=torch.int32), torch.zeros(10, dtype=torch.int32)
    elsewhere = torch.zeros((3, 5), dtype=torch.int32, device="meta")
    for make in (lambda: rtp.kv4_cache(codes, scales, table.float()), lambda: rtp.kv4_cache(codes, scales, elsewhere),
                 lambda: rtp.kv4_cache(codes, scales.to("meta"), table), lambda: rtp.page_map(table.float(), refs, 16),
                 lambda: rtp.page_map(table, refs.float(), 16), lambda: rtp.page_map(elsewhere, refs, 16),
                 lambda: rtp.page_pools([codes, scales.to("meta")])):
        with pytest.raises(rtp.RtpError):
            make()
    pools = rtp.page_pools([codes, scales[:, :8]])
    assert pools.n_pages == 8
    with pytest.raises(rtp.RtpError, match="n_pages"):
        rtp.rtp_kv_pages_copy(pools, 9, A, A, 4)


def test_workspaces_serve_smaller_calls():
    """What the size functions answer does not fall when the batch, the context or the selection grows."""
    for hq, hkv in ((8, 1), (8, 2), (32, 8), (64, 8), (16, 16)):
        layer = rtp.layer_desc(hq, hkv, [0, 1], 4, 8192)
        grid = [1, 2, 3, 5, 8, 15, 16, 17, 20, 25, 31, 32, 33, 40, 64, 65, 100, 128, 200, 255, 256, 257, 500, 512]
        lens = [1, 100, 1024, 1025, 1100, 3000, 5000, 9000, 12000, 13000, 20000, 40000, 131072, 1 << 20, 1 << 26]
        for size in (rtp.rtp_dense_attn_kv4_workspace_bytes, rtp.rtp_local_attn_kv4_workspace_bytes,
                     rtp.rtp_sparse_attn_decode_kv4_workspace_bytes):
            got = np.array([[size(layer, b, n) for n in lens] for b in grid])
            assert (got % 256 == 0).all() and got.min() >= 256
            assert (np.diff(got, axis=0) >= 0).all() and (np.diff(got, axis=1) >= 0).all(), (hq, hkv, size.__name__)


@pytest.mark.parametrize("name", ["append", "read", "sparse", "local", "dense"])
def test_calls_beyond_what_the_cache_holds_are_refused(name):
    """A pool with fewer KV heads than the layer, a page table with fewer rows than the batch: the strides alone allow both."""
    import torch
    codes, scales = torch.zeros((2, 10, 16, 128), dtype=torch.uint8), torch.zeros((2, 10, 128), dtype=torch.uint8)
    cache = rtp.kv4_cache(codes, scales, torch.zeros((3, 64), dtype=torch.int32))
    for layer, B in ((_layer(n_kv_heads=4), 3), (_layer(n_kv_heads=8), 1), (_layer(), 4), (_layer(n_kv_heads=1), 400)):
        call, args = _calls(layer=layer, cache=cache)[name]
        args["B"] = B
        with pytest.raises(rtp.RtpError, match="2 KV heads and 3 sequences") as e:
            call(**args)
        assert e.value.code == rtp.RTP_ERR_INVALID_ARG


@pytest.mark.parametrize("form", ["select_attend", "decode_attention", "step_one_stream", "make_ring", "ring_append", "local_attn_ring",
                                  "step", "step_two_streams", "select_then_attend"])
def test_forms_of_a_step_that_only_read_16_bits_are_refused(form):
    """What DecodeRun offers beside its plain step does not read the 4-bit cache behind the caller's back."""
    from paper_2605_16928_amd.pipeline import Kv4DecodeRun
    run = object.__new__(Kv4DecodeRun)                  # (refused before any buffer is looked at)
    args = {"ring_append": (None, None, None), "step": (True,), "step_two_streams": (None, True), "select_then_attend": (True,)}
    with pytest.raises(rtp.RtpError) as e:
        getattr(run, form)(*args.get(form, ()))
    assert e.value.code == rtp.RTP_ERR_UNSUPPORTED
    assert run.carries_local_heads is False             # step_fastest takes two streams


def test_nothing_to_do_asks_for_nothing():
    """No local head, no retrieval head: no workspace either, however long the contexts are."""
    lib, cache, vp = rtp.lib(), _cache(pt_stride=1 << 21), C.c_void_p
    every, none = _layer(ret_heads=list(range(8)), window=1 << 20), _layer(ret_heads=[])
    assert rtp.rtp_local_attn_kv4_workspace_bytes(every, 2, 1 << 26) > 256
    assert lib.rtp_local_attn_kv4(C.byref(every), vp(A), C.byref(cache), vp(A), 2, 1 << 26, vp(A), None, None, 0, None) == rtp.RTP_OK
    assert lib.rtp_sparse_attn_decode_kv4(C.byref(none), vp(A), C.byref(cache), vp(A), 1 << 20, vp(A), 1 << 20, 2, vp(A), None, None, 0,
                                          None) == rtp.RTP_OK


def test_largest_values_by_hand():
    """Where a block's maximum rounds up beyond the 16-bit types: 57344 and 1.75 * 2^127 are halfway between 3 and 4 steps."""
    assert _one_block([57312.0])[2] == [49152.0] and _one_block([57344.0])[2] == [65536.0] and _one_block([65504.0])[2] == [65536.0]
    top = 2.0 ** 127
    assert _one_block([1.7421875 * top])[2] == [1.5 * top] and _one_block([1.75 * top])[2] == [2 * top]


def test_a_page_that_all_its_holders_leave():
    """Every holder of a shared last page that grows takes a page; the one they leave is the next call's first, not this one's."""
    m = Pages(4, 3, 6, 16)
    assert m.extend([0], [0], [20]) == ([(-1, -1)], [0, 4])
    m.fork([0, 0], [1, 2], [20, 20])
    assert m.extend([0, 1, 2], [20] * 3, [21] * 3) == ([(1, 2), (1, 3), (1, 4)], [0, 1])
    assert m.refs.tolist() == [3, 0, 1, 1, 1, 0]
    assert m.extend([3], [0], [17]) == ([(-1, -1)], [0, 0]) and m.table[3].tolist() == [1, 5, -1]
    # three holders and two free pages: one is lacking
    m = Pages(4, 3, 4, 16)
    m.extend([0], [0], [20])
    m.fork([0, 0], [1, 2], [20, 20])
    assert m.extend([0, 1, 2], [20] * 3, [21] * 3) == ([(-1, -1)] * 3, [1, 2])


def test_decode_run_refuses_rows_that_are_laid_out_differently():
    """One set of strides goes to the library: K and V of different ones would be read from the wrong places."""
    import torch
    from paper_2605_16928_amd.pipeline import Kv4DecodeRun
    run = object.__new__(Kv4DecodeRun)
    run.desc = _layer()
    k, fused = torch.zeros((3, 2, 2, 128)), torch.zeros((3, 2, 12, 128))
    for bad in ((k, fused[:, :, 10:]), (k, k[:, :1]), (k.transpose(0, 1), k), (fused[:, :, 8:11], fused[:, :, 9:12]), (k[..., :64], k[..., :64]),
                (k.expand(3, 2, 2, 128)[..., :1].expand(3, 2, 2, 128),) * 2):
        with pytest.raises(rtp.RtpError) as e:
            run.append(*bad, None)
        assert e.value.code == rtp.RTP_ERR_INVALID_ARG


def test_decode_run_refuses_growth_before_it_hands_out_pages():
    import torch
    from paper_2605_16928_amd.pipeline import Kv4DecodeRun
    run = object.__new__(Kv4DecodeRun)                  # (no map, no buffers: what passed the checks would fail otherwise)
    run.desc, run.B, run.n_ret, run.len_most, run.len_limit = _layer(), 3, 2, [5, 9, 0], [9, 13, 4]
    k, keys = torch.zeros((3, 4, 2, 128)), torch.zeros((2, 3, 4, 16))
    for bad in ((k[:2], k[:2], keys), (k, k, keys[:, :2]), (k, k, keys[:, :, :1]), (k, k[:, :2], keys), (k[:, :0], k[:, :0], keys[:, :, :0]),
                (torch.zeros((3, 5, 2, 128)),) * 2 + (torch.zeros((2, 3, 5, 16)),)):
        with pytest.raises(rtp.RtpError) as e:
            run.grow(*bad)
        assert e.value.code == rtp.RTP_ERR_INVALID_ARG
