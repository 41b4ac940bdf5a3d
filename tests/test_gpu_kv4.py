"""The 4-bit K/V cache on the GPU: what append stores and read gives back, bit by bit, and decode attention over it against 64 bits."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as k4
from paper_2605_16928_amd import rtp
from gpu_util import DEV, i32, launches, ws_alloc
from kv4_util import EPS, TYPES, Cache, check_row, queries

pytestmark = pytest.mark.gpu


def _layer(hq, hkv, ret, dtype="bf16", sink=4, window=64):
    return rtp.layer_desc(hq, hkv, ret, sink, window, kv_dtype=rtp.RTP_DTYPE_FP16 if dtype == "fp16" else rtp.RTP_DTYPE_BF16)


# ---- store -----------------------------------------------------------------------------------------------------------------------
def _special_rows(dtype):
    """Rows that meet every rounding case: all finite 16-bit values as multiples of their block's scale, zeros, the smallest and largest
    values, infinities and NaN."""
    t = TYPES[dtype]
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(t)
    finite = bits[bits.isfinite()]
    rows = [finite[torch.randperm(len(finite), generator=torch.Generator().manual_seed(i))][:finite.numel() // 128 * 128].view(-1, 128)
            for i in range(2)]
    # halfway points and their neighbours, under a maximum of 6 and of just under 7 units
    y = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 6.9375, 0.0, -0.0])
    y = torch.cat([y, y * (1 + 2.0 ** -7), y * (1 - 2.0 ** -8), -y])[:32]
    for e in (-9, 0, 7):
        for top in (6.0, 6.9375, 7.0, 4.0, 3.4375):
            b = y * 2.0 ** e
            b[0] = top * 2.0 ** e
            rows.append(b.clamp(-top * 2.0 ** e, top * 2.0 ** e).repeat(4).to(t).view(1, 128))
    odd = torch.zeros((6, 128), dtype=t)
    odd[0, 5] = float("inf")
    odd[1, 40] = float("nan")
    odd[2, 127] = float("-inf")
    odd[3, 64] = torch.finfo(t).max
    odd[4, 33] = torch.finfo(t).smallest_normal
    odd[5, 3] = torch.tensor([1], dtype=torch.int16).view(t)[0]          # the smallest subnormal
    return torch.cat(rows + [odd])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_append_and_read_every_value(dtype):
    print(f"[case] kv4 store, all values, {dtype}", flush=True)
    x = _special_rows(dtype)
    T, ps = x.shape[0], 64
    n_pages = -(-T // ps) + 1
    codes = torch.full((1, n_pages, ps, 128), 0xAA, dtype=torch.uint8, device=DEV)
    scales = torch.full((1, n_pages, ps * 8), 0x55, dtype=torch.uint8, device=DEV)
    table = torch.randperm(n_pages, generator=torch.Generator().manual_seed(3)).int()[None].to(DEV)
    cache, layer = rtp.kv4_cache(codes, scales, table), _layer(1, 1, [], dtype)
    k, v = x.view(1, T, 1, 128).to(DEV), x.flip(0).contiguous().view(1, T, 1, 128).to(DEV)
    rtp.rtp_kv4_append(layer, cache, k, v, T * 128, 128, 128, i32([0]), None, 1, T)
    ko, vo = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    rtp.rtp_kv4_read(layer, cache, i32([0]), None, 1, T, ko, vo, T * 128, 128, 128)
    torch.cuda.synchronize()
    code, s = k4.quantise(x.double().numpy())
    want = k4.values(code, s)
    kc, _ = k4.rows_of(codes.cpu().numpy()[0], scales.cpu().numpy()[0], table.cpu().numpy()[0], ps, np.arange(T))
    np.testing.assert_array_equal(kc, want)
    want16 = torch.from_numpy(want).to(TYPES[dtype]).double().numpy()
    np.testing.assert_array_equal(ko.double().cpu().numpy()[0, :, 0], want16)
    np.testing.assert_array_equal(vo.double().cpu().numpy()[0, :, 0], want16[::-1])
    # within the codes' precision of what was stored: half a step, a quarter of the block's maximum at most ((4 + 6) / 2 - 4 of 4)
    fin = np.isfinite(want).all(-1)
    blocks = x.double().numpy()[fin].reshape(-1, 4, 32)
    err = np.abs(want[fin].reshape(-1, 4, 32) - blocks)
    assert (err <= np.maximum(np.abs(blocks).max(-1, keepdims=True) * 0.25, 2.0 ** -127)).all()


@pytest.mark.parametrize("dtype,page_size,page_major", [("bf16", 16, False), ("fp16", 64, True), ("bf16", 256, True)])
def test_append_touches_its_positions_only(dtype, page_size, page_major):
    """Ragged starts and counts in a strided projection output: every byte of the pool is the old one or what the oracle stores."""
    print(f"[case] kv4 append, ragged, page size {page_size}", flush=True)
    rng = np.random.default_rng(5)
    H, B, T = 3, 7, 37
    start = [0, 1, 14, 30, -1, 63, 5]
    count = [37, 1, 19, 50, 9, 0, 2]                  # 50: cut to T; -1: skipped
    c = Cache(rng, H, [100] * B, page_size, page_major)
    old_codes, old_scales = c.codes.copy(), c.scales.reshape(H, c.P, page_size // 4, 2, 4, 4).copy()
    qkv = torch.from_numpy(rng.standard_normal((B, T, 4 + 2 * H, 128))).to(TYPES[dtype]).to(DEV)
    k, v = qkv[:, :, 4:4 + H], qkv[:, :, 4 + H:]
    layer = _layer(H * 2, H, [], dtype)
    rtp.rtp_kv4_append(layer, c.desc, k, v, k.stride(0), k.stride(1), k.stride(2), i32(start), i32(count), B, T)
    torch.cuda.synchronize()
    for b in range(B):
        n = 0 if start[b] < 0 else min(count[b], T)
        for t in range(n):
            page, slot = divmod(start[b] + t, page_size)
            page = c.table[b, page]
            for w, x in ((0, k), (1, v)):
                code, s = k4.quantise(x[b, t].double().cpu().numpy())
                old_codes[:, page, slot, 64 * w:64 * w + 64] = code[:, 0::2] | (code[:, 1::2] << 4)
                old_scales[:, page, slot // 4, w, :, slot % 4] = s
    np.testing.assert_array_equal(c.codes_d.cpu().numpy(), old_codes)
    np.testing.assert_array_equal(c.scales_d.cpu().numpy(), old_scales.reshape(H, c.P, -1))
    # read back with other strides (head-major), unaligned starts, rows behind the counts left alone
    first, rd = [3, 0, 15, 29, 0, -2, 99], [40, 100, 18, 0, 1, 5, 1]
    R = 41
    ko, vo = (torch.full((H, B, R, 128), 9.0, dtype=TYPES[dtype], device=DEV) for _ in range(2))
    rtp.rtp_kv4_read(layer, c.desc, i32(first), i32(rd), B, R, ko, vo, R * 128, 128, B * R * 128)
    torch.cuda.synchronize()
    c.codes, c.scales = old_codes, old_scales.reshape(H, c.P, -1)
    for b in range(B):
        n = 0 if first[b] < 0 else min(rd[b], R)
        for h in range(H):
            rows = c.rows(b, h, first[b] + np.arange(n)) if n else (np.zeros((0, 128)),) * 2
            for got, want in zip((ko, vo), rows):
                g = got[h, b].double().cpu().numpy()
                np.testing.assert_array_equal(g[:n], torch.from_numpy(want).to(TYPES[dtype]).double().numpy())
                assert (g[n:] == 9.0).all()


def test_store_follows_no_page_outside_the_pool():
    """Entries of -1, of n_pages and beyond, and positions behind the table: nothing is stored, zeros come back."""
    print("[case] kv4 store, pages outside the pool", flush=True)
    rng = np.random.default_rng(6)
    c = Cache(rng, 2, [64, 64], 16)
    c.table[0, 1], c.table[0, 2], c.table[1, 3] = -1, c.P, 2 ** 31 - 1
    c.table_d.copy_(torch.from_numpy(c.table))
    before = c.codes_d.clone(), c.scales_d.clone()
    k = torch.ones((2, 80, 2, 128), dtype=torch.bfloat16, device=DEV)
    layer = _layer(2, 2, [])
    rtp.rtp_kv4_append(layer, c.desc, k[:, :32], k[:, :32], k.stride(0), k.stride(1), k.stride(2), i32([16, 48]), i32([32, 32]), 2, 32)
    ko, vo = torch.full_like(k, 5.0), torch.full_like(k, 5.0)
    rtp.rtp_kv4_append(layer, c.desc, k, k, k.stride(0), k.stride(1), k.stride(2), i32([2 ** 31 - 40, 1 << 20]), None, 2, 80)
    torch.cuda.synchronize()
    assert torch.equal(c.codes_d, before[0]) and torch.equal(c.scales_d, before[1])
    rtp.rtp_kv4_read(layer, c.desc, i32([0, 0]), None, 2, 80, ko, vo, k.stride(0), k.stride(1), k.stride(2))
    torch.cuda.synchronize()
    for b, bad in ((0, range(16, 48)), (1, range(48, 64))):
        for t in range(80):
            z = t in bad or t >= 64
            for h in range(2):
                want = np.zeros(128) if z else c.rows(b, h, [t])[0][0]
                np.testing.assert_array_equal(ko[b, t, h].double().cpu().numpy(), want)


# ---- attention --------------------------------------------------------------------------------------------------------------------
def _dense(layer, q, c, ctx, max_ctx=None, what="dense"):
    B, Hq = q.shape[:2]
    max_ctx = max_ctx or max(max(ctx), 1)
    size, call = (rtp.rtp_dense_attn_kv4_workspace_bytes, rtp.rtp_dense_attn_kv4) if what == "dense" else \
        (rtp.rtp_local_attn_kv4_workspace_bytes, rtp.rtp_local_attn_kv4)
    ws = ws_alloc(size(layer, B, max_ctx))
    ws.fill_(0xff)
    out = torch.full_like(q, 3.0)
    lse = torch.full((B, Hq), 3.0, dtype=torch.float32, device=DEV)
    call(layer, q, c.desc, i32(ctx), B, max_ctx, out, lse, ws)
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


LENS = [1, 15, 16, 17, 31, 33, 0, 255, 257, 1000]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("hq,hkv,page_size", [(2, 2, 16), (4, 2, 64), (8, 2, 32), (16, 2, 256)])
def test_dense_attention(hq, hkv, page_size, dtype):
    print(f"[case] kv4 dense, {hq}/{hkv} heads, page {page_size}, {dtype}", flush=True)
    rng = np.random.default_rng(hq)
    c = Cache(rng, hkv, LENS, page_size, page_major=hq == 4)
    q, qd = queries(rng, len(LENS), hq, dtype)
    out, lse = _dense(_layer(hq, hkv, [0], dtype), q, c, LENS)
    for b, n in enumerate(LENS):
        for h in range(hq):
            k, v = c.rows(b, h // (hq // hkv), np.arange(n))
            check_row(out[b, h], lse[b, h], qd[b, h], k, v, dtype, what=f"n {n}, head {h}")


@pytest.mark.parametrize("sink,window", [(4, 64), (0, 1), (17, 16), (20, 0), (4, 500), (1, 15), (40, 33)])
def test_local_attention(sink, window):
    print(f"[case] kv4 local, sink {sink}, window {window}", flush=True)
    rng = np.random.default_rng(window)
    hq, hkv, ret = 8, 4, [0, 1, 4]                     # KV head 0 serves retrieval heads only, KV head 2 one of each
    c = Cache(rng, hkv, LENS, 16)
    q, qd = queries(rng, len(LENS), hq, "bf16")
    out, lse = _dense(_layer(hq, hkv, ret, sink=sink, window=window), q, c, LENS, what="local")
    for b, n in enumerate(LENS):
        for h in range(hq):
            if h in ret:
                assert (out[b, h] == 3.0).all() and lse[b, h] == 3.0
                continue
            k, v = c.rows(b, h // 2, k4.local_positions(n, sink, window))
            check_row(out[b, h], lse[b, h], qd[b, h], k, v, "bf16", what=f"n {n}, head {h}")


@pytest.mark.parametrize("size", [0.0, 20.0])
@pytest.mark.parametrize("what,n,B", [("dense", 70001, 1), ("local", 70001, 2), ("dense", 9000, 3)])
def test_long_contexts_and_wide_logits(what, n, B, size):
    """Many splits to merge; logits that are all equal, and logits that differ by hundreds, so that the running maximum moves."""
    print(f"[case] kv4 {what}, {n} tokens, queries of size {size}", flush=True)
    rng = np.random.default_rng(n)
    hq, hkv = 8, 2
    lens = [n] + [n // 3 + 5 * b for b in range(1, B)]
    c = Cache(rng, hkv, lens, 64)
    q, qd = queries(rng, B, hq, "bf16", size)
    out, lse = _dense(_layer(hq, hkv, [], sink=4, window=8192), q, c, lens, what=what)
    for b in range(B):
        pos = np.arange(lens[b]) if what == "dense" else k4.local_positions(lens[b], 4, 8192)
        for kvh in range(hkv):
            k, v = c.rows(b, kvh, pos)
            for h in range(kvh * 4, kvh * 4 + 4):
                check_row(out[b, h], lse[b, h], qd[b, h], k, v, "bf16", what=f"sequence {b}, head {h}")


@pytest.mark.parametrize("B,hkv,group,lens", [
    (34, 4, 8, "equal"), (34, 4, 4, "one long"), (20, 8, 8, "any"), (40, 8, 1, "near"), (40, 8, 2, "any"), (256, 1, 2, "equal"),
    (256, 1, 8, "one long"), (256, 1, 4, "empty"), (130, 8, 2, "one long"), (2, 8, 4, "one long")])
def test_many_units_are_shared_out(B, hkv, group, lens):
    """More (sequence, KV head) pairs than half of the compute units, with contexts that may be long: equal lengths, about equal ones,
    one long context among short ones, any, none at all."""
    print(f"[case] kv4 dense, {B} sequences, {hkv} KV heads of {group}, {lens}", flush=True)
    rng = np.random.default_rng(B + group)
    max_ctx = 16 * (B * hkv + 48) + 600
    ctx = {"equal": [700] * B, "near": [int(x) for x in rng.integers(610, 700, B)], "any": [int(x) for x in rng.integers(0, 900, B)],
           "one long": [max_ctx - 3 if b == B // 2 else int(x) for b, x in enumerate(rng.integers(1, 200, B))], "empty": [0] * B}[lens]
    c = Cache(rng, hkv, ctx, 64)
    c.table = np.pad(c.table, ((0, 0), (0, max(0, -(-max_ctx // 64) - c.table.shape[1]))), constant_values=-1)
    c.upload()
    q, qd = queries(rng, B, hkv * group, "bf16")
    out, lse = _dense(_layer(hkv * group, hkv, []), q, c, ctx, max_ctx=max_ctx)
    for b in sorted({0, 1, B // 2, B - 1} | {int(x) for x in rng.integers(0, B, 6)}):
        for kvh in range(hkv):
            k, v = c.rows(b, kvh, np.arange(ctx[b]))
            for h in range(kvh * group, kvh * group + group):
                check_row(out[b, h], lse[b, h], qd[b, h], k, v, "bf16", what=f"sequence {b}, head {h}")
    assert np.isfinite(out).all() and (lens == "empty" or np.isfinite(lse[np.array(ctx) > 0]).all())


@pytest.mark.parametrize("B,hkv,ret,lens", [(20, 8, [0, 3, 4, 5], "any"), (40, 8, [1, 2, 3], "equal"), (256, 1, [], "one long")])
def test_many_windows_are_shared_out(B, hkv, ret, lens):
    """The same for sinks and windows, where heads and whole KV heads are not the call's."""
    print(f"[case] kv4 local, {B} sequences, {hkv} KV heads, {lens}", flush=True)
    rng = np.random.default_rng(B)
    hq, sink, window = 2 * hkv, 20, 16 * (B * hkv + 48) + 100 if hkv > 1 else 13000
    ctx = {"equal": [900] * B, "any": [int(x) for x in rng.integers(0, 900, B)],
           "one long": [window + 700 if b == 5 else int(x) for b, x in enumerate(rng.integers(1, 200, B))]}[lens]
    max_ctx = window + 1000
    c = Cache(rng, hkv, ctx, 64)
    c.table = np.pad(c.table, ((0, 0), (0, max(0, -(-max_ctx // 64) - c.table.shape[1]))), constant_values=-1)
    c.upload()
    q, qd = queries(rng, B, hq, "bf16")
    out, lse = _dense(_layer(hq, hkv, ret, sink=sink, window=window), q, c, ctx, max_ctx=max_ctx, what="local")
    for b in sorted({0, 5, B - 1} | {int(x) for x in rng.integers(0, B, 6)}):
        for h in range(hq):
            if h in ret:
                assert (out[b, h] == 3.0).all() and lse[b, h] == 3.0
                continue
            k, v = c.rows(b, h // 2, k4.local_positions(ctx[b], sink, window))
            check_row(out[b, h], lse[b, h], qd[b, h], k, v, "bf16", what=f"sequence {b}, head {h}")


@pytest.mark.parametrize("lens", ["full", "half", "any", "one", "empty"])
@pytest.mark.parametrize("B,hkv,group,whole", [(29, 8, 2, True), (32, 8, 4, True), (58, 8, 1, True), (120, 2, 8, True), (20, 8, 2, False), (33, 8, 2, False)])
def test_windows_where_whole_units_fill_their_rounds(B, hkv, group, whole, lens):
    """Just under 256 or 512 units with windows of 8192 stay whole, one launch; other numbers of units are shared out.  All sequences read
    one context's pages, as forks of it do."""
    print(f"[case] kv4 local, {B} sequences, {hkv} KV heads of {group}, {lens}", flush=True)
    rng = np.random.default_rng(B)
    window, sink, longest = 8192, 20, 9001
    c = Cache(rng, hkv, [longest], 64)
    c.table = np.repeat(c.table, B, axis=0)
    c.upload()
    full = [int(x) for x in rng.integers(window, longest + 1, B)]
    short = [int(x) for x in rng.integers(0, window, B)]
    ctx = {"full": full, "half": [x for pair in zip(full, short) for x in pair][:B], "any": short,
           "one": [longest if b == B // 3 else x % 500 for b, x in enumerate(short)], "empty": [0] * B}[lens]
    hq, ret = hkv * group, [1, group * (hkv - 1)] + ([group * hkv - 1] if group > 1 else [])
    layer = _layer(hq, hkv, ret, sink=sink, window=window)
    q, qd = queries(rng, B, hq, "bf16")
    results = []
    names = launches(lambda: results.append(_dense(layer, q, c, ctx, max_ctx=longest, what="local")))
    assert len(names) == (1 if whole else 2), names
    out, lse = results[0]
    for b in sorted({0, 1, B // 3, B - 1} | {int(x) for x in rng.integers(0, B, 3)}):
        pos = k4.local_positions(ctx[b], sink, window)
        for kvh in range(hkv):
            k, v = c.rows(b, kvh, pos)
            for h in range(kvh * group, kvh * group + group):
                if h in ret:
                    assert (out[b, h] == 3.0).all() and lse[b, h] == 3.0
                else:
                    check_row(out[b, h], lse[b, h], qd[b, h], k, v, "bf16", what=f"sequence {b}, head {h}")
    assert np.isfinite(out).all() and (lens == "empty" or np.isfinite(lse[np.array(ctx) > 0]).all())


def _sparse(layer, q, c, sel, max_sel=None, n_ret=1):
    B, Hq = q.shape[:2]
    counts = [len(s) for s in sel]
    max_sel = max_sel or max(max(counts), 1)
    stride = max(max(counts), max_sel) + 3             # (rows of the index list start anywhere)
    idx = np.full((len(sel), stride), -2 ** 31, dtype=np.int32)
    for r, s in enumerate(sel):
        idx[r, :len(s)] = s
    ws = ws_alloc(rtp.rtp_sparse_attn_decode_kv4_workspace_bytes(layer, B, max_sel))
    ws.fill_(0xff)
    out = torch.full_like(q, 3.0)
    lse = torch.full((B, Hq), 3.0, dtype=torch.float32, device=DEV)
    rtp.rtp_sparse_attn_decode_kv4(layer, q, c.desc, torch.from_numpy(idx).to(DEV), stride, i32(counts), max_sel, B, out, lse, ws)
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("hq,hkv,ret,page_size", [(2, 2, [1], 16), (8, 2, [0, 4, 5], 64), (16, 2, [3, 15], 256)])
def test_sparse_attention(hq, hkv, ret, page_size, dtype):
    print(f"[case] kv4 sparse, {hq}/{hkv} heads, page {page_size}, {dtype}", flush=True)
    rng = np.random.default_rng(hq + 1)
    lens = [1, 40, 700, 5000]
    c = Cache(rng, hkv, lens, page_size, page_major=hq == 8)
    q, qd = queries(rng, len(lens), hq, dtype)
    want = [0, 1, 63, 64, 65, 129, 700, 2500, 5000]
    sel = []
    for r in range(len(lens) * len(ret)):
        n = lens[r // len(ret)]
        s = rng.permutation(n)[:min(n, want[(5 * r) % len(want)] if r else 1)]
        sel.append(np.sort(s) if r % 2 else s)         # any order
    out, lse = _sparse(_layer(hq, hkv, ret, dtype), q, c, sel)
    for b in range(len(lens)):
        for h in range(hq):
            if h not in ret:
                assert (out[b, h] == 3.0).all() and lse[b, h] == 3.0
                continue
            k, v = c.rows(b, h // (hq // hkv), sel[b * len(ret) + ret.index(h)])
            check_row(out[b, h], lse[b, h], qd[b, h], k, v, dtype, what=f"sequence {b}, head {h}")


def test_sparse_attention_long_rows_and_limits():
    """One long row among short ones; counts beyond max_sel are cut there; a position selected twice counts twice; positions that are
    negative, behind the table or on a page outside the pool are left out."""
    print("[case] kv4 sparse, long row, limits", flush=True)
    rng = np.random.default_rng(9)
    lens = [60000, 300]
    c = Cache(rng, 1, lens, 32)
    q, qd = queries(rng, 2, 2, "bf16")
    layer = _layer(2, 1, [0, 1])
    sel = [np.sort(rng.permutation(60000)[:41000]), np.arange(5), np.array([7, 7, 299, 7]), np.arange(300)]
    out, lse = _sparse(layer, q, c, sel)
    for r in range(4):
        k, v = c.rows(r // 2, 0, sel[r])
        check_row(out[r // 2, r % 2], lse[r // 2, r % 2], qd[r // 2, r % 2], k, v, "bf16", what=f"row {r}")
    out, lse = _sparse(layer, q, c, sel, max_sel=200)
    for r in range(4):
        k, v = c.rows(r // 2, 0, sel[r][:200])
        check_row(out[r // 2, r % 2], lse[r // 2, r % 2], qd[r // 2, r % 2], k, v, "bf16", what=f"cut row {r}")
    c.table[1, 2] = -1                                  # positions 64 .. 95 of the second sequence have no page any more
    c.table_d.copy_(torch.from_numpy(c.table))
    sel[2] = np.array([7, -1, 5, 2 ** 30, 70, 95, 96, -2 ** 31])
    sel[1] = np.array([-5, -6, 2 ** 31 - 1])
    out, lse = _sparse(layer, q, c, sel)
    kept = [sel[0], np.zeros(0, int), np.array([7, 5, 96]), np.concatenate([np.arange(64), np.arange(96, 300)])]
    for r in range(4):
        k, v = c.rows(r // 2, 0, kept[r])
        check_row(out[r // 2, r % 2], lse[r // 2, r % 2], qd[r // 2, r % 2], k, v, "bf16", what=f"left out, row {r}")


def test_range_attention_limits():
    """Contexts beyond max_ctx are cut there, negative ones are empty, tokens without a page are left out."""
    print("[case] kv4 range, limits", flush=True)
    rng = np.random.default_rng(10)
    lens = [500, 90, 64]
    c = Cache(rng, 2, lens, 32)
    q, qd = queries(rng, 3, 4, "fp16")
    layer = _layer(4, 2, [], "fp16", sink=4, window=40)
    c.table[0, 1], c.table[0, 14] = -1, c.P
    c.table_d.copy_(torch.from_numpy(c.table))
    for what in ("dense", "local"):
        out, lse = _dense(layer, q, c, [500, -7, 64], max_ctx=480, what=what)
        for b, n in enumerate([480, 0, 64]):
            pos = np.arange(n) if what == "dense" else k4.local_positions(n, 4, 40)
            pos = pos[c.table[b, pos // 32] < c.P]
            pos = pos[c.table[b, pos // 32] >= 0]
            for h in range(4):
                k, v = c.rows(b, h // 2, pos)
                check_row(out[b, h], lse[b, h], qd[b, h], k, v, "fp16", what=f"{what}, sequence {b}, head {h}")


def test_not_a_number_stays_where_it_is():
    """A NaN block of K makes the rows that attend the token NaN, one of V the block's 32 dims, and no other."""
    print("[case] kv4 NaN blocks", flush=True)
    rng = np.random.default_rng(11)
    lens = [40, 40, 2000]
    c = Cache(rng, 2, lens, 16)
    sc = c.scales.reshape(2, c.P, 4, 2, 4, 4)

    def poison(b, kvh, t, w, blk):
        page, slot = c.table[b, t // 16], t % 16
        sc[kvh, page, slot // 4, w, blk, slot % 4] = 255
    poison(0, 0, 33, 0, 2)                              # K
    poison(1, 1, 0, 1, 3)                               # V, dims 96 .. 127
    for t in range(2000):
        poison(2, 0, t, 0, 0)                           # no finite logit at all
    c.upload()
    q, qd = queries(rng, 3, 4, "bf16")
    out, lse = _dense(_layer(4, 2, []), q, c, lens)
    so, sl = _sparse(_layer(4, 2, [0, 1, 2, 3]), q, c, [np.arange(lens[r // 4]) for r in range(12)])
    for out, lse in ((out, lse), (so, sl)):
        for b in range(3):
            for h in range(4):
                if (b, h // 2) in ((0, 0), (2, 0)):
                    assert np.isnan(out[b, h]).all() and np.isnan(lse[b, h])
                elif (b, h // 2) == (1, 1):
                    assert np.isnan(out[b, h, 96:]).all() and np.isfinite(out[b, h, :96]).all() and np.isfinite(lse[b, h])
                else:
                    k, v = c.rows(b, h // 2, np.arange(lens[b]))
                    check_row(out[b, h], lse[b, h], qd[b, h], k, v, "bf16", what=f"sequence {b}, head {h}")


def test_pool_beyond_two_to_the_32_bytes():
    """Pages whose bytes lie behind 2^32: a view of a large pool whose used pages are its last ones."""
    print("[case] kv4 pool of 5 GB", flush=True)
    rng = np.random.default_rng(12)
    c = Cache(rng, 2, [200], 64)
    big = 320000
    codes = torch.zeros((2, big, 64, 128), dtype=torch.uint8, device=DEV)
    scales = torch.zeros((2, big, 512), dtype=torch.uint8, device=DEV)
    codes[:, big - c.P:] = c.codes_d
    scales[:, big - c.P:] = c.scales_d
    table = torch.where(c.table_d >= 0, c.table_d + (big - c.P), c.table_d)
    q, qd = queries(rng, 1, 4, "bf16")
    layer = _layer(4, 2, [0, 3])
    c.codes_d, c.scales_d, c.table_d = codes, scales, table
    c.desc = rtp.kv4_cache(codes, scales, table)
    out, lse = _dense(layer, q, c, [200])
    so, sl = _sparse(layer, q, c, [np.arange(200)] * 2)
    for h in range(4):
        k, v = c.rows(0, h // 2, np.arange(200))
        check_row(out[0, h], lse[0, h], qd[0, h], k, v, "bf16", what=f"head {h}")
        if h in (0, 3):
            check_row(so[0, h], sl[0, h], qd[0, h], k, v, "bf16", what=f"sparse head {h}")
    new = torch.from_numpy(rng.standard_normal((1, 3, 2, 128))).to(torch.bfloat16).to(DEV)
    rtp.rtp_kv4_append(layer, c.desc, new, new, 768, 256, 128, i32([190]), None, 1, 3)
    back = torch.zeros_like(new)
    rtp.rtp_kv4_read(layer, c.desc, i32([190]), None, 1, 3, back, torch.zeros_like(new), 768, 256, 128)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(back.double().cpu().numpy(), k4.values(*k4.quantise(new.double().cpu().numpy())))
