"""The 4-bit cache and its pages as a server uses them together: decode steps, forks that diverge, compaction under running sequences,
a prefill chunk behind a 4-bit context, captured steps, two streams."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import kv4_oracle as k4
from paper_2605_16928_amd import rtp, workloads as wl
from paper_2605_16928_amd.pipeline import Kv4DecodeRun, layer_desc_of
from gpu_util import DEV, check_out, i32, i64, ws_alloc
from kv4_util import TYPES, check_row

pytestmark = pytest.mark.gpu


def _stored(x):
    """What the cache holds of 16-bit rows, in 64 bits."""
    return k4.values(*k4.quantise(x.double().cpu().numpy()))


@pytest.mark.parametrize("kw", [dict(), dict(n_q_heads=16, n_kv_heads=2, ret_heads=(3, 8), window=700, kv_dtype="fp16"),
                                dict(n_q_heads=4, n_kv_heads=4, ret_heads=(1, 3))], ids=["g4", "g8_fp16", "g1"])
@pytest.mark.parametrize("page_size", [16, 128])
def test_decode_step(kw, page_size):
    """Index scores, top-p, attention of the retrieval heads over the selected tokens and of the other heads over sink + window, from
    pages that the library handed out and tokens that it stored: every head against 64 bits over the set it reports."""
    print(f"[case] decode step over 4 bits, {kw}", flush=True)
    w = wl.small_decode(DEV, seed=5, ctx=(700, 1531, 64, 2048, 1, 13), **kw)
    L = w.layer
    run = Kv4DecodeRun(w, page_size)
    assert run.status.tolist() == [0, 8]
    run.step()
    sets, counts = run.sel_sets()
    assert (counts > 0).all()
    out, lse, q = run.out_f64(), run.lse.double().cpu().numpy(), w.q.double().cpu().numpy()
    K, V = _stored(w.K), _stored(w.V)
    scale = L.softmax_scale if L.softmax_scale else 128.0 ** -0.5
    for b in range(w.B):
        t0, n = w.seq_start[b], w.ctx_len[b]
        for h in range(L.n_q_heads):
            pos = sets[b * L.n_ret + L.ret_heads.index(h)] if h in L.ret_heads else k4.local_positions(n, L.sink, L.window)
            kvh = h // (L.n_q_heads // L.n_kv_heads)
            check_row(out[b, h], lse[b, h], q[b, h], K[kvh, t0 + pos], V[kvh, t0 + pos], L.kv_dtype, scale, f"sequence {b}, head {h}")


def _check_heads(run, w, q, K, V, lens, what=""):
    """Every head of the workload's sequences against 64 bits over the set it reports; K and V: rows [n_kv_heads, n, 128] per sequence."""
    L = w.layer
    sets, _ = run.sel_sets()
    out, lse = run.out_f64(), run.lse.double().cpu().numpy()
    for b in range(w.B):
        for h in range(L.n_q_heads):
            pos = sets[b * L.n_ret + L.ret_heads.index(h)] if h in L.ret_heads else k4.local_positions(lens[b], L.sink, L.window)
            kvh = h // (L.n_q_heads // L.n_kv_heads)
            check_row(out[b, h], lse[b, h], q[b, h], K[b][kvh, pos], V[b][kvh, pos], L.kv_dtype, what=f"{what}sequence {b}, head {h}")


@pytest.mark.parametrize("form", ["two streams", "fastest"])
def test_step_on_two_streams(form):
    """The local heads on a second stream: the plain step's results, and both against 64 bits over the 4-bit rows (the 16-bit rows that
    the workload also holds differ from them by far more than the bound)."""
    print(f"[case] 4-bit decode step, {form}", flush=True)
    w = wl.small_decode(DEV, seed=15, ctx=(700, 1531, 64, 2048), n_q_heads=8, n_kv_heads=2, ret_heads=(0, 5))
    run = Kv4DecodeRun(w, 32)
    side = torch.cuda.Stream()
    K, V = ([_stored(x[:, t:t + n]) for t, n in zip(w.seq_start, w.ctx_len)] for x in (w.K, w.V))
    for _ in range(3):
        run.out.zero_()
        run.lse.zero_()
        (run.step_two_streams if form == "two streams" else run.step_fastest)(side)
        _check_heads(run, w, w.q.double().cpu().numpy(), K, V, w.ctx_len)
    out, lse = run.out.clone(), run.lse.clone()
    run.step()
    torch.cuda.synchronize()
    assert torch.equal(out, run.out) and torch.equal(lse, run.lse)


def _more(rng, w, T):
    """T further tokens for every sequence of a workload: K and V rows, index keys near the index queries, so that they are selected."""
    H, n_ret = w.layer.n_kv_heads, w.layer.n_ret
    k, v = (torch.from_numpy(rng.standard_normal((w.B, T, H, 128))).to(TYPES[w.layer.kv_dtype]).to(DEV) for _ in range(2))
    keys = 9.0 * w.qI.float().transpose(0, 1)[:, :, None] + torch.from_numpy(0.1 * rng.standard_normal((n_ret, w.B, T, 16))).to(DEV)
    return k, v, keys.to(torch.bfloat16)


def _grown(w, parts):
    """The workload with `parts` ([_more] in order) behind its sequences."""
    T, cut = sum(k.shape[1] for k, _, _ in parts), list(zip(w.seq_start, w.ctx_len))

    def join(old, new):                                # old: [rows, tokens, dims], new: per sequence
        return torch.cat([x for b, (t, n) in enumerate(cut) for x in [old[:, t:t + n]] + [m[b] for m in new]], dim=1)
    k, v = ([p[i].permute(0, 2, 1, 3) for p in parts] for i in (0, 1))
    return dataclasses.replace(w, ctx_len=[n + T for n in w.ctx_len], seq_start=[t + b * T for b, t in enumerate(w.seq_start)],
                               K=join(w.K, k), V=join(w.V, v), kI=join(w.kI, [p[2].transpose(0, 1) for p in parts]))


@pytest.mark.parametrize("kw", [dict(), dict(n_q_heads=4, n_kv_heads=4, ret_heads=(0, 3), window=700, kv_dtype="fp16")], ids=["g4", "g1_fp16"])
def test_steps_over_growing_contexts(kw):
    """Tokens join every context, some over a page that a fork shares: a step selects from and attends to all of them, as a run over
    the whole workload does; a rejected draft is cut off again; contexts changed behind the index keys' back are refused."""
    print(f"[case] steps over growing contexts, {kw}", flush=True)
    rng = np.random.default_rng(21)
    w = wl.small_decode(DEV, seed=21, ctx=(700, 16, 31, 1, 2048), **kw)
    run = Kv4DecodeRun(w, 16, spare_seqs=1, spare_pages=20, room=30)
    run.fork([0], [5], [700])
    parts, q, side = [], w.q.double().cpu().numpy(), torch.cuda.Stream()
    for step, T in enumerate((1, 17, 5, 7)):
        parts.append(_more(rng, w, T))
        run.grow(*parts[-1])
        assert run.status[0].item() == 0
        run.step() if step % 2 else run.step_two_streams(side)
        full = _grown(w, parts)
        sets, _ = run.sel_sets()
        whole = Kv4DecodeRun(full, 64)
        whole.step()
        for r, (a, b) in enumerate(zip(sets, whole.sel_sets()[0])):
            np.testing.assert_array_equal(a, b)
            assert a.max() >= w.ctx_len[r // w.layer.n_ret], "no new token was selected"
        K, V = ([_stored(x[:, t:t + n]) for t, n in zip(full.seq_start, full.ctx_len)] for x in (full.K, full.V))
        _check_heads(run, full, q, K, V, full.ctx_len, f"after {T} more, ")
    with pytest.raises(rtp.RtpError, match="no room"):
        run.grow(*_more(rng, w, 1))
    # the last 7 tokens are rejected, in one sequence all of its tokens
    run.truncate(range(5), [n + 23 for n in w.ctx_len[:3]] + [0, w.ctx_len[4] + 23])
    kept = _grown(w, parts[:3])
    lens = kept.ctx_len[:3] + [0] + kept.ctx_len[4:]
    run.step()
    _check_heads(run, kept, q, K, V, lens, "after a cut, ")
    run.fork([0], [3], [40])
    with pytest.raises(rtp.RtpError, match="alone"):
        run.step()
    run = Kv4DecodeRun(w, 16)
    run.extend([1], [16], [17])
    with pytest.raises(rtp.RtpError, match="alone"):
        run.step_two_streams(side)


def test_contexts_that_begin_empty():
    """Sequences without a token yet, the last one of the batch among them: zeros, then their first tokens."""
    print("[case] contexts that begin empty", flush=True)
    rng = np.random.default_rng(23)
    w = wl.small_decode(DEV, seed=23, ctx=(50, 0, 70, 0), n_q_heads=8, n_kv_heads=2, ret_heads=(0, 5))
    run, q = Kv4DecodeRun(w, 16, room=8), w.q.double().cpu().numpy()
    run.step()
    K, V = ([_stored(x[:, t:t + n]) for t, n in zip(w.seq_start, w.ctx_len)] for x in (w.K, w.V))
    _check_heads(run, w, q, K, V, w.ctx_len)
    new = _more(rng, w, 3)
    run.grow(*new)
    run.step()
    full = _grown(w, [new])
    K, V = ([_stored(x[:, t:t + n]) for t, n in zip(full.seq_start, full.ctx_len)] for x in (full.K, full.V))
    _check_heads(run, full, q, K, V, full.ctx_len)


def test_growth_without_pages_changes_nothing():
    """No free page for a shared last page's copy or for a new one: no byte, no context and no result changes."""
    print("[case] growth without pages", flush=True)
    rng = np.random.default_rng(22)
    w = wl.small_decode(DEV, seed=22, ctx=(30, 16), n_q_heads=8, n_kv_heads=2, ret_heads=(0, 5))
    run = Kv4DecodeRun(w, 16, spare_seqs=2, spare_pages=0, room=20)
    run.fork([0], [2], [20])
    run.extend([3], [0], [64])
    assert run.status.tolist() == [0, 0]
    run.step()
    state = run.codes, run.scales, run.page_table, run.page_refs, run.ctx_len, run.row_len, run.out, run.lse
    before = [x.clone() for x in state]
    new = _more(rng, w, 1)
    run.grow(*new)
    run.step()
    assert run.status.tolist() == [2, 0]
    assert all(torch.equal(a, b) for a, b in zip(state, before))
    run.truncate([3])
    run.grow(*new)
    run.step()
    assert run.status[0].item() == 0 and run.ctx_len.tolist() == [31, 17]
    full = _grown(w, [new])
    K, V = ([_stored(x[:, t:t + n]) for t, n in zip(full.seq_start, full.ctx_len)] for x in (full.K, full.V))
    _check_heads(run, full, w.q.double().cpu().numpy(), K, V, full.ctx_len)


def test_forks_diverge_and_survive_compaction():
    """Two forks of a prompt and the prompt itself grow by tokens of their own, another sequence ends, the pool is compacted: what every
    sequence attends to stays its own, bit for bit across the move."""
    print("[case] forks, growth, compaction", flush=True)
    w = wl.small_decode(DEV, seed=6, ctx=(300, 77, 128), n_q_heads=8, n_kv_heads=2, ret_heads=(0, 4))
    H, ps = 2, 32
    run = Kv4DecodeRun(w, ps, spare_seqs=2, spare_pages=12)
    desc = layer_desc_of(w.layer)
    text = [(w.K[:, t:t + n].double().cpu().numpy(), w.V[:, t:t + n].double().cpu().numpy()) for t, n in zip(w.seq_start, w.ctx_len)]
    rng = np.random.default_rng(6)
    q = torch.from_numpy(rng.standard_normal((5, 8, 128))).to(torch.bfloat16).to(DEV)
    qd = q.double().cpu().numpy()

    def attend(lens):
        out, lse = torch.zeros_like(q), torch.zeros((5, 8), dtype=torch.float32, device=DEV)
        ws = ws_alloc(rtp.rtp_dense_attn_kv4_workspace_bytes(desc, 5, 384))
        rtp.rtp_dense_attn_kv4(desc, q, run.cache, i32(lens), 5, 384, out, lse, ws)
        torch.cuda.synchronize()
        return out, lse

    def check(out, lse, what):
        for b, (K, V) in enumerate(text):
            for h in range(8):
                check_row(out[b, h].double().cpu().numpy(), float(lse[b, h]), qd[b, h], k4.values(*k4.quantise(K[h // 4])),
                          k4.values(*k4.quantise(V[h // 4])), "bf16", what=f"{what}, sequence {b}, head {h}")

    # rows 3 and 4: forks of the whole first sequence (its last page is partly filled) and of 64 of its tokens (whole pages)
    run.fork([0, 0], [3, 4], [300, 64])
    text += [text[0], tuple(x[:, :64] for x in text[0])]
    check(*attend([300, 77, 128, 300, 64]), "after the fork")
    # all but sequence 1 grow by 10 tokens of their own
    grown = [0, 2, 3, 4]
    lens = [300, 77, 128, 300, 64]
    run.extend(grown, [lens[b] for b in grown], [lens[b] + 10 for b in grown])
    assert run.status[0].item() == 0
    new = [torch.from_numpy(rng.standard_normal((5, 10, H, 128))).to(torch.bfloat16).to(DEV) for _ in range(2)]
    start = [n if b in grown else -1 for b, n in enumerate(lens)]
    run.append(new[0], new[1], i32(start))
    for b in grown:
        text[b] = tuple(np.concatenate([x, n[b].double().cpu().numpy().transpose(1, 0, 2)], axis=1) for x, n in zip(text[b], new))
        lens[b] += 10
    check(*attend(lens), "after the growth")
    # sequence 2 ends, sequence 3 is cut back by 20, the pool is compacted
    run.truncate([2, 3], [0, 290])
    lens[2], lens[3] = 0, 290
    text[2], text[3] = tuple(x[:, :0] for x in text[2]), tuple(x[:, :290] for x in text[3])
    before = attend(lens)
    check(*before, "after the end")
    run.compact()
    used, moves = run.status.tolist()
    assert used == int((run.page_refs > 0).sum()) and moves > 0 and int(run.page_table.max()) < used and int((run.page_refs[used:] != 0).sum()) == 0
    after = attend(lens)
    assert all(torch.equal(a, b) for a, b in zip(before, after))
    # and the sequence that was cut back grows again, into a page of its own
    run.extend([3], [290], [330])
    more = [torch.from_numpy(rng.standard_normal((1, 40, H, 128))).to(torch.bfloat16).to(DEV) for _ in range(2)]
    row = rtp.kv4_cache(run.codes, run.scales, run.page_table[3:4])
    rtp.rtp_kv4_append(desc, row, more[0], more[1], 40 * 256, 256, 128, i32([290]), None, 1, 40)
    lens[3] = 330
    text[3] = tuple(np.concatenate([x, n[0].double().cpu().numpy().transpose(1, 0, 2)], axis=1) for x, n in zip(text[3], more))
    check(*attend(lens), "after growing again")


def test_prefill_chunk_behind_a_4_bit_context():
    """The context is read back to 16 bits, the chunk's own rows follow it as they are, and the dense prefill runs over both."""
    print("[case] prefill behind a 4-bit context", flush=True)
    rng = np.random.default_rng(8)
    H, n, T, ps = 2, 333, 40, 64
    desc = rtp.layer_desc(8, H, [], 4, 64)
    rows = [torch.from_numpy(rng.standard_normal((H, n + T, 128))).to(torch.bfloat16).to(DEV) for _ in range(2)]
    codes = torch.zeros((H, 7, ps, 128), dtype=torch.uint8, device=DEV)
    scales = torch.zeros((H, 7, ps * 8), dtype=torch.uint8, device=DEV)
    cache = rtp.kv4_cache(codes, scales, i32([5, 0, 3, 1, 6, 2]).view(1, 6))
    K, V = (torch.zeros_like(r) for r in rows)
    hs = (n + T) * 128
    rtp.rtp_kv4_append(desc, cache, rows[0], rows[1], 0, 128, hs, i32([0]), None, 1, n)
    rtp.rtp_kv4_read(desc, cache, i32([0]), None, 1, n, K, V, 0, 128, hs)
    K[:, n:], V[:, n:] = rows[0][:, n:], rows[1][:, n:]
    q = torch.from_numpy(rng.standard_normal((1, T, 8, 128))).to(torch.bfloat16).to(DEV)
    out, lse = torch.zeros_like(q), torch.zeros((1, T, 8), dtype=torch.float32, device=DEV)
    rtp.rtp_dense_attn(desc, q, K, V, 128, hs, i64([0]), i32([n + T]), i32([n]), 1, T, n + T, out, lse, ws_alloc(1 << 20))
    torch.cuda.synchronize()
    Kd, Vd = (np.concatenate([_stored(r[:, :n]), r[:, n:].double().cpu().numpy()], axis=1) for r in rows)
    for t in (0, 7, T - 1):
        for h in range(8):
            ref = k4.attend(q[0, t, h].double().cpu().numpy(), Kd[h // 4, :n + t + 1], Vd[h // 4, :n + t + 1], 128.0 ** -0.5)[0]
            check_out(out[0, t, h].double().cpu().numpy(), ref, f"query {t}, head {h}", tight="mfma")


def test_captured_steps_replay():
    """Growth, the copies of shared pages, an append and all three attentions captured into one graph; replays with new tokens, lengths
    and selections, eager work between them, each against the same calls made eagerly on a copy of the state."""
    print("[case] captured steps", flush=True)
    rng = np.random.default_rng(9)
    H, hq, B, ps = 2, 8, 3, 16
    lens0 = [3000, 40, 500]
    w = wl.small_decode(DEV, seed=9, ctx=tuple(lens0), n_q_heads=hq, n_kv_heads=H, ret_heads=(0, 5))
    run = Kv4DecodeRun(w, ps, spare_seqs=3, spare_pages=60)
    run.fork([0, 1, 2], [3, 4, 5], lens0)              # so that the first growth copies pages
    desc, n_ret, max_ctx = layer_desc_of(w.layer), 2, 3100
    table = run.page_table
    wide = torch.full((6, -(-max_ctx // ps) + 1), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    state = (wide, run.page_refs, run.codes, run.scales)
    twin = tuple(x.clone() for x in state)
    k_new, v_new, q = (torch.zeros((B, 1, H, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((B, 1, H, 128), dtype=torch.bfloat16, device=DEV),
                       torch.zeros((B, hq, 128), dtype=torch.bfloat16, device=DEV))
    seqs, old, new = i32([0, 1, 2]), i32(lens0), i32([n + 1 for n in lens0])
    idx, count = torch.zeros((B * n_ret, 2000), dtype=torch.int32, device=DEV), i32([0] * (B * n_ret))

    def calls(state, tmp):
        wide, refs, codes, scales = state
        m, cache, pools = rtp.page_map(wide, refs, ps), rtp.kv4_cache(codes, scales, wide), rtp.page_pools([codes, scales])
        src, dst, status, ws_p, ws_s, ws_l, ws_d, outs = tmp
        rtp.rtp_kv_pages_extend(m, seqs, old, new, B, src, dst, status, ws_p)
        rtp.rtp_kv_pages_copy(pools, codes.shape[1], src, dst, B)
        rtp.rtp_kv4_append(desc, cache, k_new, v_new, H * 128, H * 128, 128, old, None, B, 1)
        rtp.rtp_sparse_attn_decode_kv4(desc, q, cache, idx, 2000, count, 2000, B, outs[0], outs[1], ws_s)
        rtp.rtp_local_attn_kv4(desc, q, cache, new, B, max_ctx, outs[0], outs[1], ws_l)
        rtp.rtp_dense_attn_kv4(desc, q, cache, new, B, max_ctx, outs[2], outs[3], ws_d)

    def scratch():
        m = rtp.page_map(wide, run.page_refs, ps)
        outs = [torch.zeros((B, hq, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((B, hq), dtype=torch.float32, device=DEV)]
        return (i32([0] * B), i32([0] * B), i32([0, 0]), ws_alloc(rtp.rtp_kv_pages_workspace_bytes(m, B)),
                ws_alloc(rtp.rtp_sparse_attn_decode_kv4_workspace_bytes(desc, B, 2000)), ws_alloc(rtp.rtp_local_attn_kv4_workspace_bytes(desc, B, max_ctx)),
                ws_alloc(rtp.rtp_dense_attn_kv4_workspace_bytes(desc, B, max_ctx)), outs + [torch.zeros_like(x) for x in outs])
    tmp, tmp2 = scratch(), scratch()
    torch.cuda.synchronize()
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=side):
        calls(state, tmp)
    for step in range(5):
        for x in (k_new, v_new, q):
            x.copy_(torch.from_numpy(rng.standard_normal(tuple(x.shape))))
        cur = [n + step for n in lens0]
        old.copy_(i32(cur))
        new.copy_(i32([n + 1 for n in cur]))
        sel = [min(cur[r // n_ret], int(rng.integers(0, 2000))) for r in range(B * n_ret)]
        for r, n in enumerate(sel):
            idx[r, :n] = torch.from_numpy(np.sort(rng.permutation(cur[r // n_ret] + 1)[:n]).astype(np.int32)).to(DEV)
        count.copy_(i32(sel))
        g.replay()
        torch.cuda.synchronize()
        calls(twin, tmp2)
        torch.cuda.synchronize()
        for name, a, b in zip(("table", "counts", "codes", "scales"), state, twin):
            assert torch.equal(a, b), f"step {step}: {name}"
        for a, b in zip(tmp[7] + [tmp[2]], tmp2[7] + [tmp2[2]]):
            assert torch.equal(a, b), f"step {step}"
        assert tmp[2][0].item() == 0 and torch.isfinite(tmp[7][2].float()).all()


def test_calls_on_two_streams():
    """Two streams with workspaces of their own, many times over: the results of calls made alone."""
    print("[case] two streams", flush=True)
    w = wl.small_decode(DEV, seed=12, ctx=(5000, 9000), n_q_heads=8, n_kv_heads=2, ret_heads=(0, 4))
    run = Kv4DecodeRun(w, 64)
    run.step()
    torch.cuda.synchronize()
    want = run.out.clone(), run.lse.clone()
    dense = torch.zeros_like(run.out), torch.zeros_like(run.lse)
    run.dense_attn(*dense)
    torch.cuda.synchronize()
    want_dense = [x.clone() for x in dense]
    side = torch.cuda.Stream()
    for _ in range(20):
        run.out.zero_()
        for x in dense:
            x.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            run.dense_attn(*dense)
        run.sparse_attn()
        run.local_attn(stream=side)
        torch.cuda.synchronize()
        assert torch.equal(run.out, want[0]) and torch.equal(run.lse, want[1])
        assert all(torch.equal(a, b) for a, b in zip(dense, want_dense))


def test_large_batches():
    """More than 256 sequences (items by unit), batches whose lengths differ by a factor of a thousand, units of one item."""
    print("[case] kv4 large batches", flush=True)
    from kv4_util import Cache, queries
    rng = np.random.default_rng(13)
    for B, hkv, longest, window in ((300, 1, 90, 64), (40, 2, 9000, 2000), (257, 4, 40, 2000), (200, 2, 3000, 2500)):
        lens = [longest] + [int(x) for x in np.exp(rng.uniform(0, np.log(longest), B - 1))]
        lens[B // 2] = 0
        c = Cache(rng, hkv, lens, 16)
        layer = rtp.layer_desc(2 * hkv, hkv, [0], 4, window)
        q, qd = queries(rng, B, 2 * hkv, "bf16")
        for what, size, call in (("dense", rtp.rtp_dense_attn_kv4_workspace_bytes, rtp.rtp_dense_attn_kv4),
                                 ("local", rtp.rtp_local_attn_kv4_workspace_bytes, rtp.rtp_local_attn_kv4)):
            out, lse = torch.zeros_like(q), torch.zeros((B, 2 * hkv), dtype=torch.float32, device=DEV)
            ws = ws_alloc(size(layer, B, longest))
            ws.fill_(0xff)
            call(layer, q, c.desc, i32(lens), B, longest, out, lse, ws)
            torch.cuda.synchronize()
            o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
            for b in [0, 1, B // 2, B - 1] + [int(x) for x in rng.integers(0, B, 20)]:
                pos = np.arange(lens[b]) if what == "dense" else k4.local_positions(lens[b], 4, window)
                for h in range(1 if what == "local" else 0, 2 * hkv):
                    k, v = c.rows(b, h // 2, pos)
                    check_row(o[b, h], l[b, h], qd[b, h], k, v, "bf16", what=f"{what}, batch {B}, sequence {b}, head {h}")
