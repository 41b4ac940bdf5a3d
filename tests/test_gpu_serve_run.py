"""New tokens over pages as a server uses them together: prompts in chunks beside drafts and single tokens, places that wait, rejected drafts,
conversations that end; the rows that the cache holds and the attention over them, after every step, against 64 bits."""
import numpy as np
import pytest
import torch

from chunk_util import Batch, check
from kv4_util import TYPES, check_row
from oracle import kv4_oracle as k4
from paper_2605_16928_amd import rtp, workloads as wl
from paper_2605_16928_amd.pipeline import Kv4DecodeRun, ServeRun, ws_alloc
from test_gpu_append import near, turned
from test_gpu_kv4_run import _more, _stored

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _layer(**kw):
    return wl.Layer(**{**dict(n_q_heads=8, n_kv_heads=2, ret_heads=[0, 5], sink=4, window=64), **kw})


def _batch(run, new, lens):
    """The step as a batch of the tests' own: the rows and the queries that the device holds."""
    b = Batch.__new__(Batch)
    b.new, b.ctx, b.hq, b.hkv, b.dtype, b.page = list(new), list(lens), run.layer.n_q_heads, run.layer.n_kv_heads, run.K.dtype, run.page_size
    b.off = [sum(new[:i]) for i in range(len(new) + 1)]
    b.total, b.n_pages = b.off[-1], run.n_pages
    b.table, b.rows, b.q = run.page_table.cpu(), torch.stack([run.K, run.V]).cpu(), run.q.cpu()
    return b


class Server:
    """A run and what its places were given, on the host."""

    def __init__(self, layer, seed=0, rotary=64, **kw):
        self.g = torch.Generator().manual_seed(seed)
        self.freq = (1e4 ** (-torch.arange(rotary // 2) / (rotary // 2))).float()
        self.run = ServeRun(layer, inv_freq=self.freq.to(DEV), **kw)
        self.layer, self.B = layer, self.run.B
        self.given = [torch.zeros((0, layer.n_q_heads + 2 * layer.n_kv_heads, 128)) for _ in range(self.B)]

    def step(self, new):
        L, run = self.layer, self.run
        fused = torch.randn((sum(new), L.n_q_heads + 2 * L.n_kv_heads, 128), generator=self.g).to(run.K.dtype)
        for b, part in enumerate(fused.split(list(new))):
            self.given[b] = torch.cat([self.given[b], part.float()])
        q, k, v = fused.to(DEV).split([L.n_q_heads, L.n_kv_heads, L.n_kv_heads], 1)
        out, lse = run.step(q, k, v, list(new))
        lens = [len(x) for x in self.given]
        assert run.ctx_len == lens
        batch, dtype, Hq, Hk = _batch(run, new, lens), run.K.dtype, L.n_q_heads, L.n_kv_heads
        used = [int(p) for b, n in enumerate(lens) for p in batch.table[b, :run.pages(n)]]
        assert len(set(used)) == len(used) and all(0 <= p < run.n_pages for p in used)
        for b, n in enumerate(lens):                            # every row of every place, whichever step it came with
            spots = [batch.spot(b, t) for t in range(n)]
            if n:
                held = batch.rows[:, :, [p for p, _ in spots], [s for _, s in spots]].transpose(1, 2)        # [2, tokens, heads, 128]
                near(held[0], *turned(self.given[b][:, Hq:Hq + Hk], torch.arange(n), self.freq, False, 1.0), dtype)
                assert torch.equal(held[1].float(), self.given[b][:, Hq + Hk:])
                if new[b]:
                    near(batch.q[batch.off[b]:batch.off[b + 1]], *turned(self.given[b][n - new[b]:, :Hq], torch.arange(n - new[b], n), self.freq, False, 1.0), dtype)
        want = batch.expected(L.ret_heads)
        want.update(batch.expected([h for h in range(Hq) if h not in L.ret_heads], L.sink, L.window))
        check(batch, want, out, lse)

    def truncate(self, keep):
        self.run.truncate(keep)
        self.given = [x[:n] for x, n in zip(self.given, keep)]


@pytest.mark.parametrize("kw", [dict(), dict(n_q_heads=16, ret_heads=[1, 7, 9], window=33, kv_dtype="fp16"), dict(n_q_heads=4, n_kv_heads=4, ret_heads=[]),
                                dict(n_q_heads=4, n_kv_heads=1, ret_heads=[0, 1, 2, 3])], ids=["g4", "g8_fp16", "g1_local", "g4_ret"])
@pytest.mark.parametrize("page_size", [16, 64])
def test_a_server(kw, page_size):
    print(f"[case] server, {kw}, pages of {page_size}", flush=True)
    s = Server(_layer(**kw), seed=3, seqs=4, n_pages=1 + sum(-(-n // page_size) for n in (700, 300, 200, 200)), page_size=page_size, max_ctx=800,
               max_tokens=260)
    s.step((200, 0, 1, 37))                 # prompts begin
    s.step((260, 0, 0, 0))                  # a chunk that fills the step
    s.step((1, 130, 5, 1))                  # single tokens and a draft beside a prompt
    s.truncate([460, 130, 3, 38])           # the draft was right in two tokens, one token is taken back
    s.step((1, 1, 1, 1))
    s.step((64, 3, 0, 120))
    s.truncate([0, 134, 4, 159])            # a conversation ends
    s.step((7, 100, 33, 9))                 # another one takes its place
    s.step((1, 1, 1, 1))
    s.step((0, 0, 0, 0))


def test_steps_without_room_are_refused_and_change_nothing():
    s = Server(_layer(), seqs=2, n_pages=6, page_size=16, max_ctx=56, max_tokens=50)
    s.step((20, 15))
    table, lens = s.run.page_table.clone(), list(s.run.ctx_len)
    # more tokens than a step takes; a context that is too long; seven pages; a count that is missing; a negative one; rows without a place
    for new, n in (((51, 0), 51), ((37, 0), 37), ((29, 18), 47), ((1,), 1), ((-1, 1), 0), ((1, 1), 3)):
        q, k, v = (torch.zeros((n, heads, 128), dtype=torch.bfloat16, device=DEV) for heads in (8, 2, 2))
        with pytest.raises(rtp.RtpError):
            s.run.step(q, k, v, list(new))
    with pytest.raises(rtp.RtpError):
        s.run.truncate([1])
    assert torch.equal(table, s.run.page_table) and s.run.ctx_len == lens
    s.step((33, 7))


def test_rows_that_a_step_cannot_take_change_nothing():
    """Other heads, types, strides, alignments and devices are refused before pages are handed out."""
    s = Server(_layer(), seqs=2, n_pages=6, page_size=16, max_ctx=56, max_tokens=50)
    s.step((15, 3))
    table, refs, lens = s.run.page_table.clone(), s.run.page_refs.clone(), list(s.run.ctx_len)
    fine = {name: torch.zeros((5, heads, 128), dtype=torch.bfloat16, device=DEV) for name, heads in (("q", 8), ("k", 2), ("v", 2))}
    wide = torch.zeros((5, 8, 136), dtype=torch.bfloat16, device=DEV)
    odd = torch.zeros((5, 2 * 128 + 4), dtype=torch.bfloat16, device=DEV)
    for bad in (dict(q=fine["k"]), dict(k=fine["q"]), dict(v=fine["v"][..., :64]), dict(q=fine["q"].half()), dict(k=fine["k"].float()), dict(v=fine["v"].cpu()),
                dict(q=wide[..., :128]), dict(k=odd[:, :256].unflatten(1, (2, 128))), dict(v=odd.flatten()[4:1284].view(5, 2, 128)),
                dict(k=fine["k"][:1].expand(5, 2, 128)), dict(v=fine["v"].flatten(1))):
        with pytest.raises(rtp.RtpError):
            s.run.step(*{**fine, **bad}.values(), [4, 1])
    assert torch.equal(table, s.run.page_table) and torch.equal(refs, s.run.page_refs) and s.run.ctx_len == lens
    s.step((4, 1))


@pytest.mark.parametrize("kw", [dict(), dict(n_q_heads=4, n_kv_heads=4, ret_heads=(0, 3), window=700, kv_dtype="fp16")], ids=["g4", "g1_fp16"])
@pytest.mark.parametrize("T", [1, 4])
def test_drafts_over_four_bits(kw, T):
    """A draft joins every context of a 4-bit run; each of its tokens attends up to itself."""
    print(f"[case] drafts of {T} over 4 bits, {kw}", flush=True)
    rng = np.random.default_rng(8)
    w = wl.small_decode(DEV, seed=8, ctx=(700, 16, 31, 1, 2048), **kw)
    L, run = w.layer, Kv4DecodeRun(w, 16, room=8)
    k, v, kI = _more(rng, w, T)
    run.grow(k, v, kI)
    q = torch.from_numpy(rng.standard_normal((w.B, T, L.n_q_heads, 128))).to(TYPES[L.kv_dtype]).to(DEV)
    out, lse = run.draft_attn(q)
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for b, (t0, n) in enumerate(zip(w.seq_start, w.ctx_len)):
        K, V = (_stored(torch.cat([x[:, t0:t0 + n], y[b].transpose(0, 1)], 1)) for x, y in ((w.K, k), (w.V, v)))
        for t in range(T):
            for h in range(L.n_q_heads):
                pos = np.arange(n + t + 1) if h in L.ret_heads else k4.local_positions(n + t + 1, L.sink, L.window)
                kvh = h // (L.n_q_heads // L.n_kv_heads)
                check_row(out[b, t, h], lse[b, t, h], q[b, t, h].double().cpu().numpy(), K[kvh, pos], V[kvh, pos], L.kv_dtype,
                          what=f"sequence {b}, token {t}, head {h}")
    with pytest.raises(rtp.RtpError):
        run.draft_attn(q[:1])


@pytest.mark.parametrize("cache", ["16", "4"])
def test_two_calls_at_once(cache):
    """The retrieval heads on one stream, the others on another, a workspace each: the results of one after the other, several times."""
    batch = Batch((40, 1, 300, 5), (500, 3000, 10, 900), cache=cache, page=32, seed=4)
    q, c, chunk = batch.device()
    layer = rtp.layer_desc(8, 2, [1, 4, 6], 4, 128)
    four = "_kv4" if cache == "4" else ""
    args = (batch.total, chunk.max_q, chunk.max_ctx)
    ws = [ws_alloc(rtp.rtp_dense_attn_chunk_workspace_bytes(layer, 4, *args, rtp.RTP_HEADS_RETRIEVAL)),
          ws_alloc(rtp.rtp_local_attn_chunk_workspace_bytes(layer, 4, *args))]
    out, lse = torch.zeros((batch.total, 8, 128), dtype=q.dtype, device=DEV), torch.zeros((batch.total, 8), device=DEV)

    def dense():
        getattr(rtp, "rtp_dense_attn_chunk" + four)(layer, q, q.stride(0), c, chunk, rtp.RTP_HEADS_RETRIEVAL, out, lse, ws[0])

    def local():
        getattr(rtp, "rtp_local_attn_chunk" + four)(layer, q, q.stride(0), c, chunk, out, lse, ws[1])
    dense()
    local()
    torch.cuda.synchronize()
    want, side = (out.clone(), lse.clone()), torch.cuda.Stream()
    for _ in range(5):
        out.zero_()
        lse.zero_()
        side.wait_stream(torch.cuda.current_stream())
        dense()
        with torch.cuda.stream(side):
            local()
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
