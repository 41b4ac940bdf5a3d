"""New tokens over a cache in pages, as measurable cases.

  append  q, k and v of new tokens, as a fused projection leaves them, are rotated by their positions; k and v go to the pages of a
          16-bit cache, q to the attention (rtp_kv_append).
  dense   attention of a batch of new tokens, packed without padding, one or thousands to a sequence, over every cached token up to their own:
          every head's, or the retrieval heads' alone, from 16-bit pages or from the 4-bit cache (rtp_dense_attn_chunk, _kv4).
  local   the same of the other heads over the sink and the window (rtp_local_attn_chunk, _kv4).

A sequence's new tokens are the last ones of its context and are in the cache when the attention reads it.  16-bit pages: K and V
[KV heads, pages, page_size, 128], or the pages in front.  4-bit cache: a row's 128 values are 4 blocks of 32; a block is a scale byte
s, standing for 2^(s - 127), and 32 codes of a sign, 2 exponent bits and 1 mantissa bit (0, .5, 1, 1.5, 2, 3, 4, 6).  codes: uint8
[KV heads, pages, page_size, 128], a token's K in the first 64 bytes (dim 2i in the low half of byte i) and its V in the rest;
scales: uint8 [KV heads, pages, page_size / 4, K or V, block, token % 4].

Sizes are fixed by the case alone; the seed draws the values and the placing of the pages.
"""
import math
import random

import torch

DEV = "cuda:0"
own = False

HEADS = [(8, 2), (32, 8), (64, 8), (32, 4), (16, 16), (8, 4)]     # query heads, KV heads: groups of 1, 2, 4 and 8
PAGES = [16, 32, 64, 128, 256]
MOST_FLOPS = 2.0e12        # of the largest case
MOST_LOGITS = 4.3e9        # of a padded batch: what a plain form holds
MOST_ROWS = 1 << 23        # (token, KV head) rows of the largest cache


def _case(name, kind, **kw):
    c = dict(name=name, kind=kind, hq=32, hkv=8, dtype="bf16", page=64, batch=1, new=(1, 1), past=(4096, 4096), cache="16", front="heads", fused=True)
    c.update({"append": dict(rotary=128, pairs="halves", base=1e6), "dense": dict(heads="all", lse=True),
              "local": dict(heads="local", lse=True, sink=4, window=8192, n_ret=4)}[kind])
    c.update(kw)
    return _flat(c)


def _flat(c):
    """A pair as its lower and its upper bound."""
    return {n: x for k, v in c.items() for n, x in (((k + "_lo", v[0]), (k + "_hi", v[1])) if isinstance(v, tuple) else ((k, v),))}


def listed():
    return [
        # a decode step of 32 sequences: one new token each, at positions up to 262143
        _case("append_step", "append", batch=32, past=(16384, 262143)),
        # a mixed batch of a server in fp16: up to 1000 new tokens a sequence, some with none, half of the dims rotated, in neighbouring pairs
        _case("append_ragged_fp16", "append", hkv=4, batch=6, new=(0, 1000), past=(0, 3000), dtype="fp16", page=16, rotary=64,
              pairs="neighbours", base=1e4, front="pages"),
        # one chunk of a chunked prefill: 4096 tokens behind 28672
        _case("append_chunk", "append", new=(4096, 4096), past=(28672, 28672)),
        # one token of one short conversation on a small layer
        _case("dense_700", "dense", hq=8, hkv=2, past=(699, 699)),
        # a decode step of 32 ragged contexts, every head over every token
        _case("dense_step", "dense", batch=32, past=(1499, 30010)),
        # five tokens of a draft to be verified, 16 sequences, fp16, small pages
        _case("dense_draft_fp16", "dense", hkv=4, batch=16, new=(5, 5), past=(2000, 32763), dtype="fp16", page=16),
        # a server's mixed batch: prompts' chunks of up to 500 tokens beside single tokens and sequences that wait
        _case("dense_mixed", "dense", batch=12, new=(0, 500), past=(0, 16001), front="pages", lse=False),
        # the paper's prefill rule for the retrieval heads: 4096 tokens behind 126976, 4 of 32 heads
        _case("dense_ret_128k", "dense", heads="ret", n_ret=4, new=(4096, 4096), past=(126976, 126976), lse=False),
        # a decode step of the other heads: sink and window of 32 contexts, some shorter than the window
        _case("local_step", "local", batch=32, past=(999, 100002), page=16),
        # a chunk of a chunked prefill, the paper's window
        _case("local_chunk", "local", new=(4096, 4096), past=(28672, 28672), lse=False),
        # four tokens of a draft over the longest contexts that a 4-bit cache is kept for
        _case("dense_kv4_draft", "dense", batch=8, new=(4, 4), past=(131068, 131068), cache="4"),
        # a chunk over a prompt that is held in 4 bits, every head
        _case("dense_kv4_chunk", "dense", new=(4096, 4096), past=(28672, 28672), cache="4", lse=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(hi + 0.49)))))))


def draw(rng):
    hq, hkv = rng.choice(HEADS)
    kind = rng.choice(["append", "dense", "dense", "dense", "local", "local"])
    c = dict(kind=kind, hq=hq, hkv=hkv, dtype=rng.choice(["bf16", "bf16", "fp16"]), page=rng.choice(PAGES), front=rng.choice(["heads", "heads", "pages"]),
             fused=rng.random() < 0.7, cache="16")
    if kind == "append":
        batch = _log(rng, 1, 64)
        most = _log(rng, 1, max(1, 16384 * 8 // (batch * hkv)))
        past = _log(rng, 1, 1 << 20)
        c.update(batch=batch, new=(rng.choice([0, 1, most]), most), past=(rng.choice([0, past // 9, past]), past), rotary=rng.choice([128, 128, 64, 32]),
                 pairs=rng.choice(["halves", "halves", "neighbours"]), base=rng.choice([1e4, 5e5, 1e6]))
        return _flat(c)
    c.update(cache=rng.choice(["16", "16", "4"]), lse=rng.random() < 0.5)
    if c["cache"] == "4":
        c["front"] = "heads"
    batch = _log(rng, 1, 32)
    most = rng.choice([1, rng.randint(2, 16), _log(rng, 1, 4096), _log(rng, 16, 4096)])
    past = _log(rng, 1, 131072)
    if kind == "local":
        c.update(heads="local", n_ret=rng.randint(0, min(8, hq - 1)), sink=rng.choice([0, 4, 4, 17]), window=_log(rng, 16, 8192))
    else:
        c.update(heads=rng.choice(["all", "all", "ret"]), n_ret=rng.randint(1, min(8, hq)))
    lo = rng.choice([0, 1, 3]), rng.choice([0, 1, 4, 30])
    while True:
        c.update(batch=batch, new=(lo[0] and max(1, most // lo[0]), most), past=(lo[1] and past // lo[1], past))
        n = most + past
        keys = min(n, c["sink"] + c["window"] + most) if kind == "local" else n
        served = c["n_ret"] if c["heads"] == "ret" else hq
        if batch * hkv * n <= MOST_ROWS // 2 and batch * served * most * keys <= MOST_LOGITS / 2 and work(_flat(c))["flops"] <= MOST_FLOPS:
            return _flat(c)
        past, most, batch = max(1, past // 2), max(1, most * 3 // 4), max(1, batch * 3 // 4)


# ---- sizes, from the case alone ---------------------------------------------------------------------------------------------
def _lengths(lo, hi, n, salt):
    """n lengths between lo and hi, spread over their logarithm; the first is hi.  lo = 0: a quarter of the others are 0."""
    rng = random.Random("%s %d %d %d" % (salt, lo, hi, n))
    return [hi] + [0 if lo < 1 and rng.random() < 0.25 else _log(rng, max(lo, 1), hi) if hi else 0 for _ in range(n - 1)]


def _counts(case):
    """New tokens and contexts (the new ones among them) of the sequences."""
    new = _lengths(case["new_lo"], case["new_hi"], case["batch"], "new")
    past = _lengths(case["past_lo"], case["past_hi"], case["batch"], "past")
    return new, [p + n for p, n in zip(past, new)]


def _served(case):
    """The query heads that a call serves, by KV head: [(KV head, its heads)]."""
    hq, hkv, n = case["hq"], case["hkv"], case.get("n_ret", 0)
    ret = {(j * hq) // n for j in range(n)} if n else set()
    mine = [h for h in range(hq) if case["heads"] == "all" or (h in ret) == (case["heads"] == "ret")]
    group = hq // hkv
    return [(k, [h for h in mine if h // group == k]) for k in range(hkv) if any(h // group == k for h in mine)]


def _ret_heads(case):
    n = case.get("n_ret", 0)
    return sorted({(j * case["hq"]) // n for j in range(n)}) if n else []


def _pairs(case, new, ctx):
    """(query, key) pairs of one head, and the rows that its sequence's queries see."""
    first, pairs = ctx - new, 0
    if case["heads"] != "local":
        return new * first + new * (new + 1) // 2, ctx if new else 0
    s, w = case["sink"], case["window"]
    see = lambda m: min(s, m + 1) + max(0, m + 1 - max(s, m - w + 1))  # noqa: E731
    full = max(first, min(ctx, s + w))                                  # from here on every query sees sink + window
    pairs = sum(see(m) for m in range(first, full)) + (ctx - full) * (s + w)
    lo = max(s, first - w + 1)
    return pairs, (min(s, ctx) + max(0, ctx - lo)) if new else 0


def work(case):
    """Bytes and operations that a pass cannot do without."""
    new, ctx = _counts(case)
    hq, hkv = case["hq"], case["hkv"]
    if case["kind"] == "append":
        return {"bytes": sum(new) * (2 * hq + 4 * hkv) * 256 + 8 * case["batch"], "flops": sum(new) * (hq + hkv) * case["rotary"] * 3}
    served, pairs, rows = _served(case), 0, 0
    for n, c in zip(new, ctx):
        p, r = _pairs(case, n, c)
        pairs, rows = pairs + p, rows + r
    heads = sum(len(h) for _, h in served)
    return {"bytes": rows * len(served) * (512 if case["cache"] == "16" else 136) + sum(new) * heads * (512 + (4 if case["lse"] else 0))
            + 4 * sum(-(-c // case["page"]) for c in ctx), "flops": pairs * heads * 512}


# ---- inputs ---------------------------------------------------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


_GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _to_codes(x):
    """Rows [..., 128] as (codes uint8 [..., 64], scales uint8 [..., 4]): a value that the cache could hold for them."""
    y = x.unflatten(-1, (4, 32))
    e = torch.ceil(torch.log2(y.abs().amax(-1, keepdim=True).clamp(min=1e-30) / 7.0))
    y = y * torch.exp2(-e)
    mid = torch.tensor([(a + b) / 2 for a, b in zip(_GRID, _GRID[1:])], device=DEV)
    code = (torch.bucketize(y.abs(), mid).byte() | ((y < 0).byte() << 3)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e.squeeze(-1) + 127).byte()


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    new, ctx = _counts(case)
    hq, hkv, page, dt, B = case["hq"], case["hkv"], case["page"], _dtype(case), case["batch"]
    total, append = sum(new), case["kind"] == "append"
    off = [0]
    for n in new:
        off.append(off[-1] + n)
    # every sequence's pages, anywhere in the pool.  An append touches the new tokens' pages alone: the old ones stand for other pages of a
    # pool that is kept small.
    first = [(c - n) // page if append else 0 for n, c in zip(new, ctx)]
    need = [-(-c // page) - f if c else 0 for c, f in zip(ctx, first)]
    n_pages = sum(need) + 3
    ids = torch.randperm(n_pages, generator=g, device=DEV).int()
    table = torch.full((B, max(max(-(-c // page) for c in ctx), 1) + 1), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b in range(B):
        table[b, :first[b]] = ids[-1]
        table[b, first[b]:first[b] + need[b]] = ids[at:at + need[b]]
        at += need[b]
    st = dict(case=case, kind=case["kind"], table=table, n_pages=n_pages, total=total, max_new=max(new), max_ctx=max(max(ctx), 1), off=_i32(off),
              new=_i32(new), ctx=_i32(ctx))
    # channels of keys and values are of different size, as a model's are
    gain = [torch.exp(sigma * torch.randn((hkv, 1, 1, 128), generator=g, device=DEV)) for sigma in (0.5, 0.2)]
    pools = []
    for w in (0, 1):
        if case["cache"] == "16":
            x = torch.empty((hkv, n_pages, page, 128) if case["front"] == "heads" else (n_pages, hkv, page, 128), dtype=dt, device=DEV)
            x = x if case["front"] == "heads" else x.transpose(0, 1)
        elif w == 0:
            st["codes"] = torch.empty((hkv, n_pages, page, 128), dtype=torch.uint8, device=DEV)
            st["scales"] = torch.empty((hkv, n_pages, page // 4, 2, 4, 4), dtype=torch.uint8, device=DEV)
        step = max(1, (1 << 21) // (page * hkv))
        for p0 in range(0, n_pages, step):
            p1 = min(n_pages, p0 + step)
            rows = torch.randn((hkv, p1 - p0, page, 128), generator=g, device=DEV) * gain[w]
            if case["cache"] == "16":
                x[:, p0:p1] = rows
            else:
                c, s = _to_codes(rows)
                st["codes"][:, p0:p1, :, 64 * w:64 * w + 64] = c
                st["scales"][:, p0:p1, :, w] = s.view(hkv, p1 - p0, page // 4, 4, 4).transpose(3, 4)
        if case["cache"] == "16":
            pools.append(x)
    if pools:
        st["K"], st["V"] = pools
    # [tokens, (hq + 2 hkv) * 128] as a fused projection leaves it, or q alone; three rows behind the last sequence
    qkv = torch.randn((total + 3, hq + 2 * hkv if case["fused"] or append else hq, 128), generator=g, device=DEV)
    if append:
        qkv[:, hq:hq + hkv] *= gain[0].view(1, hkv, 128)
        qkv[:, hq + hkv:] *= gain[1].view(1, hkv, 128)
    qkv = qkv.to(dt)
    st["q"] = qkv[:total, :hq]
    st["out"] = torch.zeros((total, hq, 128), dtype=dt, device=DEV)
    if append:
        st["k"], st["v"] = qkv[:total, hq:hq + hkv], qkv[:total, hq + hkv:]
        half = case["rotary"] // 2
        st["inv_freq"] = (case["base"] ** -(torch.arange(half, dtype=torch.float64, device=DEV) / half)).float()
    else:
        st["lse"] = torch.zeros((total, hq), dtype=torch.float32, device=DEV) if case["lse"] else None
    return st


# ---- plain forms ------------------------------------------------------------------------------------------------------------------
def _rows_of(st):
    """Sequence and position of every packed token."""
    b = torch.repeat_interleave(torch.arange(st["new"].numel(), device=DEV), st["new"], output_size=st["total"])
    t = torch.arange(st["total"], device=DEV) - st["off"][b]
    return b, (st["ctx"] - st["new"])[b] + t


def _rotated(case, x, cos, sin):
    n = case["rotary"]
    y = x.float()
    if case["pairs"] == "halves":
        a, b = y[..., :n // 2], y[..., n // 2:n]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, y[..., n:]], -1).to(x.dtype)
    a, b = y[..., 0:n:2], y[..., 1:n:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), y[..., n:]], -1).to(x.dtype)


def _plain_append(st):
    case, page = st["case"], st["case"]["page"]
    b, pos = _rows_of(st)
    angle = pos.double()[:, None] * st["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    at, slot = st["table"][b, pos // page].long(), pos % page
    st["K"][:, at, slot] = _rotated(case, st["k"], cos, sin).transpose(0, 1)
    st["V"][:, at, slot] = st["v"].transpose(0, 1)
    return _rotated(case, st["q"], cos, sin), st["K"], st["V"]


def _fetch(st, kv, at, slot):
    """K and V rows in 32 bits of KV heads `kv` [S] at pages and slots [B, N]: [S, B, N, 128]."""
    kv = kv[:, None, None]
    if st["case"]["cache"] == "16":
        return st["K"][kv, at, slot].float(), st["V"][kv, at, slot].float()
    byte = torch.arange(256, device=DEV)
    grid = torch.tensor(_GRID + [-x for x in _GRID], device=DEV)
    pairs = torch.stack([grid[byte & 15], grid[byte >> 4]], 1)
    x = pairs[st["codes"][kv, at, slot].int()].flatten(-2).unflatten(-1, (2, 4, 32))
    s = torch.exp2(st["scales"][kv, at, slot // 4, :, :, slot % 4].float() - 127.0)
    x = (x * s.unsqueeze(-1)).flatten(-2)
    return x[..., 0, :], x[..., 1, :]


def _plain_attention(st):
    """The batch padded to its longest sequence; a KV head's rows are gathered once for the heads that read them."""
    case, B, T, N = st["case"], st["case"]["batch"], st["max_new"], st["max_ctx"]
    served = _served(case)
    most = max(len(h) for _, h in served)
    kv = torch.tensor([k for k, _ in served], device=DEV)
    heads = torch.tensor([(h * most)[:most] for _, h in served], device=DEV)               # (a shorter list repeats its own heads)
    new, ctx = st["new"].long()[:, None], st["ctx"].long()[:, None]
    n = torch.arange(N, device=DEV)[None].expand(B, N)
    if case["kind"] == "local":                 # the keys that some query of the sequence sees
        sink = case["sink"]
        n = torch.arange(min(N, sink + case["window"] + T), device=DEV)[None].expand(B, -1)
        lo = (ctx - new - case["window"] + 1).clamp(min=sink)
        n = torch.where(n < sink, n, lo + n - sink)
    there = n < ctx
    n = torch.where(there, n, 0)
    k, v = _fetch(st, kv, st["table"].long().gather(1, n // case["page"]).clamp(min=0), n % case["page"])
    t = torch.arange(T, device=DEV)[None]
    row = torch.where(t < new, st["off"].long()[:-1, None] + t, 0)
    q = st["q"][row[:, :, None, None], heads].float()                                      # [B, T, S, heads, 128]
    q = q.permute(2, 0, 1, 3, 4).reshape(len(served), B, T * most, 128)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(128.0)).view(len(served), B, T, most, -1)
    m = (ctx - new + t)[:, :, None]
    keep = there[:, None] & (n[:, None] <= m) & (t < new)[:, :, None]
    if case["kind"] == "local":
        keep &= (n[:, None] < case["sink"]) | (n[:, None] > m - case["window"])
    x.masked_fill_(~keep[None, :, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top.isfinite(), top, 0.0)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(len(served), B, T * most, -1), v).view(len(served), B, T, most, 128)
    o = torch.where(total > 0, o / total, 0.0).permute(1, 2, 0, 3, 4)
    b, t = torch.nonzero(t < new, as_tuple=True)
    out, lse = torch.zeros_like(st["out"]), None
    out[row[b, t][:, None, None], heads] = o[b, t].to(out.dtype)
    if st["lse"] is None:
        return out
    lse = torch.zeros_like(st["lse"])
    lse[row[b, t][:, None, None], heads] = (torch.log(total) + top).squeeze(-1).permute(1, 2, 0, 3)[b, t]
    return out, lse


# ---- the framework's calls -----------------------------------------------------------------------------------------------------------
def _handles(st):
    """What a program keeps from call to call: the descriptors of the layer, the cache, the batch and the rotation, a workspace."""
    if "layer" in st:
        return
    from paper_2605_16928_amd import rtp
    case = st["case"]
    st["layer"] = rtp.layer_desc(case["hq"], case["hkv"], _ret_heads(case), case.get("sink", 4), case.get("window", 64),
                                 kv_dtype=rtp.RTP_DTYPE_BF16 if case["dtype"] == "bf16" else rtp.RTP_DTYPE_FP16)
    if case["cache"] == "16":
        st["cache"] = rtp.kv_cache(st["K"], st["V"], st["table"])
    else:
        st["cache"] = rtp.kv4_cache(st["codes"], st["scales"], st["table"])
    st["chunk"] = rtp.chunk_desc(st["off"], st["ctx"], st["total"], st["max_new"], st["max_ctx"])
    if case["kind"] == "append":
        st["rope"] = rtp.rope_desc(st["inv_freq"], interleaved=case["pairs"] == "neighbours")
        return
    if case["kind"] == "local":
        size = rtp.rtp_local_attn_chunk_workspace_bytes(st["layer"], case["batch"], st["total"], st["max_new"], st["max_ctx"])
    else:
        st["which"] = rtp.RTP_HEADS_ALL if case["heads"] == "all" else rtp.RTP_HEADS_RETRIEVAL
        size = rtp.rtp_dense_attn_chunk_workspace_bytes(st["layer"], case["batch"], st["total"], st["max_new"], st["max_ctx"], st["which"])
    st["ws"] = torch.empty(max(256, size), dtype=torch.uint8, device=DEV)


def _own(st):
    from paper_2605_16928_amd import rtp
    _handles(st)
    case, q = st["case"], st["q"]
    if case["kind"] == "append":
        rtp.rtp_kv_append(st["layer"], st["cache"], st["chunk"], st["rope"], q, q.stride(0), st["k"], st["k"].stride(0), st["v"],
                          st["v"].stride(0), st["out"], st["out"].stride(0))
        return st["out"], st["K"], st["V"]
    if case["kind"] == "local":
        call = rtp.rtp_local_attn_chunk if case["cache"] == "16" else rtp.rtp_local_attn_chunk_kv4
        call(st["layer"], q, q.stride(0), st["cache"], st["chunk"], st["out"], st["lse"], st["ws"])
    else:
        call = rtp.rtp_dense_attn_chunk if case["cache"] == "16" else rtp.rtp_dense_attn_chunk_kv4
        call(st["layer"], q, q.stride(0), st["cache"], st["chunk"], st["which"], st["out"], st["lse"], st["ws"])
    return st["out"] if st["lse"] is None else (st["out"], st["lse"])


def run(state):
    if own:
        return _own(state)
    return _plain_append(state) if state["kind"] == "append" else _plain_attention(state)


# ---- the definition, in 64 bits ---------------------------------------------------------------------------------------------------------
def _exact_rows(st, b, kvh, pos):
    """K and V in 64 bits of positions `pos` of sequence b, one KV head."""
    page = st["case"]["page"]
    at, slot = st["table"][b].long()[pos // page], pos % page
    if st["case"]["cache"] == "16":
        return st["K"][kvh, at, slot].double(), st["V"][kvh, at, slot].double()
    value = torch.tensor(_GRID + [-x for x in _GRID], dtype=torch.float64, device=DEV)
    code = st["codes"][kvh, at, slot]
    x = torch.empty((pos.numel(), 256), dtype=torch.float64, device=DEV)
    x[:, 0::2], x[:, 1::2] = value[(code & 15).long()], value[(code >> 4).long()]
    s = torch.pow(2.0, st["scales"][kvh, at, slot // 4, :, :, slot % 4].double() - 127.0).reshape(-1, 8)
    x = x * s.repeat_interleave(32, dim=1)
    return x[:, :128], x[:, 128:]


def exact(case, seed):
    st = prepare(case, seed)
    new, ctx = _counts(case)
    off = st["off"].tolist()
    if case["kind"] == "append":
        q, K, V = st["q"].double(), st["K"].double(), st["V"].double()
        n = case["rotary"]
        first = [2 * i for i in range(n // 2)] if case["pairs"] == "neighbours" else list(range(n // 2))
        other = [2 * i + 1 for i in range(n // 2)] if case["pairs"] == "neighbours" else list(range(n // 2, n))
        for b in range(case["batch"]):
            pos = torch.arange(ctx[b] - new[b], ctx[b], device=DEV)
            turn = torch.exp(1j * (pos.double()[:, None] * st["inv_freq"].double()))[:, None]      # (a pair of dims as a complex number)
            at, slot = st["table"][b].long()[pos // case["page"]], pos % case["page"]
            k = st["k"][off[b]:off[b + 1]].double()
            for x in (k, q[off[b]:off[b + 1]]):
                z = torch.complex(x[..., first], x[..., other]) * turn
                x[..., first], x[..., other] = z.real, z.imag
            for h in range(case["hkv"]):
                K[h, at, slot] = k[:, h]
                V[h, at, slot] = st["v"][off[b]:off[b + 1], h].double()
        return q, K, V
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(out.shape[:2], dtype=torch.float64, device=DEV)
    for b in range(case["batch"]):
        if not new[b]:
            continue
        m = torch.arange(ctx[b] - new[b], ctx[b], device=DEV)[:, None]
        pos = torch.arange(ctx[b], device=DEV)
        if case["kind"] == "local":
            pos = pos[(pos < case["sink"]) | (pos > ctx[b] - new[b] - case["window"])]
        unseen = pos[None] > m
        if case["kind"] == "local":
            unseen |= (pos[None] >= case["sink"]) & (m - pos[None] >= case["window"])
        for kvh, heads in _served(case):
            k, v = _exact_rows(st, b, kvh, pos)
            for h in heads:
                x = (st["q"][off[b]:off[b + 1], h].double() @ k.T) * 128.0 ** -0.5
                x[unseen] = -math.inf
                z = torch.logsumexp(x, 1)
                out[off[b]:off[b + 1], h] = torch.exp(x - z[:, None]) @ v
                lse[off[b]:off[b + 1], h] = z
    return out if st["lse"] is None else (out, lse)
