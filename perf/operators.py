"""The 4-bit K/V cache and the pages it lives in, as measurable cases.

  store   tokens are quantised into a paged 4-bit cache (rtp_kv4_append) and read back at 16 bits (rtp_kv4_read): one token per
          sequence in a decode step, a chunk and the whole context behind it in a chunked prefill.
  sparse  decode attention of the retrieval heads over selected tokens of that cache (rtp_sparse_attn_decode_kv4).
  local   sink + sliding-window attention of the other heads over that cache, decode (rtp_local_attn_kv4).
  dense   attention of every head over every token of that cache, decode (rtp_dense_attn_kv4).
  fork    samples are dropped and drawn anew from kept prompts: their pages are released, the prompts' pages shared, fresh pages
          handed out and the shared last pages copied before they are written to (rtp_kv_pages_truncate, _fork, _extend, _copy).
  compact the pages in use move to the front of the pools (rtp_kv_pages_compact, _copy).

The 4-bit format: a row's 128 values are 4 blocks of 32; a block is a scale byte s that stands for 2^(s - 127) and 32 codes of a
sign, 2 exponent bits and 1 mantissa bit (0, .5, 1, 1.5, 2, 3, 4, 6).  s puts the block's largest magnitude into [3.5, 7) steps; 255
marks a block with a value that is not finite.  codes: uint8 [kv heads, pages, page_size, 128], a token's K in the first 64 bytes (dim
2i in the low half of byte i) and its V in the rest; scales: uint8 [kv heads, pages, page_size / 4, K or V, block, token % 4].

Sizes are fixed by the case alone; the seed draws the values and the placing of the pages.
"""
import math
import random

import torch

DEV = "cuda:0"
own = False

HEADS = [(8, 2), (32, 8), (64, 8), (32, 4), (16, 16), (8, 4)]     # query heads, KV heads: groups of 1, 2, 4 and 8
PAGES = [16, 32, 64, 128, 256]
MOST_ROWS = 1 << 23        # (token, KV head) rows of the largest case


def _case(name, kind, **kw):
    c = dict(name=name, kind=kind, hq=32, hkv=8, dtype="bf16", page=64, batch=1, lo=4096, hi=4096)
    c.update(kw)
    return c


def listed():
    return [
        # a decode step of 32 sequences: K and V of one new token each, slices of the fused projection
        _case("store_step", "store", batch=32, lo=16384, hi=262144, T=1, ragged=False, read="new", layout="qkv"),
        # a mixed batch of a server: up to 1000 new tokens a sequence, some with none, fp16
        _case("store_ragged_fp16", "store", hkv=4, batch=6, lo=1, hi=3000, T=1000, ragged=True, read="new", layout="qkv",
              dtype="fp16", page=16),
        # one chunk of a chunked prefill: 4096 tokens are stored, the 32768 tokens so far are read back for its attention
        _case("store_chunk", "store", lo=28672, hi=28672, T=4096, ragged=False, read="all", layout="heads"),
        # a short conversation on a small layer: a hundred selected tokens
        _case("sparse_4k", "sparse", hq=8, hkv=2, n_ret=2, sel_lo=100, sel_hi=100),
        # a server's ordinary batch of ragged contexts in fp16, some rows without a selected token
        _case("sparse_ragged_fp16", "sparse", hkv=4, n_ret=4, batch=12, lo=1500, hi=30011, sel_lo=0, sel_hi=4001, dtype="fp16"),
        # a large mixed batch: 32 contexts from 16K to 262K, selections that differ by a factor of 100 and more
        _case("sparse_mixed", "sparse", hq=64, n_ret=8, batch=32, lo=16384, hi=262144, sel_lo=200, sel_hi=30000),
        # a short window on a small layer
        _case("local_512", "local", hq=8, hkv=2, n_ret=2, sink=4, window=512),
        # the paper's window on a batch of ragged contexts, some shorter than the window
        _case("local_8k", "local", n_ret=4, batch=32, lo=1000, hi=100003, sink=4, window=8192, page=16),
        # one short sequence, every token
        _case("dense_4k", "dense", hq=8, hkv=2),
        # long contexts, every token: the largest cache that one step streams
        _case("dense_128k", "dense", batch=8, lo=131072, hi=131072),
        # 64 samples drawn anew from 8 kept prompts of up to 30K tokens, 100 tokens of room each
        _case("fork_64", "fork", batch=8, children=8, lo=1500, hi=30011, grow=100),
        # a pool of 4096 pages of which 40 % are in use, all over it
        _case("compact_4096", "compact", pool=4096, used=1638, moves=983, batch=24),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    hq, hkv = rng.choice(HEADS)
    kind = rng.choice(["store", "sparse", "sparse", "local", "dense", "dense", "fork", "compact"])
    c = dict(kind=kind, hq=hq, hkv=hkv, dtype=rng.choice(["bf16", "bf16", "fp16"]), page=rng.choice(PAGES))
    if kind == "store":
        T = _log(rng, 1, 8192)
        c.update(batch=_log(rng, 1, max(1, min(64, 65536 // (T * hkv)))), T=T, lo=0, hi=_log(rng, 1, 32768 // hkv),
                 ragged=rng.random() < 0.5, read=rng.choice(["new", "all"]), layout=rng.choice(["qkv", "heads"]))
    elif kind == "sparse":
        n_ret = rng.randint(1, min(8, hq))
        batch = _log(rng, 1, 32)
        hi = _log(rng, 64, min(262144, MOST_ROWS // (2 * batch * hkv)))
        sel = _log(rng, 1, min(hi, MOST_ROWS // (2 * batch * n_ret)))
        c.update(batch=batch, n_ret=n_ret, lo=max(1, hi // rng.choice([1, 3, 16])), hi=hi,
                 sel_lo=rng.choice([0, 1, max(1, sel // 7), sel]), sel_hi=sel)
    elif kind == "local":
        batch = _log(rng, 1, 64)
        window = _log(rng, 16, 8192)
        hi = _log(rng, 1, min(131072, MOST_ROWS // (2 * batch * hkv)))
        c.update(batch=batch, n_ret=rng.randint(0, min(8, hq - 1)), lo=max(1, hi // rng.choice([1, 4, 50])), hi=hi,
                 sink=rng.choice([0, 4, 4, 17]), window=window)
    elif kind == "dense":
        batch = _log(rng, 1, 32)
        hi = _log(rng, 1, min(262144, MOST_ROWS // (2 * batch * hkv)))
        c.update(batch=batch, lo=max(1, hi // rng.choice([1, 2, 10])), hi=hi)
    elif kind == "fork":
        c.update(batch=_log(rng, 1, 16), children=_log(rng, 1, 16), hi=_log(rng, 1, 32768 // hkv), grow=_log(rng, 1, 500))
        c["lo"] = max(1, c["hi"] // 5)
    else:
        pool = _log(rng, 32, max(64, (1 << 19) // (c["page"] * hkv)))
        used = rng.randint(1, pool)
        c.update(pool=pool, used=used, moves=rng.randint(0, min(used, pool - used)), batch=_log(rng, 1, 32))
    return c


# ---- sizes, from the case alone ---------------------------------------------------------------------------------------------
def _lengths(case, lo, hi, n, salt):
    """n lengths between lo and hi, spread over their logarithm; the first is hi.  lo = 0: a quarter of the others are 0."""
    rng = random.Random("%s %d %d %d" % (salt, lo, hi, n))
    return [hi] + [0 if lo < 1 and rng.random() < 0.25 else _log(rng, max(lo, 1), hi) for _ in range(n - 1)]


def _ret_heads(case):
    """Retrieval heads, spread over the KV heads."""
    n, hq = case.get("n_ret", 0), case["hq"]
    return sorted({(j * hq) // n for j in range(n)}) if n else []


def _counts(case):
    """Stored tokens, start positions / context lengths, selected tokens: what the case's calls work on."""
    ctx = _lengths(case, case["lo"], case["hi"], case["batch"], "context")
    if case["kind"] == "store":
        new = _lengths(case, 0, case["T"], case["batch"], "new") if case["ragged"] else [case["T"]] * case["batch"]
        return ctx, new
    if case["kind"] == "sparse":
        rows = case["batch"] * case["n_ret"]
        sel = _lengths(case, case["sel_lo"], case["sel_hi"], rows, "selected")
        return ctx, [min(s, ctx[r // case["n_ret"]]) for r, s in enumerate(sel)]
    return ctx, None


def _local_tokens(n, sink, window):
    return min(sink, n) + max(0, n - max(sink, n - window))


def work(case):
    """Bytes and operations that a pass cannot do without."""
    kind, hq, hkv, B = case["kind"], case["hq"], case["hkv"], case.get("batch", 1)
    row = 136                                   # 64 + 64 bytes of codes, 4 + 4 of scales
    if kind == "store":
        ctx, new = _counts(case)
        read = sum(new) if case["read"] == "new" else sum(c + n for c, n in zip(ctx, new))
        return {"bytes": hkv * (sum(new) * (512 + row) + read * (row + 512)), "flops": 0}
    if kind in ("sparse", "local", "dense"):
        ctx, sel = _counts(case)
        group, ret = hq // hkv, _ret_heads(case)
        if kind == "sparse":
            rows, pairs, heads = sum(sel), sum(sel), len(ret)
            extra = 4 * sum(sel)
        else:
            n = sum(ctx) if kind == "dense" else sum(_local_tokens(c, case["sink"], case["window"]) for c in ctx)
            heads = hq - (len(ret) if kind == "local" else 0)
            streams = len({h // group for h in range(hq) if kind == "dense" or h not in ret})
            rows, pairs = n * streams, n * heads
            extra = 4 * sum(-(-c // case["page"]) for c in ctx)
        return {"bytes": rows * row + extra + B * heads * (256 + 256 + 4), "flops": pairs * 4 * 128}
    page = case["page"] * hkv * 512
    if kind == "fork":
        lens = _lengths(case, case["lo"], case["hi"], B, "context")
        kids = case["children"]
        shared = sum(1 for n in lens if n % case["page"]) * kids
        entries = sum(-(-(n + case["grow"]) // case["page"]) for n in lens) * kids
        return {"bytes": 2 * shared * page + 4 * 6 * entries, "flops": 0}
    return {"bytes": 2 * case["moves"] * page + 8 * case["pool"] + 8 * case["used"], "flops": 0}


# ---- inputs ---------------------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def _rows_like(shape, g, gain):
    """Keys or values: normal, with channels of different size, as a model's are."""
    return torch.randn(shape, generator=g, device=DEV) * gain


def _gains(g, hkv, sigma):
    return torch.exp(sigma * torch.randn((hkv, 1, 128), generator=g, device=DEV))


def _pool(case, g, n_pages):
    """A 4-bit pool filled with quantised rows (codes, scales)."""
    hkv, page = case["hkv"], case["page"]
    codes = torch.empty((hkv, n_pages, page, 128), dtype=torch.uint8, device=DEV)
    scales = torch.empty((hkv, n_pages, page // 4, 2, 4, 4), dtype=torch.uint8, device=DEV)
    gains = _gains(g, hkv, 0.5), _gains(g, hkv, 0.2)
    step = max(1, (1 << 20) // (page * hkv))
    for p0 in range(0, n_pages, step):
        p1 = min(n_pages, p0 + step)
        for w in (0, 1):
            x = _rows_like((hkv, (p1 - p0) * page, 128), g, gains[w]).to(_dtype(case))
            c, s = quantise(x)
            codes[:, p0:p1, :, 64 * w:64 * w + 64] = c.view(hkv, p1 - p0, page, 64)
            scales[:, p0:p1, :, w] = s.view(hkv, p1 - p0, page // 4, 4, 4).transpose(3, 4)
    return codes, scales


def _table(case, g, lens, n_spare=3):
    """Every sequence's pages, anywhere in the pool; -1 behind them."""
    need = [-(-n // case["page"]) for n in lens]
    n_pages = sum(need) + n_spare
    ids = torch.randperm(n_pages, generator=g, device=DEV).int()
    table = torch.full((len(lens), max(max(need), 1) + 1), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = ids[at:at + k]
        at += k
    return table, n_pages


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g = _gen(seed)
    kind, hq, hkv, B = case["kind"], case["hq"], case["hkv"], case["batch"]
    st = dict(case=case, kind=kind)
    if kind == "store":
        start, new = _counts(case)
        T = case["T"]
        table, n_pages = _table(case, g, [s + n for s, n in zip(start, new)])
        st["codes"], st["scales"] = _pool(case, g, n_pages)
        gk, gv = _gains(g, hkv, 0.5), _gains(g, hkv, 0.2)
        if case["layout"] == "qkv":             # [B, T, (hq + 2 hkv) * 128], as a fused projection leaves it
            qkv = torch.randn((B, T, hq + 2 * hkv, 128), generator=g, device=DEV)
            qkv[:, :, hq:hq + hkv] *= gk.view(1, 1, hkv, 128)
            qkv[:, :, hq + hkv:] *= gv.view(1, 1, hkv, 128)
            qkv = qkv.to(_dtype(case))
            st["k"], st["v"] = qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]
        else:                                   # [hkv, B, T, 128], as the prefill's own cache has it
            st["k"] = _rows_like((hkv, B * T, 128), g, gk).to(_dtype(case)).view(hkv, B, T, 128).permute(1, 2, 0, 3)
            st["v"] = _rows_like((hkv, B * T, 128), g, gv).to(_dtype(case)).view(hkv, B, T, 128).permute(1, 2, 0, 3)
        first = [0] * B if case["read"] == "all" else start
        count = [s + n - f for s, n, f in zip(start, new, first)]
        st.update(table=table, start=_i32(start), new=_i32(new), first=_i32(first), count=_i32(count), R=max(count))
        st["out"] = [torch.zeros((hkv, B, st["R"], 128), dtype=_dtype(case), device=DEV) for _ in range(2)]
        return st
    if kind in ("sparse", "local", "dense"):
        ctx, sel = _counts(case)
        st["table"], n_pages = _table(case, g, ctx)
        st["codes"], st["scales"] = _pool(case, g, n_pages)
        st["q"] = torch.randn((B, hq, 128), generator=g, device=DEV).to(_dtype(case))
        st.update(ctx=_i32(ctx), max_ctx=max(ctx), ret=_ret_heads(case))
        st["out"] = torch.zeros((B, hq, 128), dtype=_dtype(case), device=DEV)
        st["lse"] = torch.zeros((B, hq), dtype=torch.float32, device=DEV)
        if kind == "sparse":                    # ascending positions, as a selector leaves them: half scattered, half in runs
            st["max_sel"] = max(max(sel), 1)
            idx = torch.zeros((len(sel), (st["max_sel"] + 3) // 4 * 4), dtype=torch.int32, device=DEV)
            for r, n in enumerate(sel):
                c = ctx[r // case["n_ret"]]
                runs = torch.randperm(-(-c // 8), generator=g, device=DEV)
                pos = (runs[:-(-n // 8), None] * 8 + torch.arange(8, device=DEV)).flatten()
                pos = pos[pos < c][:n // 2]
                free = torch.ones(c, dtype=torch.bool, device=DEV)
                free[pos] = False
                rest = free.nonzero().flatten()
                rest = rest[torch.randperm(rest.numel(), generator=g, device=DEV)[:n - pos.numel()]]
                idx[r, :n] = torch.cat([pos, rest]).sort().values.int()
            st.update(sel_idx=idx, sel_count=_i32(sel))
        return st
    page, dt = case["page"], _dtype(case)
    if kind == "fork":
        lens = _lengths(case, case["lo"], case["hi"], B, "context")
        kids, grow = case["children"], case["grow"]
        room = max(-(-(n + grow) // page) for n in lens)
        need = [-(-n // page) for n in lens]
        n_pages = sum(need) + kids * sum(-(-(n + grow) // page) - n // page for n in lens) + 5
        ids = torch.randperm(n_pages, generator=g, device=DEV).int()
        table = torch.full((B * (1 + kids), room), -1, dtype=torch.int32, device=DEV)
        at = 0
        for b, k in enumerate(need):
            table[b, :k] = ids[at:at + k]
            at += k
        refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
        refs[ids[:at].long()] = 1
        parents = [b for b in range(B) for _ in range(kids)]
        st.update(table=table, refs=refs, n_pages=n_pages, parents=_i32(parents),
                  children=_i32(list(range(B, B + B * kids))), old=_i32([lens[b] for b in parents]),
                  new=_i32([lens[b] + grow for b in parents]))
    else:
        pool, used, moves = case["pool"], case["used"], case["moves"]
        low = torch.randperm(used, generator=g, device=DEV)[:used - moves]
        high = used + torch.randperm(max(pool - used, 1), generator=g, device=DEV)[:moves]
        ids = torch.cat([low, high])
        ids = ids[torch.randperm(used, generator=g, device=DEV)]
        room = -(-used // B) + 2
        table = torch.full((B, room), -1, dtype=torch.int32, device=DEV)
        refs = torch.zeros(pool, dtype=torch.int32, device=DEV)
        refs[ids] = 1
        for b in range(B):                      # every sequence a slice of the pages; each but the first shares the first page
            mine = ids[b * used // B:(b + 1) * used // B]
            table[b, :mine.numel()] = mine.int()
            if b:
                table[b, room - 1] = ids[0].int()
                refs[ids[0]] += 1
        st.update(table=table.clone(), refs=refs.clone(), table0=table, refs0=refs, n_pages=pool)
    st["K"] = torch.randn((hkv, st["n_pages"], page * 128), generator=g, device=DEV, dtype=torch.float32).to(dt)
    st["V"] = torch.randn((hkv, st["n_pages"], page * 128), generator=g, device=DEV, dtype=torch.float32).to(dt)
    return st


# ---- plain forms ------------------------------------------------------------------------------------------------------------------
def quantise(x):
    """(codes uint8 [..., 64], scales uint8 [..., 4]) of rows [..., 128]."""
    y = x.float().unflatten(-1, (4, 32))
    amax = y.abs().amax(-1, keepdim=True)
    bits = amax.view(torch.int32)
    e = (bits >> 23) - 2 + ((bits & 0x7fffff) >= 0x600000).int()
    e = torch.where(amax.isfinite(), e.clamp(min=2), 255)
    y = y * torch.exp2(127.0 - e.clamp(max=254).float())
    a = y.abs()
    code = (a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() + (a >= 3.5).byte() \
        + (a > 5.0).byte()
    code = torch.where(e == 255, 0, code | ((y < 0).byte() << 3)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), e.squeeze(-1).byte()


def _value_pairs():
    """The two values of every byte, [256, 2]."""
    byte = torch.arange(256, device=DEV)
    nibble = torch.stack([byte & 15, byte >> 4], dim=1)
    mag = torch.where((nibble & 7) < 2, 0.5 * (nibble & 7), (1 + 0.5 * (nibble & 1)) * torch.exp2(((nibble & 7) >> 1) - 1.0))
    return torch.where(nibble < 8, mag, -mag).float()


def _values(codes, scales):
    """Rows [..., 128] in 32 bits of codes [..., 64] and scale bytes [..., 4]."""
    x = _value_pairs()[codes.int()].flatten(-2).unflatten(-1, (4, 32))
    s = torch.exp2(scales.float() - 127.0)
    return (x * torch.where(scales == 255, math.nan, s).unsqueeze(-1)).flatten(-2)


def _fetch(st, page, slot, head=None):
    """K and V rows in 32 bits of the tokens at `slot` of pool page `page`; every KV head's ([hkv, ...]), or `head`'s of the same shape."""
    h = slice(None) if head is None else head
    codes = st["codes"][h, page, slot]
    scales = st["scales"][h, page, slot // 4, :, :, slot % 4]
    if head is None:                            # (an index in front of and behind the slices: its dims come first)
        scales = scales.movedim(-3, 0)
    return _values(codes[..., :64], scales[..., 0, :]), _values(codes[..., 64:], scales[..., 1, :])


def _softmax(st, logits, keep):
    """Probabilities and log-sum of the kept logits; rows that keep nothing have none."""
    x = torch.where(keep, logits, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.where(keep, torch.exp(x - torch.where(m.isfinite(), m, 0.0)), 0.0)
    total = p.sum(-1, keepdim=True)
    lse = torch.log(total) + torch.where(m.isfinite(), m, 0.0)
    return torch.where(total > 0, p / total, 0.0), lse.squeeze(-1)


def _plain_store(st):
    case, B, R, T = st["case"], st["case"]["batch"], st["R"], st["case"]["T"]
    page, table = case["page"], st["table"].long()
    t = torch.arange(T, device=DEV)
    b, t = torch.nonzero(t[None, :] < st["new"][:, None], as_tuple=True)
    pos = st["start"][b].long() + t
    at, slot = table[b, pos // page], pos % page
    for w, x in enumerate((st["k"], st["v"])):
        code, scale = quantise(x[b, t].transpose(0, 1))
        st["codes"][:, at, slot, 64 * w:64 * w + 64] = code
        st["scales"][:, at, slot // 4, w, :, slot % 4] = scale.transpose(0, 1)
    r = torch.arange(R, device=DEV)
    b, r = torch.nonzero(r[None, :] < st["count"][:, None], as_tuple=True)
    pos = st["first"][b].long() + r
    rows = _fetch(st, table[b, pos // page], pos % page)
    st["out"][0][:, b, r] = rows[0].to(_dtype(case))
    st["out"][1][:, b, r] = rows[1].to(_dtype(case))
    return st["out"]


def _plain_dense(st):
    """Every token of the padded batch; `local` keeps the sink and the window of them."""
    case, B, group = st["case"], st["case"]["batch"], st["case"]["hq"] // st["case"]["hkv"]
    n = st["ctx"].long()[:, None]
    pos = torch.arange(st["max_ctx"], device=DEV)[None, :].expand(B, -1)
    if st["kind"] == "local":                   # the tokens of the set alone, padded to the longest
        width = min(st["max_ctx"], case["sink"] + case["window"])
        i = torch.arange(width, device=DEV)[None, :]
        w0 = (n - case["window"]).clamp(min=case["sink"])
        s0 = n.clamp(max=case["sink"])
        pos = torch.where(i < s0, i, w0 + i - s0)
    keep = pos < n
    pos = torch.where(keep, pos, 0)
    k, v = _fetch(st, st["table"].long().gather(1, pos // case["page"]).clamp(min=0), pos % case["page"])   # [hkv, B, n, 128]
    q = st["q"].float().view(B, case["hkv"], group, 128).transpose(0, 1)
    logits = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(128.0)
    p, lse = _softmax(st, logits, keep[None, :, None, :])
    out = torch.matmul(p, v).transpose(0, 1).reshape(B, case["hq"], 128)
    lse = lse.transpose(0, 1).reshape(B, case["hq"])
    if st["kind"] == "local" and st["ret"]:     # the retrieval heads' rows stay as they were
        ret = torch.zeros(case["hq"], dtype=torch.bool, device=DEV).index_fill(0, torch.tensor(st["ret"], device=DEV), True)
        out, lse = torch.where(ret[:, None], 0.0, out), torch.where(ret, 0.0, lse)
    return out.to(_dtype(case)), lse


def _plain_sparse(st):
    case, n_ret = st["case"], st["case"]["n_ret"]
    group, page = case["hq"] // case["hkv"], case["page"]
    rows = st["sel_count"].numel()
    b = torch.arange(rows, device=DEV) // n_ret
    h = torch.tensor(st["ret"], device=DEV)[torch.arange(rows, device=DEV) % n_ret]
    keep = torch.arange(st["max_sel"], device=DEV)[None, :] < st["sel_count"][:, None]
    pos = torch.where(keep, st["sel_idx"][:, :st["max_sel"]], 0).long()
    at = st["table"].long()[b[:, None], pos // page].clamp(min=0)
    k, v = _fetch(st, at, pos % page, (h // group)[:, None])
    logits = torch.matmul(k, st["q"][b, h].float().unsqueeze(-1)).squeeze(-1) / math.sqrt(128.0)
    p, lse = _softmax(st, logits, keep)
    out = torch.zeros_like(st["out"])
    out[b, h] = torch.matmul(p.unsqueeze(1), v).squeeze(1).to(out.dtype)
    all_lse = torch.zeros_like(st["lse"])
    all_lse[b, h] = lse
    return out, all_lse


def _plain_fork(st):
    case, page, room = st["case"], st["case"]["page"], st["table"].shape[1]
    table, refs, kids = st["table"], st["refs"], st["children"].long()
    # the children's pages are released
    held = table[kids]
    refs.index_add_(0, held.clamp(min=0).flatten().long(), -(held >= 0).int().flatten())
    # the parents' pages are shared
    k = torch.arange(room, device=DEV)[None, :]
    old, new = st["old"][:, None], st["new"][:, None]
    mine = torch.where(k * page < old, table[st["parents"].long()], -1)
    refs.index_add_(0, mine.clamp(min=0).flatten().long(), (mine >= 0).int().flatten())
    # fresh pages, the lowest free ones in order: for the shared last page, then for the new tokens
    last = (k == old // page) & (old % page != 0) & (refs[mine.clamp(min=0).long()] > 1) & (new > old)
    fresh = last | ((k * page >= old) & (k * page < new))
    rank = torch.cumsum(fresh.flatten().int(), 0).view(fresh.shape) - 1
    ids = torch.arange(st["n_pages"], device=DEV)
    free = torch.argsort(torch.where(refs == 0, ids, ids + st["n_pages"]))
    given = torch.where(fresh, free[rank.clamp(min=0)], 0)
    n_free = (refs == 0).sum()
    refs.index_add_(0, torch.where(last, mine, 0).flatten().long(), -last.flatten().int())
    refs.index_add_(0, given.flatten(), fresh.flatten().int())
    table[kids] = torch.where(fresh, given.int(), mine)
    # the shared last pages are copied: where there is none, a page onto itself
    src = torch.where(last, mine, 0).sum(1).long()
    dst = torch.where(last, given, 0).sum(1).long()
    st["K"][:, dst] = st["K"][:, src]
    st["V"][:, dst] = st["V"][:, src]
    status = torch.stack([torch.zeros_like(n_free), n_free - fresh.sum()]).int()
    return table, refs, status, st["K"], st["V"]


def _plain_compact(st):
    table, refs, n = st["table"], st["refs"], st["n_pages"]
    table.copy_(st["table0"])
    refs.copy_(st["refs0"])
    used = refs > 0
    n_used = used.sum()
    ids = torch.arange(n, device=DEV)
    holes = torch.nonzero(~used & (ids < n_used)).flatten()              # ascending
    movers = torch.nonzero(used & (ids >= n_used)).flatten().flip(0)     # the highest first
    to = ids.clone()
    to[movers] = holes
    st["K"][:, holes] = st["K"][:, movers]
    st["V"][:, holes] = st["V"][:, movers]
    refs[holes] = refs[movers]
    refs[movers] = 0
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].int(), table))
    status = torch.stack([n_used, torch.full_like(n_used, holes.numel())]).int()
    return table, refs, status, st["K"], st["V"]


# ---- the framework's calls -----------------------------------------------------------------------------------------------------------
def _handles(st):
    """What a program keeps from call to call: the layer's and the cache's descriptors, workspaces."""
    if "layer" in st:
        return
    from paper_2605_16928_amd import rtp
    case = st["case"]
    st["layer"] = rtp.layer_desc(case["hq"], case["hkv"], _ret_heads(case), case.get("sink", 4), case.get("window", 64),
                                 kv_dtype=rtp.RTP_DTYPE_BF16 if case["dtype"] == "bf16" else rtp.RTP_DTYPE_FP16)
    size = 256
    if "codes" in st:
        st["cache"] = rtp.kv4_cache(st["codes"], st["scales"], st["table"])
        if st["kind"] == "sparse":
            size = rtp.rtp_sparse_attn_decode_kv4_workspace_bytes(st["layer"], case["batch"], st["max_sel"])
        elif st["kind"] == "local":
            size = rtp.rtp_local_attn_kv4_workspace_bytes(st["layer"], case["batch"], st["max_ctx"])
        elif st["kind"] == "dense":
            size = rtp.rtp_dense_attn_kv4_workspace_bytes(st["layer"], case["batch"], st["max_ctx"])
    else:
        st["map"] = rtp.page_map(st["table"], st["refs"], case["page"])
        st["pools"] = rtp.page_pools([st["K"], st["V"]])
        pairs = st["children"].numel() if st["kind"] == "fork" else st["n_pages"]
        st["src"], st["dst"] = (torch.empty(pairs, dtype=torch.int32, device=DEV) for _ in range(2))
        st["status"] = torch.zeros(2, dtype=torch.int32, device=DEV)
        size = rtp.rtp_kv_pages_workspace_bytes(st["map"], pairs)
    st["ws"] = torch.empty(max(256, size), dtype=torch.uint8, device=DEV)


def _own(st):
    from paper_2605_16928_amd import rtp
    _handles(st)
    case, kind = st["case"], st["kind"]
    if kind == "store":
        k, v, (ko, vo) = st["k"], st["v"], st["out"]
        rtp.rtp_kv4_append(st["layer"], st["cache"], k, v, k.stride(0), k.stride(1), k.stride(2), st["start"], st["new"],
                           case["batch"], case["T"])
        rtp.rtp_kv4_read(st["layer"], st["cache"], st["first"], st["count"], case["batch"], st["R"], ko, vo,
                         ko.stride(1), ko.stride(2), ko.stride(0))
        return st["out"]
    if kind == "sparse":
        rtp.rtp_sparse_attn_decode_kv4(st["layer"], st["q"], st["cache"], st["sel_idx"], st["sel_idx"].stride(0), st["sel_count"],
                                       st["max_sel"], case["batch"], st["out"], st["lse"], st["ws"])
        return st["out"], st["lse"]
    if kind in ("local", "dense"):
        call = rtp.rtp_local_attn_kv4 if kind == "local" else rtp.rtp_dense_attn_kv4
        call(st["layer"], st["q"], st["cache"], st["ctx"], case["batch"], st["max_ctx"], st["out"], st["lse"], st["ws"])
        return st["out"], st["lse"]
    if kind == "fork":
        n = st["children"].numel()
        rtp.rtp_kv_pages_truncate(st["map"], st["children"], None, n)
        rtp.rtp_kv_pages_fork(st["map"], st["parents"], st["children"], st["old"], n)
        rtp.rtp_kv_pages_extend(st["map"], st["children"], st["old"], st["new"], n, st["src"], st["dst"], st["status"], st["ws"])
        rtp.rtp_kv_pages_copy(st["pools"], st["n_pages"], st["src"], st["dst"], n, None)
    else:
        st["table"].copy_(st["table0"])
        st["refs"].copy_(st["refs0"])
        rtp.rtp_kv_pages_compact(st["map"], st["src"], st["dst"], st["status"], st["ws"])
        rtp.rtp_kv_pages_copy(st["pools"], st["n_pages"], st["src"], st["dst"], st["n_pages"], st["status"][1:])
    return st["table"], st["refs"], st["status"], st["K"], st["V"]


def run(state):
    if own:
        return _own(state)
    kind = state["kind"]
    if kind == "store":
        return _plain_store(state)
    if kind == "sparse":
        return _plain_sparse(state)
    if kind in ("local", "dense"):
        return _plain_dense(state)
    return _plain_fork(state) if kind == "fork" else _plain_compact(state)


# ---- the definition, in 64 bits ---------------------------------------------------------------------------------------------------------
_GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _exact_rows(st, b, pos, kvh):
    """K and V in 64 bits of positions `pos` of sequence b, one KV head."""
    page = st["case"]["page"]
    at, slot = st["table"][b].long()[pos // page], pos % page
    sign = torch.tensor(_GRID + [-x for x in _GRID], dtype=torch.float64, device=DEV)
    code = st["codes"][kvh, at, slot]
    x = sign[torch.stack([code & 15, code >> 4], dim=-1).long()].view(pos.numel(), 2, 4, 32)
    s = st["scales"][kvh, at, slot // 4, :, :, slot % 4].double() - 127.0
    x = (x * torch.pow(2.0, s).unsqueeze(-1)).view(pos.numel(), 2, 128)
    return x[:, 0], x[:, 1]


def _exact_nearest(x):
    """Rows [..., 128] as the values that their 4-bit form stands for: the nearest point of the grid, of two the one with the even code."""
    y = x.double().unflatten(-1, (4, 32))
    m, e = torch.frexp(y.abs().amax(-1, keepdim=True))
    e = (e - 3 + (m >= 0.875).int()).clamp(min=-125).double()
    unit = torch.pow(2.0, e)
    far = [((y.abs() / unit - p).abs() + (1e-9 if i % 2 else 0.0)) for i, p in enumerate(_GRID)]
    best = torch.stack(far, 0).argmin(0)
    return (torch.tensor(_GRID, dtype=torch.float64, device=DEV)[best] * unit * torch.where(y < 0, -1.0, 1.0)).flatten(-2)


def exact(case, seed):
    st = prepare(case, seed)
    kind, hq, hkv, B = case["kind"], case["hq"], case["hkv"], case["batch"]
    if kind == "store":
        outs = [torch.zeros(o.shape, dtype=torch.float64, device=DEV) for o in st["out"]]
        start, new = _counts(case)
        for b in range(B):
            first, count = int(st["first"][b]), int(st["count"][b])
            for kvh in range(hkv):
                if start[b] > first:
                    old = _exact_rows(st, b, torch.arange(first, start[b], device=DEV), kvh)
                    for w in (0, 1):
                        outs[w][kvh, b, :start[b] - first] = old[w]
                for w, x in enumerate((st["k"], st["v"])):
                    if new[b]:
                        outs[w][kvh, b, start[b] - first:count] = _exact_nearest(x[b, :new[b], kvh])
        return outs
    if kind in ("sparse", "local", "dense"):
        ctx, sel = _counts(case)
        group, ret = hq // hkv, st["ret"]
        out = torch.zeros((B, hq, 128), dtype=torch.float64, device=DEV)
        lse = torch.zeros((B, hq), dtype=torch.float64, device=DEV)
        for b in range(B):
            t = torch.arange(ctx[b], device=DEV)
            if kind == "local":
                t = t[(t < case["sink"]) | (t > ctx[b] - 1 - case["window"])]
            for kvh in range(hkv):
                heads = [h for h in range(kvh * group, (kvh + 1) * group) if (h in ret) == (kind == "sparse") or kind == "dense"]
                if heads and kind != "sparse":
                    k, v = _exact_rows(st, b, t, kvh)
                for h in heads:
                    if kind == "sparse":
                        row = b * len(ret) + ret.index(h)
                        k, v = _exact_rows(st, b, st["sel_idx"][row, :sel[row]].long(), kvh)
                    if not k.shape[0]:
                        lse[b, h] = -math.inf
                        continue
                    x = (k @ st["q"][b, h].double()) * 128.0 ** -0.5
                    top = x.max()
                    w = torch.exp(x - top)
                    out[b, h], lse[b, h] = (w @ v) / w.sum(), torch.log(w.sum()) + top
        return out, lse
    page = case["page"]
    table, refs = st["table"].tolist(), st["refs"].tolist()
    if kind == "fork":
        pairs = []
        for src, dst, n in zip(st["parents"].tolist(), st["children"].tolist(), st["old"].tolist()):
            for k in range(-(-n // page)):
                table[dst][k] = table[src][k]
                refs[table[src][k]] += 1
        free = [p for p in range(len(refs)) if refs[p] == 0]
        shared, given = list(refs), 0
        for dst, n, new in zip(st["children"].tolist(), st["old"].tolist(), st["new"].tolist()):
            wanted = list(range(-(-n // page), -(-new // page)))
            if new > n and n % page and shared[table[dst][n // page]] > 1:
                wanted.insert(0, n // page)
                pairs.append((table[dst][n // page], free[given]))
                refs[table[dst][n // page]] -= 1
            for k in wanted:
                table[dst][k] = free[given]
                refs[free[given]] += 1
                given += 1
        status = [0, len(free) - given]
    else:
        used = [p for p in range(len(refs)) if refs[p] > 0]
        high = [p for p in reversed(used) if p >= len(used)]
        low = [p for p in range(len(used)) if refs[p] == 0]
        pairs, to = list(zip(high, low)), dict(zip(high, low))
        for p, q in pairs:
            refs[q], refs[p] = refs[p], 0
        table = [[to.get(p, p) for p in row] for row in table]
        status = [len(used), len(pairs)]
    pools = [st["K"].double(), st["V"].double()]
    for x in pools:
        if pairs:
            src, dst = (torch.tensor(p, device=DEV) for p in zip(*pairs))
            x[:, dst] = x[:, src].clone()
    return _i32(table), _i32(refs), _i32(status), pools[0], pools[1]
