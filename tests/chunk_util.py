"""Batches of new tokens over paged caches, for the tests: seeded inputs on the host, and the definition in 64 bits."""
import math

import numpy as np
import torch

from oracle import kv4_oracle as k4

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], dtype=torch.float64)


class Batch:
    """New tokens `new` behind `past` tokens of every sequence, a cache that holds all of them, queries; everything on the CPU."""

    def __init__(self, new, past, hq=8, hkv=2, dtype=torch.bfloat16, page=16, cache="16", order="heads", seed=0, spare=3, gain=1.0, ctx=None):
        g = torch.Generator().manual_seed(seed)
        self.new, self.ctx = list(new), list(ctx) if ctx is not None else [n + p for n, p in zip(new, past)]
        self.hq, self.hkv, self.dtype, self.page, self.kind = hq, hkv, dtype, page, cache
        self.off = [0]
        for n in self.new:
            self.off.append(self.off[-1] + n)
        self.total, B = self.off[-1], len(self.new)
        need = [-(-c // page) for c in self.ctx]
        self.n_pages = sum(need) + spare
        ids = torch.randperm(self.n_pages, generator=g).int()
        self.table = torch.full((B, max(max(need), 1) + 1), -1, dtype=torch.int32)
        at = 0
        for b, k in enumerate(need):
            self.table[b, :k] = ids[at:at + k]
            at += k
        self.q = (torch.randn((self.total + 2, hq, 128), generator=g) * gain).to(dtype)
        rows = torch.randn((2, hkv, self.n_pages, page, 128), generator=g)
        if cache == "16":
            self.rows = rows.to(dtype)
        else:
            code, scale = k4.quantise(rows.to(dtype).double().numpy())       # codes 0 .. 15 [..., 128], scales [..., 4]
            self.code, self.scale = torch.from_numpy(code.astype(np.uint8)), torch.from_numpy(scale.astype(np.uint8))
            self.rows = torch.from_numpy(k4.values(code, scale)).to(dtype)   # (as rtp_kv4_read gives them)
        self.order = order

    def spot(self, b, pos):
        """(page, slot) of a position, or None."""
        k = pos // self.page
        if pos < 0 or k >= self.table.shape[1] or not 0 <= int(self.table[b, k]) < self.n_pages:
            return None
        return int(self.table[b, k]), pos % self.page

    def expected(self, heads, sink=None, window=None, scale=128.0 ** -0.5):
        """{row, head: (out [128], lse, bound of |out - it|, bound of |lse - it|)} in 64 bits; window None: every earlier token.

        The bounds count roundings: the output's, half a step; every probability's, half a step of its own, which moves the quotient of the two sums
        by at most that times the mean distance of the values from it; a logit's 128 products and sums in 32 bits, which move a probability
        by their relative size; the sums over n tokens; in fp16 the steps of 2^-24 below 2^-14 where the sum is 2^-6 or more."""
        half = torch.finfo(self.dtype).eps / 2
        out = {}
        for b, n in enumerate(self.new):
            spots = [self.spot(b, t) for t in range(self.ctx[b])]
            have = [t for t, s in enumerate(spots) if s is not None]
            at = torch.tensor([spots[t][0] * self.page + spots[t][1] for t in have], dtype=torch.long)
            have = torch.tensor(have, dtype=torch.long)
            for h in heads:
                kv = self.rows[:, h // (self.hq // self.hkv)].reshape(2, -1, 128)
                for t in range(n):
                    m = self.ctx[b] - n + t
                    see = have <= m
                    if window is not None:
                        see &= (have < sink) | (have > m - window)
                    k, v = kv[0][at[see]].double(), kv[1][at[see]].double()
                    q = self.q[self.off[b] + t, h].double()
                    if k.shape[0] == 0:
                        out[self.off[b] + t, h] = (torch.zeros(128, dtype=torch.float64), -math.inf, 0.0, 0.0)
                        continue
                    x = (k @ q) * scale
                    lse = torch.logsumexp(x, 0)
                    p = torch.exp(x - lse)
                    o = p @ v
                    size = float((k.abs() @ q.abs()).max() * scale)
                    e_x, e_sum = 128 * 2.0 ** -24 * size + 2.0 ** -21, (k.shape[0] + 64) * 2.0 ** -24
                    spread = (p[:, None] * (v - o).abs()).sum(0)
                    tol = half * o.abs() + 1.02 * (half + 2 * e_x) * spread + 2 * e_sum * (p[:, None] * v.abs()).sum(0) + 1e-30
                    if self.dtype == torch.float16:
                        tol = tol + k.shape[0] * 2.0 ** -25 * 2.0 ** 6 * (v - o).abs().amax(0) + 2.0 ** -25
                    out[self.off[b] + t, h] = (o, float(lse), tol, e_x + e_sum + abs(float(lse)) * 2.0 ** -23 + 2.0 ** -22)
        return out

    # ---- the same on the device ----
    def device(self, fused=True):
        d = "cuda"
        table, off, ctx = self.table.to(d), torch.tensor(self.off, dtype=torch.int32, device=d), torch.tensor(self.ctx, dtype=torch.int32, device=d)
        q = torch.zeros((self.total + 2, self.hq + (2 * self.hkv if fused else 0), 128), dtype=self.dtype, device=d)
        q[:, :self.hq] = self.q.to(d)
        from paper_2605_16928_amd import rtp
        if self.kind == "16":
            K, V = pools(self.rows.to(d), self.order)
            cache = rtp.kv_cache(K, V, table)
        else:
            c = self.code.to(d)
            c = c[..., 0::2] | (c[..., 1::2] << 4)                            # [2, hkv, pages, page, 64]
            codes = torch.cat([c[0], c[1]], -1).contiguous()
            s = self.scale.to(d).view(2, self.hkv, self.n_pages, self.page // 4, 4, 4)
            scales = s.permute(1, 2, 3, 0, 5, 4).contiguous().view(self.hkv, self.n_pages, -1)
            cache = rtp.kv4_cache(codes, scales, table)
        chunk = rtp.chunk_desc(off, ctx, self.total, max(max(self.new), 1), max(max(self.ctx), 1))
        return q[:, :self.hq], cache, chunk


def pools(rows, order):
    """K and V [heads, pages, page_size, 128] of rows [2, heads, pages, page_size, 128], laid out in another order."""
    if order == "heads":
        return rows[0].clone(), rows[1].clone()
    if order == "pages":
        x = rows.permute(0, 2, 1, 3, 4).contiguous()
        return x[0].permute(1, 0, 2, 3), x[1].permute(1, 0, 2, 3)
    if order == "tokens":                                                      # [pages, page_size, heads, 128]
        x = rows.permute(0, 2, 3, 1, 4).contiguous()
        return x[0].permute(2, 0, 1, 3), x[1].permute(2, 0, 1, 3)
    x = torch.cat([rows[0], rows[1]], -1)                                      # "interleaved": K and V of a token side by side
    return x[..., :128], x[..., 128:]


def check(batch, want, out, lse, untouched=None):
    """Every row against its bound; rows and heads that the call does not serve against what they held."""
    out, lse = out.cpu(), None if lse is None else lse.cpu()
    got = out.double()
    worst = 0.0
    for (i, h), (o, z, tol, tol_z) in want.items():
        d = (got[i, h] - o).abs()
        bad = ~(d <= tol)
        assert not bad.any(), f"row {i} head {h}: off by {d[bad].max()} where {torch.as_tensor(tol).expand(128)[bad].min()} is allowed"
        if z > -math.inf:
            worst = max(worst, float((d / tol).max()))
        if lse is not None:
            assert (lse[i, h] == z) if z == -math.inf else abs(float(lse[i, h]) - z) <= tol_z, f"row {i} head {h}: lse {float(lse[i, h])}, {z}"
    if untouched is not None:
        mask = torch.ones(out.shape[:2], dtype=torch.bool)
        for i, h in want:
            mask[i, h] = False
        assert (got[mask] == untouched).all()
        assert lse is None or (lse[mask] == untouched).all()
    return worst
