"""rtp_kv_append on the GPU: rotation and storing of new tokens in 16-bit pages, against the definition in 64 bits."""
import pytest
import torch

from chunk_util import pools
from paper_2605_16928_amd import rtp

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def turned(x, pos, inv_freq, interleaved, scale):
    """Rows [tokens, heads, 128] rotated, in 64 bits, and the magnitudes that its rounding errors go by."""
    r = 2 * inv_freq.numel()
    a = pos.double()[:, None] * inv_freq.double()[None]
    cos, sin = scale * torch.cos(a)[:, None], scale * torch.sin(a)[:, None]
    y, size = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    i = slice(0, r, 2) if interleaved else slice(0, r // 2)
    j = slice(1, r, 2) if interleaved else slice(r // 2, r)
    u, v = x[..., i].double(), x[..., j].double()
    y[..., i], y[..., j] = u * cos - v * sin, v * cos + u * sin
    size[..., i] = size[..., j] = scale * (u.abs() + v.abs())
    return y, size


def near(got, want, size, dtype):
    """One rounding to 16 bits (half a step, or half of the smallest), and 32-bit products whose cos and sin are within 2^-21 of theirs: a reduced
    angle of up to pi rounded to 2^-24 of itself, a function value and its scaling of a few steps each."""
    tol = torch.finfo(dtype).eps / 2 * want.abs() * (1 + 2.0 ** -10) + 2.0 ** -21 * size + (2.0 ** -25 if dtype == torch.float16 else 1e-39)
    assert ((got.cpu().double() - want).abs() <= tol).all()


class Case:
    def __init__(self, new, past, hq=8, hkv=2, dtype=torch.bfloat16, page=16, order="heads", rotary=128, interleaved=False, scale=1.0, base=1e4, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.hq, self.hkv, self.dtype, self.page, self.scale, self.interleaved = hq, hkv, dtype, page, scale, interleaved
        self.new, self.past, B = new, past, len(new)
        self.off = [sum(new[:b]) for b in range(B + 1)]
        self.total = self.off[-1]
        first = [p // page for p in past]                                     # (old positions share one page that nothing writes)
        need = [-(-(p + n) // page) - f for p, n, f in zip(past, new, first)]
        self.n_pages = sum(need) + 2
        ids = torch.randperm(self.n_pages, generator=g).int()
        self.table = torch.full((B, max(f + k for f, k in zip(first, need)) + 1), -1, dtype=torch.int32)
        at = 1
        for b in range(B):
            self.table[b, :first[b]] = ids[0]
            self.table[b, first[b]:first[b] + need[b]] = ids[at:at + need[b]]
            at += need[b]
        self.qkv = torch.randn((self.total + 2, hq + 2 * hkv, 128), generator=g).to(dtype)
        self.rows = torch.randn((2, hkv, self.n_pages, page, 128), generator=g).to(dtype)
        self.inv_freq = (base ** -(torch.arange(rotary // 2, dtype=torch.float64) / (rotary // 2))).float() if rotary else None
        self.order = order
        self.layer = rtp.layer_desc(hq, hkv, [], 4, 64, kv_dtype=rtp.RTP_DTYPE_FP16 if dtype == torch.float16 else rtp.RTP_DTYPE_BF16)

    def call(self, in_place=False, keys_only=False):
        d = "cuda"
        qkv = self.qkv.to(d)
        q, k, v = qkv[:, :self.hq], qkv[:, self.hq:self.hq + self.hkv], qkv[:, self.hq + self.hkv:]
        K, V = pools(self.rows.to(d), self.order)
        cache = rtp.kv_cache(K, V, self.table.to(d))
        chunk = rtp.chunk_desc(torch.tensor(self.off, dtype=torch.int32, device=d),
                               torch.tensor([n + p for n, p in zip(self.new, self.past)], dtype=torch.int32, device=d), self.total,
                               max(max(self.new), 1), max(max(n + p for n, p in zip(self.new, self.past)), 1))
        rope = None if self.inv_freq is None else rtp.rope_desc(self.inv_freq.to(d), self.interleaved, 0.0 if self.scale == 1.0 else self.scale)
        out = q if in_place else torch.full((self.total + 2, self.hq, 128), 7.0, dtype=self.dtype, device=d)
        rtp.rtp_kv_append(self.layer, cache, chunk, rope, None if keys_only else q, q.stride(0), k, k.stride(0), v, v.stride(0),
                          None if keys_only else out, out.stride(0))
        torch.cuda.synchronize()
        if in_place:
            assert torch.equal(qkv[:, self.hq:].cpu(), self.qkv[:, self.hq:])
            assert torch.equal(out[self.total:].cpu(), self.qkv[self.total:, :self.hq])
        else:
            assert torch.equal(qkv.cpu(), self.qkv) and (out[self.total:] == 7.0).all()
        return out[:self.total], K, V

    def check(self, out, K, V):
        pos = torch.cat([torch.arange(p, p + n) for n, p in zip(self.new, self.past)] or [torch.zeros(0)]).long()
        seq = torch.repeat_interleave(torch.arange(len(self.new)), torch.tensor(self.new))
        x = self.qkv[:self.total]
        k, size = x[:, self.hq:self.hq + self.hkv].double(), torch.zeros(())
        if self.inv_freq is not None:
            k, size = turned(x[:, self.hq:self.hq + self.hkv], pos, self.inv_freq, self.interleaved, self.scale)
        if out is not None and self.inv_freq is not None:
            near(out, *turned(x[:, :self.hq], pos, self.inv_freq, self.interleaved, self.scale), self.dtype)
        elif out is not None:
            assert torch.equal(out.cpu(), x[:, :self.hq])
        at, slot = self.table[seq, pos // self.page].long(), pos % self.page
        K, V = K.cpu(), V.cpu()
        near(K[:, at, slot], k.transpose(0, 1), size.transpose(0, 1) if size.dim() else size, self.dtype)
        assert torch.equal(V[:, at, slot], x[:, self.hq + self.hkv:].transpose(0, 1))
        rest = torch.ones((self.n_pages, self.page), dtype=torch.bool)
        rest[at, slot] = False
        assert torch.equal(K[:, rest], self.rows[0][:, rest]) and torch.equal(V[:, rest], self.rows[1][:, rest])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rotary,interleaved", [(128, False), (128, True), (64, False), (32, True), (16, False), (48, True), (112, False), (0, False)])
def test_rotations(rotary, interleaved, dtype):
    c = Case([5, 0, 17, 1], [0, 40, 100, 31], dtype=DT[dtype], rotary=rotary, interleaved=interleaved, seed=rotary)
    c.check(*c.call())


@pytest.mark.parametrize("order", ["heads", "pages", "tokens", "interleaved"])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_pages_and_layouts(order, page):
    c = Case([33, 2, 70], [7, 15, 500], page=page, order=order, seed=page)
    c.check(*c.call())


@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 4), (8, 1), (12, 3), (64, 8), (128, 128)])
def test_heads(hq, hkv):
    c = Case([3, 1, 9], [5, 77, 0], hq=hq, hkv=hkv, seed=hq)
    c.check(*c.call())


def test_far_positions_are_as_exact_as_the_first():
    c = Case([3, 2, 1], [(1 << 20) - 1, 262143, (1 << 26) + 12345], page=1 << 20, hkv=1, base=1e6, scale=1.25, seed=4)
    c.check(*c.call())


def test_many_tokens_and_sequences():
    c = Case([(5 * i) % 11 for i in range(300)], [(7 * i) % 60 for i in range(300)], hq=4, hkv=1, seed=5)     # more than 64 sequences
    c.check(*c.call())
    c = Case([1500], [3], hq=4, hkv=1, seed=6)                                # a wave per token
    c.check(*c.call())


def test_queries_in_place_and_keys_alone():
    c = Case([30, 1], [3, 90], rotary=64, seed=7)
    c.check(*c.call(in_place=True))
    _, K, V = c.call(keys_only=True)
    c.check(None, K, V)


def test_tokens_without_a_page_are_dropped():
    c = Case([20, 4], [10, 0], seed=8)
    want = c.call()[0]
    page = int(c.table[0, 1])
    c.table[0, 1], c.table[1, 0] = -1, c.n_pages
    out, K, V = c.call()
    assert torch.equal(out, want)                                              # the queries' rotation does not go by pages
    changed = (K.cpu() != c.rows[0]).flatten(2).any(2).any(0)
    named = torch.zeros(c.n_pages, dtype=torch.bool)
    named[c.table[0, 0]] = True
    assert torch.equal(changed, named) and not changed[page]


def test_tokens_before_the_first_position_are_passed_over():
    c = Case([6], [0], seed=9)
    d = "cuda"
    qkv = c.qkv.to(d)
    K, V = pools(c.rows.to(d), "heads")
    chunk = rtp.chunk_desc(torch.tensor([0, 6], dtype=torch.int32, device=d), torch.tensor([4], dtype=torch.int32, device=d), 6, 6, 16)
    out = torch.full((6, c.hq, 128), 7.0, dtype=c.dtype, device=d)
    rtp.rtp_kv_append(c.layer, rtp.kv_cache(K, V, c.table.to(d)), chunk, rtp.rope_desc(c.inv_freq.to(d)), qkv[:, :8], qkv.stride(0), qkv[:, 8:10],
                      qkv.stride(0), qkv[:, 10:], qkv.stride(0), out, out.stride(0))
    torch.cuda.synchronize()
    assert (out[:2] == 7.0).all() and torch.equal(V[:, int(c.table[0, 0]), :4].cpu(), c.qkv[2:6, 10:].transpose(0, 1))
