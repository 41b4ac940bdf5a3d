"""A 4-bit cache drawn on the host, in torch tensors on the GPU, and the bounds that its attention is held to."""
from __future__ import annotations

import numpy as np
import torch

from oracle import kv4_oracle as k4
from paper_2605_16928_amd import rtp
from gpu_util import DEV, i32

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
EPS = {"bf16": 2.0 ** -7, "fp16": 2.0 ** -10}


class Cache:
    """Random rows for `lens` tokens per sequence in shuffled pages.  Everything that holds no token is poison: scale bytes of 255
    (not a number) and codes of all ones; table entries behind the sequences point outside the pool."""

    def __init__(self, rng, n_kv_heads, lens, page_size, page_major=False, spread=1.0, spare=3):
        self.H, self.ps, self.lens = n_kv_heads, page_size, list(lens)
        need = [-(-n // page_size) for n in lens]
        self.P = sum(need) + spare
        ids = rng.permutation(self.P)
        self.table = np.full((len(lens), max(need + [1]) + 1), -1, dtype=np.int32)
        self.table[:, -1] = self.P + 5
        self.codes = np.full((n_kv_heads, self.P, page_size, 128), 0xff, dtype=np.uint8)
        scales = np.full((n_kv_heads, self.P, page_size // 4, 2, 4, 4), 0xff, dtype=np.uint8)
        at = 0
        for b, n in enumerate(lens):
            self.table[b, :need[b]] = ids[at:at + need[b]]
            at += need[b]
            t = np.arange(n)
            page, slot = self.table[b, t // page_size], t % page_size
            for w in (0, 1):
                c, s = k4.quantise(rng.standard_normal((n_kv_heads, n, 128)) * spread * np.exp(0.5 * rng.standard_normal((n_kv_heads, 1, 128))))
                self.codes[:, page, slot, 64 * w:64 * w + 64] = c[..., 0::2] | (c[..., 1::2] << 4)
                scales[:, page, slot // 4, w, :, slot % 4] = s.transpose(1, 0, 2)     # (indexed dims come first)
        self.scales = scales.reshape(n_kv_heads, self.P, page_size * 8)
        self.upload(page_major)

    def upload(self, page_major=False):
        def put(x):
            t = torch.from_numpy(x)
            return t.transpose(0, 1).contiguous().to(DEV).transpose(0, 1) if page_major else t.to(DEV)
        self.codes_d, self.scales_d, self.table_d = put(self.codes), put(self.scales), torch.from_numpy(self.table).to(DEV)
        self.desc = rtp.kv4_cache(self.codes_d, self.scales_d, self.table_d)

    def rows(self, b, kvh, pos):
        return k4.rows_of(self.codes[kvh], self.scales[kvh], self.table[b], self.ps, pos)


def queries(rng, B, Hq, dtype, size=1.0):
    q = torch.from_numpy(rng.standard_normal((B, Hq, 128)) * size).to(TYPES[dtype])
    return q.to(DEV), q.double().numpy()


def check_row(out, lse, q, k, v, dtype, scale=128.0 ** -0.5, what=""):
    """One head's output and log-sum against 64 bits.  Counted: the output's rounding (half a step); p as a sum of two bf16 values
    (2^-16 of p); sums of n terms in fp32 (n 2^-24); a logit's 128 products (exact ones) summed in fp32 and scaled, which moves p by
    twice that relatively, in numerator and denominator; the exponential (2^-22)."""
    ref, ref_lse, wabs, mag = k4.attend(q, k, v, scale)
    n = len(k)
    if n == 0:
        assert (out == 0).all() and lse == -np.inf, f"{what}: an empty row is not zeros"
        return
    delta = 132 * 2.0 ** -24 * mag
    p_rel = 2.0 ** -16 + 2 * (2 * delta + n * 2.0 ** -24 + 2.0 ** -22)
    tol = EPS[dtype] / 2 * np.abs(ref) + p_rel * wabs * (1 + EPS[dtype]) + 2.0 ** -24      # (fp16 below its normal range: half a step)
    err = np.abs(out - ref)
    assert (err <= tol).all(), f"{what}: out off by {(err - tol).max()} beyond its bound (error {err.max()}, n = {n})"
    lse_tol = delta + (n + 8) * 2.0 ** -24 + 2.0 ** -21 * (1 + abs(ref_lse))
    assert abs(lse - ref_lse) <= lse_tol, f"{what}: lse {lse} against {ref_lse}, bound {lse_tol}"
