"""fp16 prefill whose queries keep thousands of keys, with one that they do not keep far above them in a tile that they read."""
import numpy as np
import pytest
import torch

from gpu_util import DEV
from paper_2605_16928_amd import workloads as wl
from paper_2605_16928_amd.pipeline import PrefillRun

pytestmark = pytest.mark.gpu


def test_a_strong_key_that_is_not_kept():
    """16 retrieval heads, 4096 queries: 256 query tiles, whose keys are not cut.  Nine keys of ten have one index score, the others a lower one and among them
    the first tile's best, 13 above all others: the reference of every exponential.  Values of +1 and -1 by the direction of every rounding to
    fp16's steps there, which nothing averages.  Bound: half a step of every probability, 2^-11 of the sum for those below 2^-14, the output's own rounding,
    sums of n terms and a logit's products (twice their size)."""
    T, past = 4096, 8192
    w = wl.small_prefill("cpu", chunk_start=past, T=T, p=0.85, seed=51, n_q_heads=16, n_kv_heads=2, ret_heads=tuple(range(16)), kv_dtype="fp16")
    g = torch.Generator().manual_seed(52)
    u = torch.randn((2, 128), generator=g).half().float()
    w.q[:] = u.repeat_interleave(8, 0).half()
    w.K[:] = (0.05 * torch.randn(w.K.shape, generator=g)).half()
    w.K[:, 5] = (12.8 * 128 ** 0.5 * u / u.square().sum(1, keepdim=True)).half()
    kept = torch.rand(w.N, generator=g) < 0.9
    kept[5] = False
    w.qI.zero_()
    w.qI[..., 0] = 1.0
    w.kI.zero_()
    w.kI[..., 0] = kept.to(w.kI.dtype)
    x = torch.einsum("hnd,hd->hn", w.K.double(), u.double()) * 128.0 ** -0.5
    p = torch.exp(x - x[:, 5:6]) * 2.0 ** 24
    w.V[:] = torch.where(torch.round(p) > p, 1.0, -1.0)[..., None].half()
    run = PrefillRun(w.to(DEV))
    run.sparse_prefill()
    torch.cuda.synchronize()
    out, lse = run.out.double().cpu(), run.lse.cpu()
    for t in (0, 1, 255, 256, 2000, 4095):
        for h in (0, 7, 8, 15):
            see = kept[:past + t + 1].nonzero().flatten()
            assert int(run.count[h, t]) == len(see)
            z = torch.logsumexp(x[h // 8, see], 0)
            prob, v = torch.exp(x[h // 8, see] - z), w.V[h // 8, see, 0].double().cpu()
            o = (prob * v).sum()
            size = float((w.K[h // 8].double().cpu()[see].abs() @ u[h // 8].double().abs()).max() * 128.0 ** -0.5)
            e_x, e_sum, spread = 128 * 2.0 ** -24 * size + 2.0 ** -21, (len(see) + 64) * 2.0 ** -24, float((prob * (v - o).abs()).sum())
            tol = 2.0 ** -11 * abs(float(o)) + (2.0 ** -11 + 2 * e_x + 2.0 ** -11) * spread + 2 * e_sum
            assert float((out[t, h] - o).abs().max()) <= tol, f"query {t} head {h}: off by {float((out[t, h] - o).abs().max())}, {tol} allowed"
            assert abs(float(lse[t, h]) - float(z)) <= 2.0 ** -10
